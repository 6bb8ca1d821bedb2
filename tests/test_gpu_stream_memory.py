"""Calls on a stream that is not the current one, while the current one still works on memory that it has freed: what the calls make for
themselves is not taken from there."""
import pytest
import torch

import paper_2410_20305_amd as ps

pytestmark = pytest.mark.gpu

T, H, N, V = 700, 256, 520, 300


def _data():
    g = torch.Generator(device="cuda").manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    return dict(X=rn(T, H), W=rn(N, H), Wd=rn(H, N), w=rn(H), dY=rn(T, H), ids=torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32),
                qkv=[rn(T, 2, 128) for _ in range(3)])


def _all(d, meta, stream):
    ffn = (d["X"], d["W"], d["W"], d["Wd"])
    Y, kept = ps.psattn_ffn_fwd(*ffn, stream=stream)
    out = [Y, *kept, ps.psattn_ffn_fwd(*ffn, keep=False, stream=stream)[0], *ps.psattn_ffn_bwd(*ffn, kept, d["dY"], stream=stream)]
    N_, S, mean, rstd = ps.psattn_layernorm_fwd(d["X"], d["w"], d["w"], residual=d["dY"], stream=stream)
    out += [N_, S, mean, rstd, *ps.psattn_layernorm_bwd(S, d["w"], mean, rstd, d["dY"], stream=stream)]
    out += [ps.psattn_embed_fwd(d["ids"], d["W"][:V], stream=stream), ps.psattn_embed_bwd(d["ids"], d["X"], V, stream=stream)]
    O, LSE = ps.psattn_fwd(meta, *d["qkv"], 0.1, stream=stream)
    return out + [O, LSE, *ps.psattn_bwd(meta, *d["qkv"], O, d["qkv"][0], LSE, 0.1, stream=stream)]


@pytest.mark.parametrize("as_handle", [False, True])
def test_memory_that_the_current_stream_has_freed(as_handle):
    d = _data()
    meta = ps.psattn_build_meta([0], [T - 30], [10], [20], T)
    want = [t.clone() for t in _all(d, meta, None)]
    side = torch.cuda.Stream()
    for turn in range(3):
        side.wait_stream(torch.cuda.current_stream())
        # blocks of the sizes that the calls take, freed with work on them still queued
        used = [torch.empty_like(t) for t in want]
        spans = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in used]
        for _ in range(20):
            for t in used:
                t.fill_(float("nan"))
        del t, used
        got = _all(d, meta, side.cuda_stream if as_handle else side)
        for t in got:
            at = t.data_ptr()
            assert not any(lo < at + t.numel() * t.element_size() and at < hi for lo, hi in spans), turn
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), turn
        del t, got  # the next turn's calls may have this memory, behind the comparisons above
    torch.cuda.synchronize()
    meta.free()


def test_captured_on_a_stream_that_forks_from_the_capture():
    """Calls on a second stream of a capture, which joins again: every replay as the eager calls, with eager ones between."""
    d = _data()
    meta = ps.psattn_build_meta([0], [T - 30], [10], [20], T)
    _all(d, meta, None)
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        side.wait_stream(torch.cuda.current_stream())
        out = _all(d, meta, side)
        torch.cuda.current_stream().wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for turn in range(3):
        d["X"].copy_(torch.randn(T, H, generator=gen, device="cuda"))
        d["dY"].copy_(torch.randn(T, H, generator=gen, device="cuda"))
        want = [t.clone() for t in _all(d, meta, None)]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), turn
    meta.free()

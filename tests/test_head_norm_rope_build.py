"""Static checks on the compiled kernels of the vocabulary head, the gated norms and rotary positions (CPU only: hipcc cross-compiles gfx950)."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_build import _asm, _kernels, _no_spills, _outside_asm

SOURCES = ["psattn_head.hip", "psattn_head_bf16.hip", "psattn_head_bf16_any.hip", "psattn_head_f32.hip", "psattn_head_f32_whole.hip", "psattn_gatednorm.hip", "psattn_rope_apply.hip"]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    """The sources' assembly, compiled side by side."""
    at = tmp_path_factory.mktemp("asm")
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(lambda src: _asm(at, src), SOURCES)))


def _all(text):
    return _kernels(text, "psattn_", len(re.findall(r"\.amdhsa_kernel \S*psattn_", text)))


@pytest.mark.parametrize("src", SOURCES)
def test_nothing_is_kept_in_memory(asm, src):
    kernels = _all(asm[src])
    assert kernels
    for name, _, meta in kernels:
        assert int(meta["vgpr_spill_count"]) == 0 and int(meta["private_segment_fixed_size"]) == 0, name
        assert int(meta["group_segment_fixed_size"]) <= 160 * 1024, name


@pytest.mark.parametrize("src", ["psattn_head_bf16.hip", "psattn_head_f32_whole.hip"])
def test_copies_alone_use_m0(asm, src):
    """Their asynchronous copies write M0 from inline assembly that cannot declare it: nothing else may name it."""
    for name, body, meta in _all(asm[src]):
        if "global_load_lds_dwordx4" not in body:
            continue
        offenders = [c for c in _outside_asm(body) if re.search(r"\bm0\b", c)]
        assert not offenders, (name, offenders[:5])


def test_vector_loads_of_the_loops_are_copies(asm):
    """The compiler's waits count no copies: a load of its own between two MFMAs of a loop over k would wait for all of them."""
    for src in ("psattn_head_bf16.hip", "psattn_head_f32_whole.hip"):
        for name, body, _ in _all(asm[src]):
            loop = [b for b in re.split(r"\n\.LBB\w+:", body) if "v_mfma" in b and "global_load_lds_dwordx4" in b]
            assert loop, name
            for b in loop:
                assert not re.search(r"\bglobal_load_(?!lds)", b), name


def test_packed_fp32_is_off(asm):
    for src in SOURCES:
        assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm[src]), src

"""Static checks on the compiled kernels of the feed-forward block (CPU only: hipcc cross-compiles gfx950).  Their asynchronous copies write
M0 from inline assembly that cannot declare it: nothing else may name it.  A spill would stand in the loop over k."""
import re

from test_kernel_build import _asm, _kernels, _no_spills, _outside_asm


def test_copies_alone_use_m0_and_nothing_spills(tmp_path):
    kernels = _kernels(_asm(tmp_path, "psattn_ffn_bf16.hip"), "psattn_ffn_tiles", 26)
    for name, body, meta in kernels:
        offenders = [c for c in _outside_asm(body) if re.search(r"\bm0\b", c)]
        assert not offenders, (name, offenders[:5])
        _no_spills(name, meta)
        assert "global_load_lds_dwordx4" in body, name
        assert int(meta["group_segment_fixed_size"]) <= 160 * 1024, name


def test_vector_loads_of_the_loop_are_copies(tmp_path):
    """The compiler's waits count no copies: a load of its own between two MFMAs of the loop over k would wait for all of them."""
    for name, body, _ in _kernels(_asm(tmp_path, "psattn_ffn_bf16.hip"), "psattn_ffn_tiles", 26):
        blocks = re.split(r"\n\.LBB\w+:", body)
        loop = [b for b in blocks if "v_mfma" in b and "global_load_lds_dwordx4" in b]
        assert loop, name
        for b in loop:
            assert not re.search(r"\bglobal_load_(?!lds)", b), name


def test_layer_norm_and_embedding_do_not_spill(tmp_path):
    for src, kernel in (("psattn_embed.hip", "psattn_embed"), ("psattn_layernorm.hip", "psattn_ln_fwd")):
        text = _asm(tmp_path, src)
        for name, _, meta in _kernels(text, kernel, len([n for n in re.findall(r"\.amdhsa_kernel (\S+)", text) if kernel in n])):
            assert int(meta["vgpr_spill_count"]) == 0, name

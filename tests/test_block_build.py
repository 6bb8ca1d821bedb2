"""Static checks on the compiled kernels of what stands beside attention (CPU only: hipcc cross-compiles gfx950): none keeps a
register in memory, where a loop would fetch it each time."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_build import _asm, _kernels


SOURCES = ["psattn_ffn_bf16_any.hip", "psattn_ffn_f32.hip", "psattn_layernorm.hip"]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    """The sources' assembly, compiled side by side."""
    at = tmp_path_factory.mktemp("asm")
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        return dict(zip(SOURCES, pool.map(lambda src: _asm(at, src), SOURCES)))


def _nothing_in_memory(kernels):
    for name, _, meta in kernels:
        assert int(meta["vgpr_spill_count"]) == 0 and int(meta["private_segment_fixed_size"]) == 0, name


@pytest.mark.parametrize("src", SOURCES[:2])
def test_products_of_any_alignment_and_of_fp32(asm, src):
    _nothing_in_memory(_kernels(asm[src], "psattn_ffn_tiles", 26))


def test_layer_norm_backward(asm):
    text = asm["psattn_layernorm.hip"]
    _nothing_in_memory(_kernels(text, "psattn_ln_bwd", len(re.findall(r"\.amdhsa_kernel \S*psattn_ln_bwd", text))))


def test_no_kernel_that_no_call_reaches(asm):
    """The layer norm's rows of 513 to 768 groups have a backward of their own where they are whole groups, and no other."""
    names = [name for name, _, _ in _kernels(asm["psattn_layernorm.hip"], "psattn_ln_bwd", 38)]
    assert not any("Li256ELi3ELb0E" in name for name in names) and sum("Li256ELi3ELb1E" in name for name in names) == 2

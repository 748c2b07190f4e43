"""Scratch memory of the attention kernels of 128 query rows and more of 128 dims, whose sums
and operands take all 256 registers of two waves per SIMD and a few more: bytes a lane at most,
as compiled now (all outside the loops over tiles)."""
import pytest

from test_kernel_resources import _symbols
from test_mx_resources import asm  # noqa: F401  (the sources' assembly, compiled once)

# (format, new rows, shape: 2 of 128 query rows, 3 of 256, bytes)
SPILLS = [(0, 1, 2, 148), (0, 1, 3, 20)]
for fmt in (1, 2):
    SPILLS += [(fmt, 0, 2, 44), (fmt, 1, 2, 144), (fmt, 0, 3, 44), (fmt, 1, 3, 68)]


@pytest.mark.parametrize("fmt,tree,shape,most", SPILLS)
def test_spills_are_no_more(asm, fmt, tree, shape, most):  # noqa: F811
    src = f"attend_{['bf16', 'mxfp8', 'mxfp4'][fmt]}.hip"
    prefix = f"_ZN6certkv13attend_kernelILi{fmt}ELi128ELi{shape}ELb{tree}E"
    scratch = _symbols(asm[src], prefix, "private_seg_size")
    vgprs = _symbols(asm[src], prefix, "num_vgpr")
    assert scratch, f"no kernel {prefix} in {src}"
    for name, n in scratch.items():
        assert n <= most, f"{name} spills {n} bytes per lane (at most {most})"
        assert vgprs[name] <= 256, f"{name} uses {vgprs[name]} VGPRs"

"""Register budgets of the microscaled cache's and the attention kernels, as
tests/test_kernel_resources.py checks those of the pass: no spilling to scratch memory and
no more VGPRs than the waves per SIMD that their launches count on leave."""
import concurrent.futures
import os
import shutil
import tempfile

import pytest

from paper_2608_21541_amd import build as B
from test_kernel_resources import _device_asm, _symbols

# (source, kernel symbol prefix, largest VGPR count).  Not listed: 128 query rows and more
# of 128 dims, whose sums and operands take all 256 registers of two waves per SIMD and a
# few more.
KERNELS = [("cache.hip", "_ZN6certkv17compact_mx_kernelI", 96),
           ("cache.hip", "_ZN6certkv14read_mx_kernelI", 32),
           ("attend.hip", "_ZN6certkv18attend_join_kernelI", 64)]
for fmt, name in ((0, "bf16"), (1, "mxfp8"), (2, "mxfp4")):
    for tree in ((1,) if fmt == 0 else (0, 1)):
        for d, shape, most in ((128, 0, 256), (128, 1, 256), (64, 0, 168),
                               (64, 1, 256), (64, 2, 256), (64, 3, 256)):
            KERNELS.append((f"attend_{name}.hip",
                            f"_ZN6certkv13attend_kernelILi{fmt}ELi{d}ELi{shape}ELb{tree}E", most))


@pytest.fixture(scope="module")
def asm():
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    srcs = sorted({s for s, _, _ in KERNELS})
    with tempfile.TemporaryDirectory() as d:
        with concurrent.futures.ThreadPoolExecutor(min(len(srcs), 8)) as ex:
            return dict(zip(srcs, ex.map(lambda s: _device_asm(s, d), srcs)))


@pytest.mark.parametrize("src,prefix,vmax", KERNELS, ids=[k[1][10:] for k in KERNELS])
def test_kernels_do_not_spill(asm, src, prefix, vmax):
    scratch = _symbols(asm[src], prefix, "private_seg_size")
    vgprs = _symbols(asm[src], prefix, "num_vgpr")
    assert scratch, f"no kernel {prefix} in {src}"
    for name, n in scratch.items():
        assert n == 0, f"{name} spills {n} bytes per lane"
        assert vgprs[name] <= vmax, f"{name} uses {vgprs[name]} VGPRs (budget {vmax})"

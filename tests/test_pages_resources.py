"""Register budgets of the paged cache's kernels, as tests/test_kernel_resources.py checks those of
the pass: no scratch memory, and no more VGPRs than the waves per SIMD that their launches count on
leave."""
import concurrent.futures
import os
import shutil
import tempfile

import pytest

from paper_2608_21541_amd import build as B
from test_kernel_resources import _device_asm, _symbols

# (source, kernel symbol prefix, largest VGPR count, scratch bytes a lane at most)
KERNELS = [("pages.hip", "_ZN6certkv18page_resize_kernelI", 128, 0),
           ("pages.hip", "_ZN6certkv18page_blocks_kernelE", 64, 0),
           ("pages.hip", "_ZN6certkv17page_slots_kernelE", 64, 0),
           ("pages.hip", "_ZN6certkv17page_write_kernelI", 64, 0),
           ("pages.hip", "_ZN6certkv17page_adopt_kernelI", 64, 0),
           ("pages.hip", "_ZN6certkv16page_read_kernelI", 64, 0),
           ("paged.hip", "_ZN6certkv17paged_join_kernelI", 128, 0)]
for fmt, name in ((0, "bf16"), (1, "mxfp8"), (2, "mxfp4")):
    for d in (64, 128):
        for qt in (1, 2):
            for mode in (0, 1, 2):  # pieces, whole units, four heads
                three = mode != 1 and qt == 1 and (d == 64 or fmt == 2)
                # (32 query rows of 128 dims: sums and operands take all 256 registers of two waves
                # per SIMD; what does not fit lies outside the loop over tiles)
                spill = {(0, 1): 20, (1, 0): 16, (1, 2): 12}.get((fmt, mode), 0)
                KERNELS.append((f"paged_{name}.hip",
                                f"_ZN6certkv12paged_kernelILi{fmt}ELi{d}ELi{qt}ELi{mode}E",
                                168 if three else 256, spill if d == 128 and qt == 2 else 0))


@pytest.fixture(scope="module")
def asm():
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    srcs = sorted({k[0] for k in KERNELS})
    with tempfile.TemporaryDirectory() as d:
        with concurrent.futures.ThreadPoolExecutor(min(len(srcs), 8)) as ex:
            return dict(zip(srcs, ex.map(lambda s: _device_asm(s, d), srcs)))


@pytest.mark.parametrize("src,prefix,vmax,spill", KERNELS, ids=[k[1][10:] for k in KERNELS])
def test_registers(asm, src, prefix, vmax, spill):
    scratch = _symbols(asm[src], prefix, "private_seg_size")
    vgprs = _symbols(asm[src], prefix, "num_vgpr")
    assert scratch, f"no kernel {prefix} in {src}"
    for name, n in scratch.items():
        assert n <= spill, f"{name} spills {n} bytes per lane (at most {spill})"
        assert vgprs[name] <= vmax, f"{name} uses {vgprs[name]} VGPRs (budget {vmax})"

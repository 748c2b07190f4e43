"""A cache written from fp32 rows, which new bf16 queries attend under the same problem of bf16."""
import dataclasses

import pytest
import torch

import paper_2608_21541_amd as ck
from test_gpu_mx import check, dev, gen, kept_sets, queries, tree_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_cache_written_from_fp32_is_attended(fmt, d):
    L, H, G, lens, tq, tn, g = 2, 3, 2, [500, 77], 5, 9, gen(d)
    spec = ck.ProblemSpec(L, H, G, d, 1, lens, torch.float32)
    k, v = (torch.randn((L, sum(lens), H, d), generator=g).to(dev()) for _ in range(2))
    off, idx = (x.to(dev()) for x in kept_sets(lens, L, H, g))
    star = [torch.randn((spec.units, d), generator=g).to(dev()) for _ in range(2)]
    cache = ck.compact_mx(spec, k, v, off, idx, *star, fmt)
    kk, vv = (t.cpu().double() for t in ck.read_mx(cache))
    q, qd = queries(L, 2, tq, H * G, d, g)
    with pytest.raises(ck.CertKVError):
        ck.decode_mx(spec, qd, cache, tq)
    spec = dataclasses.replace(spec, dtype=torch.bfloat16)
    out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
    check(spec, q, cache.offsets.cpu(), kk, vv, tq, out, lse)
    kn, knd = queries(L, 2, tn, H, d, g)
    mask = tree_mask(2, tq, tn, g)
    out, lse = ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()), with_lse=True)
    check(spec, q, cache.offsets.cpu(), kk, vv, tq, out, lse, kn, kn, mask)

"""Heads that keep every token: a segment of n_b rows and the slot row is attended whole, by
every decode entry point and under every bound that holds it."""
import pytest
import torch

import paper_2608_21541_amd as ck
from test_gpu_mx import check, dev, gen, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def full_cache(fmt, lens, H, d, g, slot=True):
    """(spec, cache, fp64 keys and values, offsets) of a problem whose first head keeps every
    token; the slot values are 100 times the others, so that a lost slot row shows."""
    T, status = sum(lens), torch.zeros(1, dtype=torch.int32, device=dev())
    spec = ck.ProblemSpec(1, H, 2, d, 1, lens, slot=slot, status=status)
    k, v = (torch.randn((1, T, H, d), generator=g).bfloat16().to(dev()) for _ in range(2))
    keep = [n if h == 0 else max(1, n // (2 + h)) for n in lens for h in range(H)]
    off = torch.tensor([0] + keep).cumsum(0).to(dev())
    idx = torch.cat([torch.arange(n) for n in keep]).int().to(dev())
    star = torch.randn((len(lens) * H, d), generator=g).bfloat16().float().to(dev())
    if fmt == "bf16":
        kp, vp, _, po = ck.compact(spec, k, v, off, idx, star, 100 * star)
        return spec, (kp, vp, po), kp.cpu().double(), vp.cpu().double(), po.cpu()
    cache = ck.compact_mx(spec, k, v, off, idx, star, 100 * star, fmt)
    kk, vv = ck.read_mx(cache)
    return spec, cache, kk.cpu().double(), vv.cpu().double(), cache.offsets.cpu()


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("n", [1, 33, 4096, 8192])
@pytest.mark.parametrize("tq", [1, 20])
def test_the_slot_row_of_a_head_that_keeps_all(fmt, n, tq):
    H, d, g = 2, 128, gen(n + tq)
    lens = [n, max(1, n - 5)]
    spec, cache, k, v, off = full_cache(fmt, lens, H, d, g)
    assert int(off[1] - off[0]) == n + 1
    q, qd = queries(1, 2, tq, 2 * H, d, g)
    kn, knd = queries(1, 2, tq, H, d, g)
    mask = torch.tril(torch.ones((tq, tq), dtype=torch.bool)).expand(2, tq, tq).contiguous()
    for max_rows in (0, n + 1, n + 1000):
        if fmt != "bf16":
            out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True, max_rows=max_rows)
            check(spec, q, off, k, v, tq, out, lse)
        out, lse = ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()), with_lse=True,
                                  max_rows=max_rows)
        check(spec, q, off, k, v, tq, out, lse, kn, kn, mask)
        assert int(spec.status.item()) == ck.CERTKV_OK
    if n > 1:  # a shorter bound is reported
        ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()), max_rows=n)
        assert int(spec.status.item()) == ck.CERTKV_ERANGE


@pytest.mark.parametrize("n", [33, 4096, 8192])
def test_decode_over_bf16_rows_too(n):
    H, d, tq, g = 2, 128, 3, gen(n)
    spec, cache, k, v, off = full_cache("bf16", [n, n - 5], H, d, g)
    q, qd = queries(1, 2, tq, 2 * H, d, g)
    sees_none = torch.zeros((2, tq, 1), dtype=torch.bool, device=dev())
    new = torch.zeros((1, 2, H, d), dtype=torch.bfloat16, device=dev())
    want = ck.decode_tree(spec, qd, cache, tq, new, new, sees_none)
    for max_rows in (0, n + 1):
        out = ck.decode(spec, qd, *cache, tq, max_rows=max_rows)
        assert int(spec.status.item()) == ck.CERTKV_OK
        # (weights there are two bf16, each off by 2^-18 of itself at most, and sum_j p_j |v_j| is
        # under 60 |out| for these rows: 3e-4; without its slot row an output is half of itself)
        assert float((out - want).norm(dim=-1).max() / want.norm(dim=-1).max()) < 1e-3


@pytest.mark.parametrize("fmt", ["mxfp8", "bf16"])
def test_without_slots_the_bound_is_the_longest_sequence(fmt):
    H, d, tq, g = 2, 64, 2, gen(5)
    spec, cache, k, v, off = full_cache(fmt, [64], H, d, g, slot=False)
    assert int(off[1]) == 64
    q, qd = queries(1, 1, tq, 2 * H, d, g)
    kn, knd = queries(1, 1, tq, H, d, g)
    mask = torch.ones((1, tq, tq), dtype=torch.bool)
    out, lse = ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()), with_lse=True)
    check(spec, q, off, k, v, tq, out, lse, kn, kn, mask)
    assert int(spec.status.item()) == ck.CERTKV_OK

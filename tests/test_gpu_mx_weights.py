"""A weight of the attention over caches keeps all 24 bits of its fp32 value in the product
with the values: rows whose sums leave nothing else to round, so that a weight of fewer bits
shows.

64 rows; row j's value is 1 in dim j (and j + 64) alone, its key minus the first unit vector,
or zero in one row of every 32.  A query row t times the first unit vector, t = 1 .. 128, at
scale 1/64 then has scores -t/64 and 0: dim j is w / (2 + 62 w) with w = e^(-t/64), or
1 / (2 + 62 w).  What an output may be off by, relative to itself, in halved units
(u = 2^-24):
  the exponent: its constant and its product round once each, times |z| <= 2     4
  the exponential                                                                2
  the sum of the weights, all positive: 8 in a lane, 2 lanes, 4 waves, 2 tiles   15
  the product with one value of 1: its parts' sums are exact                     0, 3 allowed
  the reciprocal and its product                                                 3
27 u in all, where two bf16 parts, rounded, are off by up to 2^-18 = 64 u, and two that are
cut off by 256 u."""
import pytest
import torch

import _mx
import paper_2608_21541_amd as ck

U = 2.0 ** -24
BOUND = 27 * U
ROWS = 64


def exact(t, zero):
    """[len(t)][64] outputs in fp64 for zero-score rows `zero`."""
    w = torch.exp(-t.double() / 64)[:, None].repeat(1, ROWS)
    w[:, zero] = 1.0
    return w / w.sum(1, keepdim=True)


def parts(p, n, cut):
    """The sum of the n bf16 parts of fp32 weights p, cut off or rounded."""
    total, rest = torch.zeros_like(p, dtype=torch.float64), p.clone()
    for _ in range(n):
        h = (rest.view(torch.int32) & -65536).view(torch.float32) if cut else rest.bfloat16().float()
        total += h.double()
        rest = rest - h
    return total


def test_the_bound_tells_two_parts_from_three():
    t = torch.arange(1, 129)
    ref = exact(t, [5, 40])
    p = ref.new_tensor(0.0) + torch.exp(-t.double() / 64)[:, None].repeat(1, ROWS)
    p[:, [5, 40]] = 1.0
    p = p.float()
    total = p.double().sum(1, keepdim=True)
    for n, cut, most in ((3, True, 3 * U), (2, False, None), (2, True, None), (1, False, None)):
        err = ((parts(p, n, cut) / total - ref).abs() / ref).max()
        assert err <= most if most else err > 1.5 * BOUND, (n, cut, float(err / U))


def make(d, H, g):
    """Keys and values [H][64][d] of H heads, and each head's rows of key zero."""
    k, v = torch.zeros((H, ROWS, d)), torch.zeros((H, ROWS, d))
    zero = [[int(torch.randint(0, 32, (1,), generator=g)) + 32 * i for i in range(2)]
            for _ in range(H)]
    k[:, :, 0] = -1.0
    for h in range(H):
        k[h, zero[h]] = 0.0
        for j in range(ROWS):
            v[h, j, j::64] = 1.0
    return k, v, zero


def packed(fmt, k, v, dev):
    from test_gpu_mx import encode
    H, d = k.shape[0], k.shape[2]
    off = (torch.arange(H + 1) * ROWS).to(dev)
    k, v = k.reshape(-1, d), v.reshape(-1, d)
    if fmt == "bf16":
        return k.bfloat16().to(dev), v.bfloat16().to(dev), off
    t = []
    for x in (k, v):
        val, byte = _mx.quantise(x, fmt)
        assert torch.equal(val, x.double())
        t += [encode(val, byte, fmt).to(dev), byte.to(dev)]
    return ck.MxCache(fmt, *t, offsets=off)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("M", [16, 32, 64, 128, 256, 512])
def test_weights_keep_all_their_bits(fmt, d, M):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev, H, g = torch.device("cuda:0"), 3, torch.Generator()
    g.manual_seed(M + d)
    k, v, zero = make(d, H, g)
    spec = ck.ProblemSpec(1, H, 2, d, 1, [100], softmax_scale=1.0 / 64)
    tq = M // 2
    t = (torch.arange(M) % 128 + 1) if M >= 128 else torch.randperm(128, generator=g)[:M] + 1
    q = torch.zeros((1, tq, H, 2, d))
    q[0, ..., 0] = t.view(tq, 1, 2).float()
    q = q.view(1, tq, 2 * H, d).bfloat16().to(dev)
    none = torch.zeros((1, 1, H, d), dtype=torch.bfloat16, device=dev)
    empty = torch.zeros(H + 1, dtype=torch.int64, device=dev)
    cache = packed(fmt, k, v, dev)
    outs = [ck.decode_tree(spec, q, cache, tq, none, none,
                           torch.zeros((1, tq, 1), dtype=torch.bool, device=dev)).clone()]
    if fmt != "bf16":
        outs.append(ck.decode_mx(spec, q, cache, tq).clone())
        bare = ck.MxCache(fmt, cache.k, cache.k_scales, cache.v, cache.v_scales, empty)
    else:
        bare = (cache[0], cache[1], empty)
    new = [x.transpose(0, 1)[None].contiguous().bfloat16().to(dev) for x in (k, v)]
    outs.append(ck.decode_tree(spec, q, bare, tq, *new,
                               torch.ones((1, tq, ROWS), dtype=torch.bool, device=dev)))
    for i, out in enumerate(outs):
        got = out.cpu().double().view(tq, H, 2, d)
        for h in range(H):
            ref = exact(t, zero[h]).repeat(1, d // 64)
            err = (got[:, h].reshape(M, d) - ref).abs() / ref
            assert float(err.max()) <= BOUND, (i, h, float(err.max() / U))

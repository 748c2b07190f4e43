"""Scores far beyond those of a model: the weights are taken against the row's largest score,
so a row's softmax stays what the definition says up to the largest scores that fp32 holds."""
import math

import pytest
import torch

import _mx
import paper_2608_21541_amd as ck
from test_gpu_mx import dev, encode, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


# Key j is n_j times the first unit vector, query row m x_m 2^k_m times it, x_m of eight bits in
# [1, 2): every raw product is exact in fp32, and scores of different n_j are 2^k_m / 12 apart or
# more: a softmax of a few rows for small k_m, the mean of the largest scores' rows for large ones.
STEPS = [0, 1, 2, 3, 4, 6]
SMALL = [-4, -3, -2]


def inputs(fmt, segs, d, M, big, sign, g):
    rows = sum(segs)
    n = torch.tensor(STEPS, dtype=torch.float64)[torch.randint(0, len(STEPS), (rows,), generator=g)]
    n = n * torch.where(torch.rand(rows, generator=g) < 0.5, 1.0, -1.0) if sign == 0 else (n + 0.0) * sign
    if sign < 0:
        n = torch.where(n == 0, torch.full_like(n, -6.0), n)
    k = torch.zeros((rows, d), dtype=torch.float64)
    k[:, 0] = n
    v = torch.randn((rows, d), generator=g, dtype=torch.float64)
    exps = torch.tensor(SMALL + big)[torch.randint(0, len(SMALL + big), (M,), generator=g)]
    exps[:len(SMALL + big)] = torch.tensor(SMALL + big)[:M]
    q = torch.zeros((M, d), dtype=torch.float64)
    q[:, 0] = torch.exp2(exps.double()) * (1 + torch.randint(0, 128, (M,), generator=g) / 128)
    off = torch.tensor([0] + segs).cumsum(0)
    if fmt == "bf16":
        v = v.bfloat16().double()
        return (k.bfloat16().to(dev()), v.bfloat16().to(dev()), off.to(dev())), k, v, q, exps, off
    t = []
    for i, x in enumerate((k, v)):
        val, byte = _mx.quantise(x, fmt)
        if i == 0:
            assert torch.equal(val, x)
        else:
            v = val
        t += [encode(val, byte, fmt).to(dev()), byte.to(dev())]
    return ck.MxCache(fmt, *t, offsets=off.to(dev())), k, v, q, exps, off


def plain(q, k, v, scale):
    """(out, lse, sum_j p_j |v_j|, the largest |z|) in fp64, against each row's largest score."""
    z = (q @ k.T) * scale
    most = z.amax(1, keepdim=True)
    p = torch.exp(z - most)
    total = p.sum(1, keepdim=True)
    p = p / total
    return p @ v, (most + total.log()).squeeze(1), p @ v.abs(), z.abs().amax(1)


def compare(out, lse, q, exps, k, v, d, what, split=0.0):
    """One unit's rows.  Scores are exact but for the factor of the scale, so that the bound's
    share of their products' sums is that of the small ones alone: the large ones' weights are
    equal or nothing.  lse: beside the bound the factor's and the product's roundings (eight of
    half a unit: the scale's root and quotient, two constants, four products)."""
    o, z, size, dz = plain(q, k, v, 1.0 / math.sqrt(d))
    dz = torch.where(exps > 0, torch.zeros_like(dz), dz)
    tol, ltol = _mx.bound(size, dz, k.shape[0], d)
    out, lse = out.cpu().double(), lse.cpu().double()
    bad = ~(((out - o).abs() <= tol + split * size).all(1) &
            ((lse - z).abs() <= ltol + 2.0 ** -21 * z.abs()))
    assert not bool(bad.any()), (what, sorted(set(exps[bad].tolist())))


BIG = [16, 20, 24, 26, 28, 29, 30, 31, 32, 33, 34, 35, 36, 40, 50, 60, 80, 100, 119]


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("M", [4, 16, 40, 100, 200, 512])
@pytest.mark.parametrize("sign", [0, 1, -1])
def test_attention_over_a_cache(fmt, M, sign):
    for d, segs in ((128, [700, 33, 5000]), (64, [1, 257, 300])):
        g = gen(M + d + sign)
        H = len(segs)
        cache, k, v, q, exps, off = inputs(fmt, segs, d, M, BIG, sign, g)
        spec = ck.ProblemSpec(1, H, M if M < 100 else 4, d, 1, [8000])
        tq = M // spec.group
        # every head the same query rows
        qd = q.view(tq, 1, spec.group, d).expand(tq, H, spec.group, d).reshape(1, tq, H * spec.group, d)
        qd = qd.bfloat16().to(dev())
        head = lambda x, h: x[0].view(tq, H, spec.group, *x.shape[3:])[:, h].reshape(M, *x.shape[3:])  # noqa: E731
        if fmt != "bf16":
            out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
            for h in range(H):
                r = slice(off[h], off[h + 1])
                compare(head(out, h), head(lse, h), q, exps, k[r], v[r], d, ("mx", d, h))
        # and 40 new rows that all queries see
        tn = 40
        kn = torch.zeros((1, tn, H, d), dtype=torch.float64)
        vn = torch.randn((1, tn, H, d), generator=g).bfloat16().double()
        kn[..., 0] = torch.tensor(STEPS[1:], dtype=torch.float64)[
            torch.randint(0, len(STEPS) - 1, (1, tn, H), generator=g)] * (sign if sign else 1)
        mask = torch.ones((1, tq, tn), dtype=torch.bool, device=dev())
        out, lse = ck.decode_tree(spec, qd, cache, tq, kn.bfloat16().to(dev()),
                                  vn.bfloat16().to(dev()), mask, with_lse=True)
        for h in range(H):
            r = slice(off[h], off[h + 1])
            compare(head(out, h), head(lse, h), q, exps, torch.cat([k[r], kn[0, :, h]]),
                    torch.cat([v[r], vn[0, :, h]]), d, ("tree", d, h))


@pytest.mark.parametrize("M", [4, 64, 200, 512])
@pytest.mark.parametrize("sign", [0, 1, -1])
def test_decode_over_bf16_rows(M, sign):
    # (its weights are two bf16, which leave 2^-18 of each)
    for d, segs in ((128, [700, 33, 5000]), (64, [1, 257, 300])):
        H = len(segs)
        cache, k, v, q, exps, off = inputs("bf16", segs, d, M, BIG, sign, gen(M + d + sign))
        spec = ck.ProblemSpec(1, H, 4, d, 1, [8000])
        tq = M // 4
        qd = q.view(tq, 1, 4, d).expand(tq, H, 4, d).reshape(1, tq, H * 4, d).bfloat16().to(dev())
        out, lse = ck.decode(spec, qd, *cache, tq, with_lse=True)
        out, lse = out[0].view(tq, H, 4, d), lse[0].view(tq, H, 4)
        for h in range(H):
            r = slice(off[h], off[h + 1])
            compare(out[:, h].reshape(M, d), lse[:, h].reshape(M), q, exps, k[r], v[r], d, (d, h),
                    2.0 ** -18)

"""Plain 64-bit forms of the microscaled cache and of attention over it (CPU)."""
import math

import torch

GRID = {
    "mxfp8": [m * 2.0 ** -9 for m in range(8)] +
             [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
    "mxfp4": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0],
}
LAST_EXP = {"mxfp8": 119, "mxfp4": 125}


def quantise(x, fmt):
    """x [..., d] to (values [..., d] fp64, scale bytes [..., d/32]): the smallest power of two
    under which the block's largest magnitude is at most the largest code, the nearest codes,
    ties to the even one; a block with a non-finite value is NaN with scale byte 255."""
    x = x.double()
    grid = torch.tensor(GRID[fmt], dtype=torch.float64)
    b = x.unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    b = torch.where(bad, torch.zeros_like(b), b)
    big = b.abs().amax(-1, keepdim=True)
    e = torch.full_like(big, -100.0)
    for k in range(-99, LAST_EXP[fmt] + 1):
        e = torch.where(big > grid[-1] * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    y = b / torch.exp2(e)
    mag = y.abs().clamp(max=float(grid[-1]))
    hi = torch.searchsorted(grid, mag.contiguous()).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    dl, dh = mag - grid[lo], grid[hi] - mag
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    v = torch.where(y < 0, -grid[pick], grid[pick]) * torch.exp2(e)
    v = torch.where(bad, torch.full_like(v, math.nan), v)
    scale = torch.where(bad, torch.full_like(e, 255.0), e + 127).squeeze(-1).to(torch.uint8)
    return v.flatten(-2), scale


def decode_codes(codes, scales, fmt):
    """Values in fp64 of codes and scale bytes (CPU uint8 tensors)."""
    if fmt == "mxfp4":
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    vals = GRID[fmt] + ([math.nan] if fmt == "mxfp8" else [])
    vals = torch.tensor(vals + [-v for v in vals], dtype=torch.float64)
    x = vals[codes.long()].unflatten(-1, (-1, 32))
    s = torch.exp2(scales.double() - 127).unsqueeze(-1)
    return torch.where(scales.unsqueeze(-1) == 255, torch.full_like(x, math.nan), x * s).flatten(-2)


def attend(q, k, v, scale, seen=None):
    """(out [M][d], lse [M], size [M][d], dz [M]) in fp64 of query rows q over rows k, v; seen
    [M][rows].  size = sum_j p_j |v_j|; dz: the largest sum of |q_i k_i| scale of a visible row."""
    q, k, v = q.double(), k.double(), v.double()
    if seen is None:
        seen = torch.ones((q.shape[0], k.shape[0]), dtype=torch.bool)
    if k.shape[0] == 0:
        z = torch.zeros((q.shape[0],), dtype=torch.float64)
        return torch.zeros_like(q), z - math.inf, torch.zeros_like(q), z
    some = seen.any(0)  # rows that nobody sees hold anything
    k = torch.where(some[:, None], k, torch.zeros_like(k))
    v = torch.where(some[:, None], v, torch.zeros_like(v))
    out, lse = torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    size, dz = torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.float64)
    whole = bool(torch.isfinite(k).all() and torch.isfinite(v).all())
    if whole:
        z = torch.where(seen, (q @ k.T) * scale, torch.full(seen.shape, -math.inf, dtype=torch.float64))
        any_row = seen.any(1)
        lse = torch.logsumexp(z, 1)
        p = torch.where(any_row[:, None], torch.exp(z - lse[:, None]), torch.zeros_like(z))
        dz = torch.where(seen, q.abs() @ k.abs().T * scale, torch.zeros_like(z)).amax(1)
        return torch.nan_to_num(p @ v), lse, torch.nan_to_num(p @ v.abs()), dz
    for m in range(q.shape[0]):
        r = seen[m]
        if r.any():
            out[m], lse[m], size[m], dz[m] = (x[0] for x in attend(q[m:m + 1], k[r], v[r], scale))
    return out, lse, size, dz


def bound(size, dz, rows, d):
    """What an output element may be off by, and lse: a weight is off by its logit's error
    (fp32 sums of d products, each addition by half a unit of the running sum, plus the scale,
    the logarithm's base and the exponential: 8 more; its bf16 parts sum to it exactly), and
    the sums over the rows by half a unit for each 16 of them (of at most 16384 rows in turn),
    64 more for joining parts and the division.  Halved units are 2^-24."""
    u = 2.0 ** -24
    rel = (d + 8) * u * dz + (min(rows, 16384) / 16 + 64) * u
    return 2 * rel[:, None] * size + 1e-30, (d + 8) * u * dz + (min(rows, 16384) / 16 + 72) * u + u * 16

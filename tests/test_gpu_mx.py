"""The microscaled packed cache (certkv_compact_mx, certkv_compress_mx, certkv_read_mx) and
attention over it and over drafted tokens (certkv_decode_mx, certkv_decode_tree) against plain
64-bit forms."""
import math

import pytest
import torch

import _mx
import paper_2608_21541_amd as ck
import synth
from _parity import spec_of

pytestmark = pytest.mark.gpu
FORMATS = ["mxfp8", "mxfp4"]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


def dev():
    return torch.device("cuda:0")


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ---- writing and reading --------------------------------------------------------


def hard_rows(shape, g, dtype):
    """Normal values with whole blocks of the hard kinds: exact ties between codes at many
    scales, zeros of both signs, numbers below the smallest scale, the largest finite ones,
    one large value among tiny ones."""
    x = torch.randn(shape, generator=g, dtype=torch.float64)
    b = x.view(-1, 32)
    kind = torch.randint(0, 12, (b.shape[0],), generator=g)
    grid = torch.tensor(_mx.GRID["mxfp8"], dtype=torch.float64)
    mids = (grid[1:] + grid[:-1]) / 2
    ties = mids[torch.randint(0, len(mids), b.shape, generator=g)]
    half = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], dtype=torch.float64)
    ties4 = half[torch.randint(0, 8, b.shape, generator=g)]
    sign = torch.where(torch.rand(b.shape, generator=g) < 0.5, -1.0, 1.0).double()
    p = torch.exp2(torch.randint(-60, 60, (b.shape[0], 1), generator=g).double())
    b[kind == 1] = (ties * sign * p)[kind == 1]
    b[kind == 2] = (ties4 * sign * p)[kind == 2]
    b[kind == 3] = (0.0 * sign)[kind == 3]
    b[kind == 4] = (b * 2.0 ** -120)[kind == 4]
    b[kind == 5] = (b.sign() * 3.3895313892515355e38)[kind == 5]
    one = b * 1e-3
    one[:, 7] = 448.0
    b[kind == 6] = one[kind == 6]
    top = torch.where(torch.rand(b.shape, generator=g) < 0.2, 449.0, 6.5).double()
    b[kind == 7] = (top * sign * p)[kind == 7]
    return b.view(shape).to(dtype)


def kept_sets(lens, L, H, g, most=0.3):
    """(kept_offsets, kept_idx) of random kept sets, some of one row or none."""
    off, idx = [0], []
    for _ in range(L):
        for n in lens:
            for h in range(H):
                c = [1, 0][h] if h < 2 else int(torch.randint(1, max(2, int(most * n)), (1,), generator=g))
                idx.append(torch.randperm(n, generator=g)[:c].sort()[0])
                off.append(off[-1] + c)
    return torch.tensor(off), torch.cat(idx).int()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype,d,slot,head_major,lens", [
    (torch.bfloat16, 128, True, False, [700, 33, 1025]),
    (torch.bfloat16, 64, True, True, [700, 1, 300]),
    (torch.float32, 64, False, False, [500, 77]),
    (torch.float32, 128, True, True, [130]),
    (torch.bfloat16, 128, False, True, [40 + i for i in range(53)]),
])
def test_written_cache_is_the_definitions(fmt, dtype, d, slot, head_major, lens):
    L, H, g = 2, 4, gen(11 * d + len(lens))
    T = sum(lens)
    src = {}
    for x in "kv":
        t = hard_rows((L, H, T, d) if head_major else (L, T, H, d), g, dtype)
        src[x] = t.transpose(1, 2) if head_major else t
    off, idx = kept_sets(lens, L, H, g)
    U = L * len(lens) * H
    star = {x: hard_rows((U, d), g, torch.float32) for x in "kv"}
    spec = ck.ProblemSpec(L, H, 2, d, 1, lens, dtype, slot=slot)
    rows = int(off[-1]) + (U if slot else 0)
    cache = ck.MxCache.empty(spec, rows + 9, fmt, dev())
    for t in (cache.k, cache.k_scales, cache.v, cache.v_scales, cache.pos):
        t.fill_(0xAB - 0x80)
    to = lambda t: t.to(dev())  # noqa: E731
    gpu = {x: (to(src[x].transpose(1, 2).contiguous()).transpose(1, 2) if head_major else to(src[x]))
           for x in "kv"}
    ck.compact_mx(spec, gpu["k"], gpu["v"], to(off), to(idx), to(star["k"]), to(star["v"]), fmt,
                  cache=cache)
    got = dict(zip("kv", ck.read_mx(cache, rows=rows)))
    got32 = dict(zip("kv", ck.read_mx(cache, dtype=torch.float32, rows=rows)))
    torch.cuda.synchronize()
    want = {"k": [], "v": []}
    pos, seg = [], [0]
    for u in range(U):
        l, b, h = u // (len(lens) * H), u // H % len(lens), u % H
        i = idx[off[u]:off[u + 1]].long()
        for x in "kv":
            want[x].append(src[x][l, sum(lens[:b]) + i, h].double())
            if slot:
                want[x].append(star[x][u:u + 1].double())
        pos += i.tolist() + ([-1] if slot else [])
        seg.append(len(pos))
    assert cache.offsets.cpu().tolist() == seg
    assert cache.pos[:rows].cpu().tolist() == pos
    for x, sc in (("k", cache.k_scales), ("v", cache.v_scales)):
        val, byte = _mx.quantise(torch.cat(want[x]), fmt)
        assert torch.equal(sc[:rows].cpu(), byte)
        assert torch.equal(got[x].cpu().double(), val)
        assert torch.equal(got32[x].cpu().double(), val)
        codes = _mx.decode_codes((cache.k if x == "k" else cache.v)[:rows].cpu(), byte, fmt)
        assert torch.equal(codes, val)
    for t in (cache.k, cache.k_scales, cache.v, cache.v_scales, cache.pos):
        assert bool((t[rows:] == 0xAB - 0x80).all())  # rows behind the last one


@pytest.mark.parametrize("fmt", FORMATS)
def test_non_finite_blocks_are_nan_and_reported(fmt):
    d, n, H = 128, 60, 2
    g = gen(3)
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    spec = ck.ProblemSpec(1, H, 1, d, 1, [n], status=status)
    k, v = (torch.randn((1, n, H, d), generator=g).bfloat16() for _ in range(2))
    off = torch.tensor([0, n - 1, 2 * (n - 1)])
    idx = torch.arange(n - 1).repeat(2).int()
    star = torch.randn((H, d), generator=g)
    run = lambda: ck.compact_mx(spec, k.to(dev()), v.to(dev()), off.to(dev()),  # noqa: E731
                                idx.to(dev()), star.to(dev()), star.to(dev()), fmt)
    run()
    assert int(status.item()) == ck.CERTKV_OK
    k[0, 5, 0, 33], k[0, 6, 1, 127], v[0, 7, 0, 0] = math.nan, math.inf, -math.inf
    cache = run()
    kk, vv = (t.cpu() for t in ck.read_mx(cache))
    assert int(status.item()) == ck.CERTKV_ENONFINITE
    for t, src in ((kk, k), (vv, v)):
        rows = torch.cat([torch.cat([src[0, :n - 1, h].double(), star[h:h + 1].double()])
                          for h in range(H)])
        want, _ = _mx.quantise(rows, fmt)
        assert torch.equal(torch.isnan(t), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(t.double()), torch.nan_to_num(want))
    # attention that meets them says so; with keys alone the weights are lost too
    status.zero_()
    q = torch.randn((1, 1, H, d), generator=g).bfloat16().to(dev())
    out = ck.decode_mx(spec, q, cache, 1)
    torch.cuda.synchronize()
    assert int(status.item()) == ck.CERTKV_ENONFINITE
    assert bool(torch.isnan(out).any(-1).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_every_code_is_read_exactly(fmt, d):
    rows, g = 997, gen(7)
    wide = d if fmt == "mxfp8" else d // 2
    c = ck.MxCache(fmt, *(torch.zeros(1, dtype=torch.uint8, device=dev()) for _ in range(4)),
                   offsets=torch.zeros(2, dtype=torch.int64, device=dev()))
    codes = [torch.randint(0, 256, (rows, wide), generator=g).to(torch.uint8) for _ in range(2)]
    if fmt == "mxfp8":
        codes = [torch.where((x & 127) == 127, x - 1, x) for x in codes]  # (NaN codes are not written)
    scales = [torch.randint(27, 245, (rows, d // 32), generator=g).to(torch.uint8) for _ in range(2)]
    scales[0][5, 0] = 255
    c.k, c.v = (x.to(dev()) for x in codes)
    c.k_scales, c.v_scales = (x.to(dev()) for x in scales)
    want = [_mx.decode_codes(x, s, fmt) for x, s in zip(codes, scales)]
    for dt in (torch.bfloat16, torch.float32):
        for first, n in ((0, None), (0, 1), (313, 500), (rows - 1, 1), (4, 0)):
            got = ck.read_mx(c, dtype=dt, first_row=first, rows=n)
            for t, w in zip(got, want):
                w = w[first:] if n is None else w[first:first + n]
                assert torch.equal(torch.isnan(t.cpu()), torch.isnan(w))
                assert torch.equal(torch.nan_to_num(t.cpu().double()), torch.nan_to_num(w))


# ---- attention -------------------------------------------------------------------


def make_cache(fmt, segs, d, g, first=0, k_scale=1.0):
    """(cache for the entry points, fp64 keys, values, offsets): packed rows of the segments'
    lengths, from row `first` on."""
    off = torch.tensor([first] + [first + int(x) for x in torch.tensor(segs).cumsum(0)])
    rows = int(off[-1])
    vals = [torch.randn((rows - first, d), generator=g) * s for s in (k_scale, 1.0)]
    if fmt == "bf16":
        vals = [x.bfloat16() for x in vals]
        full = [torch.zeros((rows, d), dtype=torch.bfloat16, device=dev()) for _ in vals]
        for f, x in zip(full, vals):
            f[first:] = x.to(dev())
        return (full[0], full[1], off.to(dev())), vals[0].double(), vals[1].double(), off - first
    wide = d if fmt == "mxfp8" else d // 2
    t, v64 = [], []
    for x in vals:
        val, byte = _mx.quantise(x, fmt)
        v64.append(val)
        codes = encode(val, byte, fmt)
        full = torch.zeros((rows, wide), dtype=torch.uint8, device=dev())
        full[first:] = codes.to(dev())
        fs = torch.full((rows, d // 32), 127, dtype=torch.uint8, device=dev())
        fs[first:] = byte.to(dev())
        t += [full, fs]
    return ck.MxCache(fmt, *t, offsets=off.to(dev())), v64[0], v64[1], off - first


def encode(val, byte, fmt):
    grid = torch.tensor(_mx.GRID[fmt], dtype=torch.float64)
    y = val.unflatten(-1, (-1, 32)) / torch.exp2(byte.double() - 127).unsqueeze(-1)
    c = torch.searchsorted(grid, y.abs().contiguous())
    c = (c + (y < 0).long() * (128 if fmt == "mxfp8" else 8)).flatten(-2).to(torch.uint8)
    return c if fmt == "mxfp8" else c[..., 0::2] | (c[..., 1::2] << 4)


def check(spec, q, off, k, v, tq, out, lse, k_new=None, v_new=None, mask=None):
    """Every output element and lse within the derived bound of the 64-bit form."""
    L, B, H, G, d = spec.layers, spec.batch, spec.kv_heads, spec.group, spec.head_dim
    scale = 1.0 / math.sqrt(d)
    out, lse = out.cpu().double(), lse.cpu().double()
    tn = 0 if k_new is None else k_new.shape[1] // B
    for l in range(L):
        for b in range(B):
            for h in range(H):
                u = (l * B + b) * H + h
                qh = q[l, b * tq:(b + 1) * tq, h * G:(h + 1) * G].reshape(tq * G, d)
                kk, vv = k[off[u]:off[u + 1]], v[off[u]:off[u + 1]]
                seen = None
                if tn:
                    new = slice(b * tn, (b + 1) * tn)
                    kk = torch.cat([kk, k_new[l, new, h].double()])
                    vv = torch.cat([vv, v_new[l, new, h].double()])
                    seen = torch.ones((tq * G, kk.shape[0]), dtype=torch.bool)
                    seen[:, -tn:] = mask[b].bool().repeat_interleave(G, 0)
                o, z, size, dz = _mx.attend(qh, kk, vv, scale, seen)
                tol, ltol = _mx.bound(size, dz, kk.shape[0], d)
                rows = (l, slice(b * tq, (b + 1) * tq), slice(h * G, (h + 1) * G))
                got, got_z = out[rows].reshape(tq * G, d), lse[rows].reshape(-1)
                fine = torch.isfinite(o)
                assert torch.equal(torch.isfinite(got), fine), (l, b, h)
                err = torch.where(fine, (got - o).abs() - tol, torch.zeros_like(tol))
                assert err.max() <= 0, (l, b, h, float(err.max()))
                ok = torch.isfinite(z)
                assert torch.equal(got_z[torch.isinf(z)], z[torch.isinf(z)])
                assert ((got_z - z).abs()[ok] <= ltol[ok] + 2.0 ** -23 * z.abs()[ok]).all(), (l, b, h)


def queries(L, B, tq, Hq, d, g, strided=False):
    q = torch.randn((L, B * tq, Hq, d), generator=g).bfloat16()
    gpu = q.to(dev())
    if strided:  # head-major with room between heads and layers
        big = torch.full((L, Hq + 1, B * tq + 3, d + 8), math.nan, dtype=torch.bfloat16, device=dev())
        big[:, :Hq, :B * tq, :d] = gpu.transpose(1, 2)
        gpu = big[:, :Hq, :B * tq, :d].transpose(1, 2)
    return q, gpu


# segments: none, one row, around a tile of 32, odd, long
SEGS = [0, 1, 31, 32, 33, 64, 100, 255, 257, 1000, 3, 700]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,G,tq", [
    (128, 1, 1), (128, 4, 1), (128, 8, 2), (128, 3, 5), (128, 8, 4), (128, 5, 7), (128, 4, 32),
    (128, 8, 33), (128, 1, 512), (64, 1, 1), (64, 4, 2), (64, 16, 1), (64, 17, 1), (64, 1, 33),
    (64, 2, 60), (64, 4, 65), (64, 8, 64)])
def test_decode_mx_matches_plain(fmt, d, G, tq):
    L, B, H = 2, 3, 2
    g = gen(d + 100 * G + tq)
    cache, k, v, off = make_cache(fmt, SEGS, d, g)
    spec = ck.ProblemSpec(L, H, G, d, 1, [1000, 2000, 1500])
    q, qd = queries(L, B, tq, H * G, d, g, strided=tq % 2 == 1)
    out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
    check(spec, q, off, k, v, tq, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("tq", [1, 20])
def test_decode_mx_long_segments_and_sharp_weights(fmt, tq):
    # keys eight times as large: a few rows hold all the weight, running maxima grow often
    g = gen(5)
    segs = [20000, 70001, 5, 33000]
    cache, k, v, off = make_cache(fmt, segs, 128, g, k_scale=8.0)
    spec = ck.ProblemSpec(1, 4, 4, 128, 1, [80000])
    q, qd = queries(1, 1, tq, 16, 128, g)
    out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
    check(spec, q, off, k, v, tq, out, lse)
    again, _ = ck.decode_mx(spec, qd, cache, tq, with_lse=True, max_rows=70001)
    assert torch.equal(out, again)  # the row bound is no part of the result


def test_decode_mx_more_rows_than_the_bound_are_reported():
    g = gen(6)
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    spec = ck.ProblemSpec(1, 2, 1, 64, 1, [4000], status=status)
    cache, k, v, off = make_cache("mxfp8", [3000, 1500], 64, g)
    q, qd = queries(1, 1, 1, 2, 64, g)
    out, lse = ck.decode_mx(spec, qd, cache, 1, with_lse=True, max_rows=1600)
    torch.cuda.synchronize()
    assert int(status.item()) == ck.CERTKV_ERANGE
    keep = torch.cat([torch.arange(1600), torch.arange(3000, 4500)])
    check(spec, q, torch.tensor([0, 1600, 3100]), k[keep], v[keep], 1, out, lse)


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_beyond_four_gib(fmt):
    # a cache of one buffer for many programs' rows: the units' rows begin beyond byte 2^32
    d = 128
    first = (1 << 32) // (d if fmt == "mxfp8" else d // 2) + 77
    g = gen(8)
    cache, k, v, off = make_cache(fmt, [500, 0, 1203, 40], d, g, first=first)
    spec = ck.ProblemSpec(1, 4, 2, d, 1, [2000])
    for tq in (1, 40):
        q, qd = queries(1, 1, tq, 8, d, g)
        out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
        check(spec, q, off, k, v, tq, out, lse)
    kk, vv = ck.read_mx(cache, first_row=first, rows=1743)
    assert torch.equal(kk.cpu().double(), k) and torch.equal(vv.cpu().double(), v)


def tree_mask(B, tq, tn, g, empty=True):
    """Random trees over the last tq rows, everything before them visible; the second sequence
    is padded: fewer drafts, fewer rows."""
    m = torch.zeros((B, tq, tn), dtype=torch.bool)
    for b in range(B):
        old = max(0, tn - tq)
        n = tq if b != 1 else max(1, tq // 2)
        m[b, :n, :old if b != 1 else old // 3] = True
        for t in range(min(n, tn)):
            if t:
                par = int(torch.randint(0, t, (1,), generator=g))
                m[b, t, old:] = m[b, par, old:]
            m[b, t, min(old + t, tn - 1)] = True
        if empty:
            m[b, n // 2] = False
    return m


@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
@pytest.mark.parametrize("d,G,tq,tn", [
    (128, 1, 1, 1), (128, 4, 4, 4), (128, 8, 2, 31), (128, 4, 8, 33), (128, 2, 16, 200),
    (128, 8, 24, 101), (128, 4, 64, 64), (128, 8, 64, 70), (128, 1, 300, 300), (64, 1, 1, 1000),
    (64, 2, 5, 1005), (64, 16, 1, 64), (64, 4, 30, 47), (64, 8, 64, 64)])
def test_tree_matches_plain(fmt, d, G, tq, tn):
    L, B, H = 2, 3, 2
    g = gen(d + 7 * G + 31 * tq + tn)
    cache, k, v, off = make_cache(fmt, SEGS, d, g)
    spec = ck.ProblemSpec(L, H, G, d, 1, [1000, 2000, 1500])
    q, qd = queries(L, B, tq, H * G, d, g, strided=tn % 2 == 1)
    kn, knd = queries(L, B, tn, H, d, g, strided=tn % 3 != 0)
    vn, vnd = queries(L, B, tn, H, d, g, strided=tn % 2 == 0)
    mask = tree_mask(B, tq, tn, g)
    out, lse = ck.decode_tree(spec, qd, cache, tq, knd, vnd, mask.to(dev()), with_lse=True)
    check(spec, q, off, k, v, tq, out, lse, kn, vn, mask)
    again = ck.decode_tree(spec, qd, cache, tq, knd, vnd, (mask.byte() * 200).to(dev()),
                           with_lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
@pytest.mark.parametrize("d,G,tq,tn", [(128, 4, 3, 3), (64, 2, 40, 140)])
def test_tree_without_a_mask_is_causal(fmt, d, G, tq, tn):
    g = gen(17 + tn)
    cache, k, v, off = make_cache(fmt, [50, 0, 333, 2], d, g)
    spec = ck.ProblemSpec(1, 2, G, d, 1, [400, 400])
    q, qd = queries(1, 2, tq, 2 * G, d, g)
    kn, knd = queries(1, 2, tn, 2, d, g)
    vn, vnd = queries(1, 2, tn, 2, d, g)
    mask = (torch.arange(tn)[None] <= tn - tq + torch.arange(tq)[:, None]).expand(2, tq, tn)
    out, lse = ck.decode_tree(spec, qd, cache, tq, knd, vnd, None, with_lse=True)
    check(spec, q, off, k, v, tq, out, lse, kn, vn, mask)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("d,G,tq", [(128, 4, 6), (64, 2, 50), (128, 8, 40)])
def test_rows_that_are_not_seen_hold_anything(fmt, d, G, tq):
    # NaN and infinities in rows that nobody sees, and in rows that only some queries see:
    # the others' outputs are as without them, and the seen ones reach their own
    tn, H = tq + 3, 2
    g = gen(23 + tq)
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    spec = ck.ProblemSpec(1, H, G, d, 1, [300], status=status)
    cache, k, v, off = make_cache(fmt, [64, 201], d, g)
    q, qd = queries(1, 1, tq, H * G, d, g)
    kn = torch.randn((1, tn, H, d), generator=g).bfloat16()
    vn = torch.randn((1, tn, H, d), generator=g).bfloat16()
    mask = torch.zeros((1, tq, tn), dtype=torch.bool)
    mask[0, :, :tq] = torch.tril(torch.ones((tq, tq), dtype=torch.bool))
    kn[0, tn - 1], vn[0, tn - 2], vn[0, tn - 3] = math.nan, math.inf, math.nan
    call = lambda: ck.decode_tree(spec, qd, cache, tq, kn.to(dev()), vn.to(dev()),  # noqa: E731
                                  mask.to(dev()), with_lse=True)
    out, lse = call()
    check(spec, q, off, k, v, tq, out, lse, kn, vn, mask)
    assert bool(torch.isfinite(out).all()) and int(status.item()) == ck.CERTKV_OK
    vn[0, tq - 2, :, 5], vn[0, tq - 1, 0, 9] = math.inf, math.nan
    out2, lse2 = call()
    assert int(status.item()) == ck.CERTKV_ENONFINITE
    assert torch.equal(out2[0, :tq - 2], out[0, :tq - 2]) and torch.equal(lse, lse2)
    bad = ~torch.isfinite(out2[0].cpu()).view(tq, H, G, d)
    want = torch.zeros_like(bad)
    want[tq - 2:, :, :, 5] = True
    want[tq - 1, 0, :, 9] = True
    assert torch.equal(bad, want)


def test_nothing_to_see_at_all():
    spec = ck.ProblemSpec(1, 2, 2, 128, 1, [8])
    g = gen(29)
    for fmt in ("bf16", "mxfp4"):
        cache, k, v, off = make_cache(fmt, [0, 0], 128, g, first=1)
        q, qd = queries(1, 1, 3, 4, 128, g)
        kn, knd = queries(1, 1, 40, 2, 128, g)
        out, lse = ck.decode_tree(spec, qd, cache, 3, knd, knd,
                                  torch.zeros((1, 3, 40), dtype=torch.bool, device=dev()),
                                  with_lse=True)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
        if fmt != "bf16":
            out, lse = ck.decode_mx(spec, qd, cache, 3, with_lse=True)
            assert bool((out == 0).all()) and bool((lse == -math.inf).all())


# ---- together, as a program uses them --------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
def test_compress_then_serve(fmt):
    cfg = synth.config("C4", seqlens=[3000, 1029, 517], layers=2)
    made = synth.make_cache(cfg, "cpu")
    spec = spec_of(cfg, layers=2)
    q, k, v = (made[x].to(dev()) for x in ("q_win", "k", "v"))
    ref = ck.compress(spec, q, k, v, made["n_keep"])
    bufs = ck.compress(spec, q, k, v, made["n_keep"], fmt=fmt)
    for x in ("scores", "budgets", "kept_offsets", "kept_idx", "k_star", "v_star", "pos_packed",
              "packed_offsets"):
        assert torch.equal(getattr(ref, x), getattr(bufs, x)), x
    staged = ck.compact_mx(spec, k, v, ref.kept_offsets, ref.kept_idx, ref.k_star, ref.v_star, fmt)
    for x in ("k", "k_scales", "v", "v_scales", "pos", "offsets"):
        assert torch.equal(getattr(staged, x), getattr(bufs.mx, x)), x
    # the rows of the bf16 cache, the slots from their fp32 values
    off = ref.packed_offsets.cpu()
    rows = []
    for t, star in ((ref.k_packed, ref.k_star), (ref.v_packed, ref.v_star)):
        x = t.cpu().double()
        x[off[1:] - 1] = star.cpu().double()
        rows.append(_mx.quantise(x, fmt)[0])
    kk, vv = ck.read_mx(bufs.mx)
    assert torch.equal(kk.cpu().double(), rows[0]) and torch.equal(vv.cpu().double(), rows[1])
    tq, tn, B, H, G, d = 6, 19, cfg.batch, cfg.kv_heads, cfg.group, cfg.head_dim
    g = gen(31)
    qn, qd = queries(2, B, tq, H * G, d, g)
    out, lse = ck.decode_mx(spec, qd, bufs.mx, tq, with_lse=True)
    check(spec, qn, off, rows[0], rows[1], tq, out, lse)
    kn, knd = queries(2, B, tn, H, d, g)
    vn, vnd = queries(2, B, tn, H, d, g)
    mask = tree_mask(B, tq, tn, g)
    out, lse = ck.decode_tree(spec, qd, bufs.mx, tq, knd, vnd, mask.to(dev()), with_lse=True)
    check(spec, qn, off, rows[0], rows[1], tq, out, lse, kn, vn, mask)
    # and a query that sees no new row is decode over the bf16 cache, up to rounding
    none = torch.zeros((B, tq, tn), dtype=torch.bool, device=dev())
    a, _ = ck.decode_tree(spec, qd, (ref.k_packed, ref.v_packed, ref.packed_offsets), tq, knd, vnd,
                          none, with_lse=True)
    b = ck.decode(spec, qd, ref.k_packed, ref.v_packed, ref.packed_offsets, tq)
    assert float((a - b).norm() / b.norm()) < 1e-5


@pytest.mark.parametrize("fmt", FORMATS)
def test_captured_and_replayed_on_a_stream_of_its_own(fmt):
    L, B, H, G, d, tq, tn = 1, 2, 4, 4, 128, 4, 12
    g = gen(37)
    lens = [1500, 900]
    spec = ck.ProblemSpec(L, H, G, d, 1, lens)
    kc, vc = (torch.randn((L, sum(lens), H, d), generator=g).bfloat16().to(dev()) for _ in range(2))
    off, idx = (x.to(dev()) for x in kept_sets(lens, L, H, g))
    ks, vs = (torch.randn((L * B * H, d), generator=g).to(dev()) for _ in range(2))
    rows = int(off[-1]) + L * B * H
    cache = ck.MxCache.empty(spec, rows, fmt, dev())
    q, qd = queries(L, B, tq, H * G, d, g)
    kn, knd = queries(L, B, tn, H, d, g)
    mask = tree_mask(B, tq, tn, g).to(dev())
    d_bufs = ck.DecodeBuffers(spec, tq, dev(), with_lse=True, fmt=fmt)
    t_bufs = ck.DecodeBuffers(spec, tq, dev(), with_lse=True, tn=tn, fmt=fmt)
    vals = [torch.empty((rows, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]

    def step():
        ck.compact_mx(spec, kc, vc, off, idx, ks, vs, fmt, cache=cache)
        ck.read_mx(cache, out=vals)
        ck.decode_mx(spec, qd, cache, tq, with_lse=True, bufs=d_bufs)
        ck.decode_tree(spec, qd, cache, tq, knd, knd, mask, with_lse=True, bufs=t_bufs)

    held = [cache.k, cache.v_scales, cache.pos, *vals, d_bufs.out, d_bufs.lse, t_bufs.out, t_bufs.lse]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for i in range(4):
        kc.copy_(torch.randn(kc.shape, generator=g).bfloat16())
        qd.copy_(torch.randn(qd.shape, generator=g).bfloat16())
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in held]
        for b in (d_bufs, t_bufs):
            b.ws.fill_(i)  # nothing in a workspace outlives a call
        step()
        torch.cuda.synchronize()
        for x, y in zip(replayed, held):
            assert torch.equal(x, y)

"""Performance cases of the microscaled packed cache and of attention for drafted tokens.

A case names one operator and the shape of its cache:

  write   the kept rows and slot rows gathered and quantised into a packed cache
          of 8- or 4-bit floating-point codes with a power-of-two scale for every
          32 dims, and the cache read back as values
  read    the codes of a whole packed cache read back as bf16 values
  decode  tq new queries per sequence over a quantised packed cache
  tree    tq drafted tokens per sequence over a packed cache and the new rows that
          each may see (the tokens since the compression and its own ancestors)

Formats: a block of 32 consecutive dims of a row is held as codes c_i times 2^e.
mxfp8 has e4m3 codes (largest 448), mxfp4 has e2m1 codes (largest 6); e is the
smallest exponent under which the block's largest magnitude is at most the
largest code, kept within [-100, 119] or [-100, 125]; a code is the nearest
value, ties to the even code, larger magnitudes take the largest code.

Shapes are those of the repository's own workloads (Llama-3-8B and 70B class
caches, a tiny fp32 cache, ragged batches) and generic ones around them.
"""
import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 32
# per format: exponent of the largest code's binade, its significand, smallest normal
# exponent, significand bits, largest code, largest block exponent
FORMATS = {"mxfp8": (8, 1.75, -6, 3, 448.0, 119), "mxfp4": (2, 1.5, 0, 1, 6.0, 125)}
MIN_EXP = -100


def _case(name, kind, layers, seqlens, fmt, heads=8, group=4, dim=128, dtype="bf16", keep=0.10,
          slot=True, layout="token", tq=0, tn=0):
    c = dict(kind=kind, layers=layers, seqlens=",".join(str(n) for n in seqlens), format=fmt,
             heads=heads, group=group, dim=dim, dtype=dtype, keep=keep, slot=slot, layout=layout,
             tq=tq, tn=tn)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The tiny fp32 cache, no slot rows: latency and launches.
        _case("write_tiny_f32_fp4", "write", 1, [1024], "mxfp4", heads=4, group=1, dim=64,
              dtype="f32", keep=0.125, slot=False),
        # One layer of an 8B-class model as its prefill ends, head-major source.
        _case("write_layer_32k_fp8", "write", 1, [32768], "mxfp8", layout="head"),
        # Two prompts of odd lengths, sixteen layers.
        _case("write_16l_2seq_fp4", "write", 16, [65537, 24001], "mxfp4"),
        # One layer's packed cache back as values, rows of 64 dims.
        _case("read_layer_d64_fp4", "read", 1, [32768], "mxfp4", dim=64, heads=16),
        # Every layer of the 8B-class cache back as values (a cache that moves to
        # another program, or back to bf16).
        _case("read_8b_32l_fp8", "read", 32, [131072], "mxfp8"),
        # One new token over one layer's packed cache: the layer-by-layer step of a
        # decoding model.
        _case("decode_layer_tq1_fp8", "decode", 1, [32768], "mxfp8", tq=1),
        # One new token over every layer of the 8B-class cache, four bits.
        _case("decode_8b_32l_tq1_fp4", "decode", 32, [131072], "mxfp4", tq=1),
        # A block of 32 new queries over the same cache, eight bits.
        _case("decode_8b_32l_tq32_fp8", "decode", 32, [131072], "mxfp8", tq=32),
        # A small draft on one layer's bf16 cache: latency.
        _case("tree_layer_8_bf16", "tree", 1, [32768], "bf16", tq=8, tn=8),
        # A ragged batch of eight prompts, four layers of a 70B-class model, drafts of
        # up to 24 tokens behind up to 77 tokens since the compression.
        _case("tree_ragged_8_bf16", "tree", 4,
              [58321, 8192, 41007, 20480, 12345, 65536, 30011, 15873], "bf16", group=8, keep=0.05,
              tq=24, tn=101),
        # A tree of 64 drafted tokens over every layer of the 8B-class cache, eight bits.
        _case("tree_8b_32l_64_fp8", "tree", 32, [131072], "mxfp8", tq=64, tn=64),
        # A narrow draft over a long generation: 1000 tokens since the compression.
        _case("tree_3seq_d64_fp4", "tree", 7, [16384, 9999, 30001], "mxfp4", dim=64, heads=16,
              group=2, tq=5, tn=1005),
    ]


MOST_ROWS = 32 * 8 * 13107  # kept rows of 128 dims of a drawn case
MOST_DOTS = MOST_ROWS * 128  # and rows x query rows


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "decode", "decode", "tree", "tree"])
    dim = rng.choice([64, 128, 128])
    heads = rng.choice([4, 8, 8, 16])
    group = rng.choice([1, 2, 4, 4, 8])
    keep = rng.choice([0.05, 0.1, 0.2])
    seqlens = [_log_int(rng, 1024, 131072) for _ in range(rng.choice([1, 1, 2, 3, 8]))]
    if rng.random() < 0.3:  # whole multiples are common too
        seqlens = [max(1024, n // 1024 * 1024) for n in seqlens]
    tq = tn = 0
    if kind == "decode":
        tq = rng.choice([1, 1, 1, 2, 4, 8, 32])
    elif kind == "tree":
        tq = min(_log_int(rng, 1, 64), 512 // group)
        tn = tq + rng.choice([0, 0, _log_int(rng, 1, 1500)])
    fmt = rng.choice(["mxfp8", "mxfp4"] + (["bf16"] if kind == "tree" else []))
    # layers: rows of the cache (and the source's, where it is written) and products in reach
    rows = heads * keep * sum(seqlens) * dim / 128
    cap = 0.5 * MOST_ROWS / rows
    if tq:
        cap = min(cap, 0.5 * MOST_DOTS / (rows * tq * group))
    if kind == "write":
        cap = min(cap, 16 * 8 * 89538 * 128 / (sum(seqlens) * heads * dim))
    layers = min(_log_int(rng, 1, 32), max(1, int(cap)))
    return _case(None, kind, layers, seqlens, fmt, heads=heads, group=group, dim=dim,
                 dtype="f32" if kind == "write" and rng.random() < 0.2 else "bf16", keep=keep,
                 slot=rng.random() < 0.8, layout=rng.choice(["token", "head"]), tq=tq, tn=tn)


def _lens(case):
    return [int(n) for n in case["seqlens"].split(",")]


def _real(case, n):
    """Real rows per head on average: n_keep - 1 of a floor(keep n) + 1 budget."""
    return int(math.floor(case["keep"] * n))


def _budgets(case, gen):
    """Kept rows [L][B][H] of an uneven allocation that sums to H floor(keep n)."""
    L, H = case["layers"], case["heads"]
    out = []
    for n in _lens(case):
        real = H * _real(case, n)
        low = max(1, int(0.2 * real / H))
        share = torch.exp(1.2 * torch.randn((L, H), generator=gen, device=DEV).double())
        share /= share.sum(-1, keepdim=True)
        b = (low + (share * (real - H * low)).long()).clamp_(max=n - 1)
        room = n - 1 - b  # takes what is left, a row at a time in the end
        left = real - b.sum(-1, keepdim=True)
        b += left * room // room.sum(-1, keepdim=True)
        left = real - b.sum(-1, keepdim=True)
        b += (b.argsort(-1).argsort(-1) < left).long()
        out.append(b)
    return torch.stack(out, 1)


def _keys(shape, gen):
    """Normal keys, a few channels eight times as large (as models' keys have)."""
    x = torch.randn(shape, generator=gen, device=DEV)
    big = torch.rand(shape[-1], generator=gen, device=DEV) < 0.05
    return x.mul_(torch.where(big, 8.0, 1.0))


def _values(shape, gen):
    """Student-t values with three degrees of freedom."""
    chi = torch.randn(shape + (3,), generator=gen, device=DEV).square_().sum(-1)
    return torch.randn(shape, generator=gen, device=DEV).mul_(torch.rsqrt(chi / 3.0))


def _draw_codes(rows, case, gen, make):
    """Codes and scale bytes of `rows` rows, as a cache holds them."""
    d, fmt = case["dim"], case["format"]
    codes = torch.empty((rows, d if fmt == "mxfp8" else d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((rows, d // BLOCK), dtype=torch.uint8, device=DEV)
    for r in range(0, rows, 1 << 19):
        x = make((min(rows - r, 1 << 19), d), gen)
        q, e = _round_blocks(x, fmt)
        codes[r:r + len(x)] = _encode(q.reshape(len(x), d), fmt)
        scales[r:r + len(x)] = (e.reshape(len(x), -1) + 127).to(torch.uint8)
    return codes, scales


def _encode(q, fmt):
    """Bytes of representable values: sign, exponent field, significand."""
    _, _, low, bits, _, _ = FORMATS[fmt]
    mag = q.abs()
    ex = torch.frexp(mag)[1] - 1
    ex = torch.where(mag == 0, torch.full_like(ex, low), ex).clamp_(min=low)
    m = torch.ldexp(mag, bits - ex).to(torch.int32)  # with the leading one, if normal
    c = ((ex - low) << bits) + m + (torch.signbit(q).to(torch.int32) << (7 if bits == 3 else 3))
    c = c.to(torch.uint8)
    return c if fmt == "mxfp8" else c[..., 0::2] | (c[..., 1::2] << 4)


def _tree_mask(case, gen):
    """[B][tq][tn]: the tokens since the compression, a random tree's ancestors and the token
    itself; sequences of a batch have their own numbers of both, the rest of the mask is empty."""
    B, tq, tn = len(_lens(case)), case["tq"], case["tn"]
    u = torch.rand((B, tq + 2), generator=gen, device=DEV).cpu()
    mask = torch.zeros((B, tq, tn), dtype=torch.bool)
    for b in range(B):
        old, drafted = tn - tq, tq
        if b:
            old, drafted = int(old * u[b, 0]), max(1, int(tq * (0.4 + 0.6 * u[b, 1])))
        mask[b, :drafted, :old] = True
        for t in range(drafted):
            if t:
                parent = max(0, t - 1 - int(4 * u[b, 2 + t]))
                mask[b, t, old:old + tq] = mask[b, parent, old:old + tq]
            mask[b, t, old + t] = True
    return mask.to(DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000003 + 29)
    L, H, G, d, fmt = (case[x] for x in ("layers", "heads", "group", "dim", "format"))
    lens = _lens(case)
    B, T, U = len(lens), sum(lens), L * len(lens) * H
    kept = _budgets(case, gen).reshape(-1)
    rows = kept + int(case["slot"])
    st = dict(case=case)
    st["offsets"] = torch.zeros(U + 1, dtype=torch.int64, device=DEV)
    st["offsets"][1:] = rows.cumsum(0)
    st["starts"] = st["offsets"].tolist()
    R = st["starts"][-1]
    if case["kind"] == "write":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        shape = (L, T, H, d) if case["layout"] == "token" else (L, H, T, d)
        for x, make in (("k", _keys), ("v", _values)):
            t = torch.empty(shape, dtype=dt, device=DEV)
            for l in range(L):
                t[l] = make(shape[1:], gen)
            st[x] = t if case["layout"] == "token" else t.transpose(1, 2)
        st["kept_offsets"] = torch.zeros(U + 1, dtype=torch.int64, device=DEV)
        st["kept_offsets"][1:] = kept.cumsum(0)
        idx = []
        for u, b in enumerate(kept.tolist()):
            n = lens[u // H % B]
            idx.append(torch.rand(n, generator=gen, device=DEV).topk(b)[1].sort()[0])
        st["kept_idx"] = torch.cat(idx).int()
        st["k_star"] = 0.1 * torch.randn((U, d), generator=gen, device=DEV)
        st["v_star"] = 0.1 * torch.randn((U, d), generator=gen, device=DEV)
    elif fmt == "bf16":
        st["k"] = torch.empty((R, d), dtype=torch.bfloat16, device=DEV)
        st["v"] = torch.empty_like(st["k"])
        for r in range(0, R, 1 << 19):
            st["k"][r:r + (1 << 19)] = _keys((min(R - r, 1 << 19), d), gen)
            st["v"][r:r + (1 << 19)] = _values((min(R - r, 1 << 19), d), gen)
    else:
        st["k"], st["ks"] = _draw_codes(R, case, gen, _keys)
        st["v"], st["vs"] = _draw_codes(R, case, gen, _values)
    if case["tq"]:
        tq, tn = case["tq"], case["tn"]
        st["q"] = torch.randn((L, B * tq, H * G, d), generator=gen, device=DEV).bfloat16()
        if tn:
            st["k_new"] = _keys((L, B * tn, H, d), gen).bfloat16()
            st["v_new"] = _values((L, B * tn, H, d), gen).bfloat16()
            st["mask"] = _tree_mask(case, gen)
        st["max_rows"] = int(rows.max())
    if own:
        _plan(st)
    return st


def _plan(st):
    """What a program keeps between calls: the problem, the cache, outputs and workspace."""
    import paper_2608_21541_amd as ck
    case = st["case"]
    lens = _lens(case)
    spec = ck.ProblemSpec(case["layers"], case["heads"], case["group"], case["dim"], 1, lens,
                          torch.float32 if case["dtype"] == "f32" else torch.bfloat16,
                          slot=case["slot"])
    st["spec"] = spec
    R, fmt = st["starts"][-1], case["format"]
    if case["kind"] == "write":
        st["cache"] = ck.MxCache.empty(spec, R, fmt, torch.device(DEV))
    elif fmt == "bf16":
        st["cache"] = (st["k"], st["v"], st["offsets"])
    else:
        st["cache"] = ck.MxCache(fmt, st["k"], st["ks"], st["v"], st["vs"], st["offsets"])
    if case["kind"] in ("write", "read"):
        st["values"] = [torch.empty((R, case["dim"]), dtype=torch.bfloat16, device=DEV)
                        for _ in range(2)]
    else:
        st["bufs"] = ck.DecodeBuffers(spec, case["tq"], torch.device(DEV), with_lse=True,
                                      max_rows=st["max_rows"], tn=case["tn"], fmt=fmt)


def _run_own(st):
    import paper_2608_21541_amd as ck
    if "spec" not in st:
        _plan(st)
    case, spec, cache = st["case"], st["spec"], st["cache"]
    if case["kind"] in ("write", "read"):
        if case["kind"] == "write":
            ck.compact_mx(spec, st["k"], st["v"], st["kept_offsets"], st["kept_idx"],
                          st["k_star"], st["v_star"], case["format"], cache=cache)
        k, v = ck.read_mx(cache, out=st["values"])
        if case["kind"] == "read":
            return dict(k=k, v=v)
        return dict(k=k, v=v, pos=cache.pos, offsets=cache.offsets)
    if case["kind"] == "decode":
        out, lse = ck.decode_mx(spec, st["q"], cache, case["tq"], with_lse=True, bufs=st["bufs"])
    else:
        out, lse = ck.decode_tree(spec, st["q"], cache, case["tq"], st["k_new"], st["v_new"],
                                  st["mask"], with_lse=True, bufs=st["bufs"])
    return dict(out=out, lse=lse)


# ---- the plain forms ----------------------------------------------------------


def _round_blocks(x, fmt):
    """Rows of x in blocks of 32: the nearest codes' values [.., d/32, 32] and the block
    exponents [.., d/32, 1]."""
    top, sig, low, bits, most, last = FORMATS[fmt]
    x = x.float().unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))  # m in [1/2, 1)
    e = (e - 1 - top + (2 * m > sig).int()).clamp_(MIN_EXP, last)
    y = torch.ldexp(x, -e)
    step = (torch.frexp(y)[1] - 1).clamp_(min=low) - bits
    q = torch.ldexp(torch.round(torch.ldexp(y, -step)), step)  # (torch.round: ties to even)
    return q.clamp_(-most, most), e


def _table(fmt):
    """Values of all codes of a format, by code."""
    _, _, low, bits, _, _ = FORMATS[fmt]
    n = 8 if fmt == "mxfp4" else 128
    c = torch.arange(n, device=DEV)
    field, frac = c >> bits, c & ((1 << bits) - 1)
    mag = torch.where(field > 0, torch.ldexp((frac + (1 << bits)).float(), field + low - 1 - bits),
                      torch.ldexp(frac.float(), torch.full_like(field, low - bits)))
    return torch.cat([mag, -mag])


def _decoded(codes, scales, fmt):
    """fp32 values of a cache's rows."""
    if fmt == "bf16":
        return codes.float()
    if fmt == "mxfp4":
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    x = _table(fmt)[codes.int()].unflatten(-1, (-1, BLOCK))
    return torch.ldexp(x, (scales.int() - 127).unsqueeze(-1)).flatten(-2)


def _source_rows(st):
    """(flat kept positions' layer, token, head), packed rows of the kept ones and of the slots."""
    case = st["case"]
    H, B, lens = case["heads"], len(_lens(case)), torch.tensor(_lens(case), device=DEV)
    U = st["kept_offsets"].numel() - 1
    u = torch.arange(U, device=DEV)
    n = st["kept_offsets"].diff()
    unit = torch.repeat_interleave(u, n)
    first = (lens.cumsum(0) - lens)[u // H % B]
    at = (unit // (H * B), first[unit] + st["kept_idx"], unit % H)
    slot = int(case["slot"])
    return at, torch.arange(unit.numel(), device=DEV) + unit * slot, st["kept_offsets"][1:] + u


def _write_plain(st):
    case = st["case"]
    at, to, slots = _source_rows(st)
    R, d = st["starts"][-1], case["dim"]
    out = {}
    for x in ("k", "v"):
        vals = torch.empty((R, d), dtype=torch.bfloat16, device=DEV)
        src = st[x][at]
        q, e = _round_blocks(src, case["format"])
        vals[to] = torch.ldexp(q, e).flatten(-2).bfloat16()  # (exact: few bits, normal exponents)
        if case["slot"]:
            q, e = _round_blocks(st[x + "_star"], case["format"])
            vals[slots] = torch.ldexp(q, e).flatten(-2).bfloat16()
        out[x] = vals
    pos = torch.full((R,), -1, dtype=torch.int32, device=DEV)
    pos[to] = st["kept_idx"]
    slot = int(case["slot"])
    return dict(out, pos=pos,
                offsets=st["kept_offsets"] + slot * torch.arange(len(st["starts"]), device=DEV))


def _attend_plain(st):
    case = st["case"]
    L, H, G, d, tq, tn = (case[x] for x in ("layers", "heads", "group", "dim", "tq", "tn"))
    B, fmt, off = len(_lens(case)), case["format"], st["starts"]
    out = torch.zeros((L, B * tq, H * G, d), device=DEV)
    lse = torch.empty((L, B * tq, H * G), device=DEV)
    scale = 1.0 / math.sqrt(d)
    for u in range(L * B * H):
        l, b, h = u // (B * H), u // H % B, u % H
        r = slice(off[u], off[u + 1])
        k = _decoded(st["k"][r], st["ks"][r] if "ks" in st else None, fmt)
        v = _decoded(st["v"][r], st["vs"][r] if "vs" in st else None, fmt)
        q = st["q"][l, b * tq:(b + 1) * tq, h * G:(h + 1) * G].float().reshape(tq * G, d)
        if tn:
            new = slice(b * tn, (b + 1) * tn)
            k = torch.cat([k, st["k_new"][l, new, h].float()])
            v = torch.cat([v, st["v_new"][l, new, h].float()])
        z = (q @ k.T).mul_(scale)
        if tn:
            z[:, -tn:].masked_fill_(~st["mask"][b].repeat_interleave(G, 0), -math.inf)
        m = z.amax(-1, keepdim=True)
        p = z.sub_(m).exp_()
        s = p.sum(-1, keepdim=True)
        rows = (l, slice(b * tq, (b + 1) * tq), slice(h * G, (h + 1) * G))
        out[rows] = ((p @ v) / s).view(tq, G, d)
        lse[rows] = (m + s.log()).view(tq, G)
    return dict(out=out, lse=lse)


def run(st):
    if own:
        return _run_own(st)
    kind = st["case"]["kind"]
    if kind == "write":
        return _write_plain(st)
    if kind == "read":
        fmt = st["case"]["format"]
        res = {}
        for x in ("k", "v"):
            vals = torch.empty((st["starts"][-1], st["case"]["dim"]), dtype=torch.bfloat16,
                               device=DEV)
            for r in range(0, len(vals), 1 << 20):
                part = slice(r, r + (1 << 20))
                vals[part] = _decoded(st[x][part], st[x + "s"][part], fmt)
            res[x] = vals
        return res
    return _attend_plain(st)


def work(case):
    L, H, G, d, tq, tn = (case[x] for x in ("layers", "heads", "group", "dim", "tq", "tn"))
    B, slot = len(_lens(case)), int(case["slot"])
    units = L * B * H
    kept = L * H * sum(_real(case, n) for n in _lens(case))
    rows = kept + slot * units
    coded = {"bf16": 2 * d, "mxfp8": d + d // BLOCK, "mxfp4": d // 2 + d // BLOCK}[case["format"]]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "write":  # source rows and positions in, the cache and its values out
        return dict(bytes=2 * kept * d * e + 8 * slot * units * d + 4 * kept + 16 * units +
                    rows * (2 * coded + 4) + 4 * rows * d, flops=8.0 * rows * d)
    if case["kind"] == "read":
        return dict(bytes=rows * (2 * coded + 4 * d), flops=2.0 * rows * d)
    M = tq * G
    new = L * B * H * tn
    return dict(bytes=2 * rows * coded + 4 * new * d + B * tq * tn + units * (M * (6 * d + 4) + 8),
                flops=4.0 * (rows + new) * M * d)


# ---- the definitions in 64 bits -------------------------------------------------


def _exact_nearest(x, fmt):
    """Quantised values of rows in 64 bits: the nearest of the format's multiples of each
    block's scale, by a search of their ordered list."""
    most, last = (448.0, 119) if fmt == "mxfp8" else (6.0, 125)
    if fmt == "mxfp8":
        grid = [m * 2.0 ** -9 for m in range(8)]
        grid += [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]
    else:
        grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    grid = torch.tensor(grid, dtype=torch.float64, device=DEV)
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    for r in range(0, len(x), 1 << 18):
        y = x[r:r + (1 << 18)].double().unflatten(-1, (-1, 32))
        big = y.abs().amax(-1, keepdim=True)
        e = torch.full_like(big, -100)
        scaled = torch.log2((big / most).clamp(min=2.0 ** -200)).ceil() - 1
        for step in range(3):  # the first exponent from below that suffices
            guess = scaled + step
            e = torch.where((big > most * torch.exp2(e)) & (guess > e), guess, e)
        s = torch.exp2(e.clamp(-100, last))
        y = y / s
        mag = y.abs().clamp(max=most)
        hi = torch.searchsorted(grid, mag).clamp(max=len(grid) - 1)
        lo = (hi - 1).clamp(min=0)
        dl, dh = mag - grid[lo], grid[hi] - mag
        pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
        out[r:r + (1 << 18)] = (grid[pick] * torch.sign(y) * s).flatten(-2)
    return out


def _exact_values(codes, scales, fmt):
    """Values of stored codes in 64 bits."""
    if fmt == "bf16":
        return codes.double()
    if fmt == "mxfp4":
        vals = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        c = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.int64, device=DEV)
        c[..., 0::2], c[..., 1::2] = codes % 16, codes // 16
        vals = vals + [-x for x in vals]
    else:
        vals = [(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
                for e in range(16) for m in range(8)]
        vals = vals + [-x for x in vals]
        c = codes.long()
    x = torch.tensor(vals, dtype=torch.float64, device=DEV)[c]
    return x * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def exact(case, seed):
    st = prepare(case, seed)
    L, H, G, d, tq, tn, fmt = (case[x] for x in ("layers", "heads", "group", "dim", "tq", "tn",
                                                 "format"))
    lens = _lens(case)
    B = len(lens)
    if case["kind"] == "read":
        return dict(k=_exact_values(st["k"], st["ks"], fmt),
                    v=_exact_values(st["v"], st["vs"], fmt))
    if case["kind"] == "write":
        ko = st["kept_offsets"].tolist()
        res, pos, off = {"k": [], "v": []}, [], [0]
        for u in range(L * B * H):
            l, b, h = u // (B * H), u // H % B, u % H
            idx = st["kept_idx"][ko[u]:ko[u + 1]]
            tokens = idx.long() + sum(lens[:b])
            for x in ("k", "v"):
                res[x].append(st[x][l, tokens, h].float())
                if case["slot"]:
                    res[x].append(st[x + "_star"][u:u + 1])
            pos.append(idx)
            if case["slot"]:
                pos.append(idx.new_full((1,), -1))
            off.append(off[-1] + len(idx) + (1 if case["slot"] else 0))
        return dict(k=_exact_nearest(torch.cat(res["k"]), fmt),
                    v=_exact_nearest(torch.cat(res["v"]), fmt), pos=torch.cat(pos),
                    offsets=torch.tensor(off, device=DEV))
    out = torch.empty((L, B, tq, H, G, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((L, B, tq, H, G), dtype=torch.float64, device=DEV)
    q = st["q"].double().view(L, B, tq, H, G, d)
    for l in range(L):
        for b in range(B):
            for h in range(H):
                i, j = st["starts"][(l * B + b) * H + h:(l * B + b) * H + h + 2]
                k = _exact_values(st["k"][i:j], st["ks"][i:j] if "ks" in st else None, fmt)
                v = _exact_values(st["v"][i:j], st["vs"][i:j] if "vs" in st else None, fmt)
                qh = q[l, b, :, h]
                z = torch.tensordot(qh, k, dims=([2], [1])) / math.sqrt(d)
                if tn:
                    kn = st["k_new"].view(L, B, tn, H, d)[l, b, :, h].double()
                    vn = st["v_new"].view(L, B, tn, H, d)[l, b, :, h].double()
                    zn = torch.tensordot(qh, kn, dims=([2], [1])) / math.sqrt(d)
                    seen = st["mask"][b].unsqueeze(1).expand(tq, G, tn)
                    zn = torch.where(seen, zn, torch.full_like(zn, -math.inf))
                    z, v = torch.cat([z, zn], -1), torch.cat([v, vn])
                total = torch.logsumexp(z, -1)
                lse[l, b, :, h] = total
                out[l, b, :, h] = torch.tensordot(torch.exp(z - total.unsqueeze(-1)), v,
                                                  dims=([2], [0]))
    return dict(out=out.view(L, B * tq, H * G, d), lse=lse.view(L, B * tq, H * G))

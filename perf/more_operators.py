"""Performance cases of the paged cache: its block tables and slot maps, rows stored in and
read from its pages, and attention over it.

Rows of K and V live in pages of a pool, `page` consecutive rows of one list to a page.  A list
is either a sequence (lists "seq": its pages hold the rows of every layer and KV head of a token,
as a model's prefill leaves them) or one (layer, sequence, KV head) unit (lists "head": after a
compression every head has a length of its own).  A block table names each list's pages, offsets
count its rows, a ring of page numbers holds the free ones.

A case names one operator and the shape of its cache:

  plan    lists grow, shrink and end: pages taken from the ring and given back, the block
          table, the new offsets, and a slot (a row of the pool) for every row to come
  append  the rows of each sequence's newest tokens written to their slots
  store   whole prompts written to their slots and read back as rows
  adopt   a packed cache, as a compression leaves it, moved into pages
  read    the rows of all lists read back from their pages
  decode  tq new queries per sequence over a paged cache, a list's last rows being those of its
          own queries: query t of n sees the rows up to len - n + t

Formats: bf16 rows, or blocks of 32 consecutive dims held as codes c_i times 2^e.  mxfp8 has
e4m3 codes (largest 448), mxfp4 has e2m1 codes (largest 6); e is the smallest exponent under
which the block's largest magnitude is at most the largest code, kept within [-100, 119] or
[-100, 125]; a code is the nearest value, ties to the even code.

Shapes are those of the repository's own workloads (Llama-3-8B and 70B class caches) and generic
ones around them.
"""
import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 32
EMPTY = -2 ** 31  # a change that empties a list
# per format: exponent of the largest code's binade, its significand, smallest normal
# exponent, significand bits, largest code, largest block exponent
FORMATS = {"mxfp8": (8, 1.75, -6, 3, 448.0, 119), "mxfp4": (2, 1.5, 0, 1, 6.0, 125)}
MIN_EXP = -100


def _case(name, kind, lists, layers, seqs, shortest, longest, page, heads=8, group=4, dim=128,
          format="bf16", order="token", keep=0.10, step="step", tq=1, idle=0, scarce=False):
    c = dict(kind=kind, lists=lists, layers=layers, seqs=seqs, shortest=shortest, longest=longest,
             page=page, heads=heads, group=group, dim=dim, format=format, order=order, keep=keep,
             step=step, tq=tq, idle=idle, scarce=scarce)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Every sequence of a decoding batch gets its next token: latency, once a step.
        _case("plan_step_64", "plan", "seq", 1, 64, 512, 32768, 16),
        # A busy server's turn: requests end, prompts come in, drafts are rolled back, the
        # others go on.
        _case("plan_turn_1024", "plan", "seq", 1, 1024, 64, 16384, 64, step="turn"),
        # The lists of an 8B-class cache of 32 layers as a compression leaves its heads.
        _case("plan_fill_32l", "plan", "head", 32, 1, 131072, 131072, 32, step="fill"),
        # The newest token's rows of one layer of a decoding batch: latency, once a layer.
        _case("append_layer_64", "append", "seq", 1, 64, 512, 16384, 16),
        # Three prompts of odd lengths stored in eight bits and read back, eight layers.
        _case("store_3seq_8l_fp8", "store", "seq", 8, 3, 2047, 32771, 64, format="mxfp8"),
        # The packed 8B-class cache moved into pages, each head's rows into its own.
        _case("adopt_8b_32l_bf16", "adopt", "head", 32, 1, 131072, 131072, 64),
        # Two prompts' rows out of their pages, as the compression takes them, 16 layers.
        _case("read_16l_2seq", "read", "seq", 16, 2, 9001, 32768, 128, order="head"),
        # One token of a tiny model over short lists: latency.
        _case("decode_tiny_d64", "decode", "seq", 1, 3, 100, 1024, 16, heads=4, group=1, dim=64),
        # One layer's step of a batch of 64 ragged sequences, two of them empty, the pages
        # token by token.
        _case("decode_layer_64", "decode", "seq", 1, 64, 512, 16384, 16, idle=2),
        # One token over the compressed 8B-class cache, all 32 layers.
        _case("decode_8b_32l", "decode", "head", 32, 1, 131072, 131072, 64),
        # A batch's step over 16 layers of uncompressed eight-bit pages, head by head.
        _case("decode_8seq_16l_fp8", "decode", "seq", 16, 8, 2000, 16384, 128, format="mxfp8",
              order="head"),
        # Drafts of up to 6 tokens over four layers of a compressed 70B-class cache in four bits.
        _case("draft_70b_4l_fp4", "decode", "head", 4, 8, 8192, 65536, 16, group=8, keep=0.05,
              format="mxfp4", tq=6),
    ]


MOST_ROWS = 1 << 24  # rows of 128 dims of a drawn case, counting every list as its longest
MOST_MOVED = 32 * 8 * 13107  # and of those that are moved
MOST_DOTS = 1 << 26  # rows x query rows


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "plan", "append", "store", "adopt", "read", "decode", "decode",
                       "decode", "decode"])
    lists = "head" if kind == "adopt" else rng.choice(["seq", "seq", "head"])
    if kind in ("append", "store"):
        lists = "seq" if kind == "store" else lists
    dim = rng.choice([64, 128, 128])
    heads = rng.choice([1, 2, 4, 8, 8, 16])
    group = rng.choice([1, 2, 3, 4, 4, 8])
    fmt = rng.choice(["bf16", "bf16", "mxfp8", "mxfp4"])
    if kind in ("append", "adopt"):
        fmt = "bf16"
    keep = rng.choice([0.05, 0.1, 0.2])
    seqs = _log_int(rng, 1, 2048 if kind == "plan" else 128)
    if lists == "head":
        seqs = min(seqs, 8)
    longest = _log_int(rng, 16 if lists == "seq" else 1024, 131072)
    if rng.random() < 0.3 and longest > 1024:  # whole multiples are common too
        longest = longest // 1024 * 1024
    shortest = _log_int(rng, 1 if lists == "seq" else 1024, longest)
    step = rng.choice(["step", "turn", "fill"]) if kind == "plan" else "step"
    tq = _log_int(rng, 1, 8) if kind in ("decode", "append", "plan") else 1
    if tq > 1 and kind == "decode" and rng.random() < 0.5:
        tq = 1
    per = longest if lists == "seq" else min(longest, keep * longest * heads) + 1
    rows = seqs * heads * per * dim / 128
    cap = MOST_ROWS / rows
    if kind == "decode":
        cap = min(cap, MOST_DOTS / (rows * tq * group))
    elif kind == "plan":
        cap = MOST_ROWS / (seqs * per * (heads if lists == "head" else 1))
    else:
        cap = min(cap, MOST_MOVED / (rows if lists == "seq" else rows / heads))
    if cap < 1:
        seqs = max(1, int(seqs * cap))
    layers = 1
    if lists == "head" or kind != "plan":
        layers = min(_log_int(rng, 1, 32), max(1, int(cap)))
    idle = rng.randint(0, seqs // 4) if lists == "seq" else 0
    return _case(None, kind, lists, layers, seqs, shortest, longest,
                 rng.choice([16, 16, 32, 64, 128, 256]), heads=heads, group=group, dim=dim,
                 format=fmt, order=rng.choice(["token", "head"]), keep=keep, step=step, tq=tq,
                 idle=idle, scarce=kind == "plan" and rng.random() < 0.3)


def _seq_lens(case):
    """Lengths of the sequences, evenly spaced over their logarithm, the idle ones empty."""
    n, a, b = case["seqs"], case["shortest"], case["longest"]
    lens = [int(round(a * (b / a) ** ((i + 1) / n))) if n > 1 else b for i in range(n)]
    return [0 if i < case["idle"] else x for i, x in enumerate(lens)]


def _roles(case):
    """(rows before, change) of the sequences of a busy server's turn: one in eight ends, one
    is a new prompt, one drops three drafted rows, one gets four, one waits, the others get one."""
    out = []
    for i, n in enumerate(_seq_lens(case)):
        out.append([(n, EMPTY), (0, n), (n, -3), (n, 4), (n, 0), (n, 1), (n, 1), (n, 1)][i % 8])
    return out


def _unit_rows(case, gen):
    """Rows [L][B][H] of an uneven allocation: heads of a (layer, sequence) sum to
    H floor(keep n) kept rows, and a slot row each."""
    L, H = case["layers"], case["heads"]
    out = []
    for n in _seq_lens(case):
        real = H * int(math.floor(case["keep"] * n))
        low = max(1, int(0.2 * real / H))
        share = torch.exp(1.2 * torch.randn((L, H), generator=gen, device=DEV).double())
        share /= share.sum(-1, keepdim=True)
        b = (low + (share * (real - H * low)).long()).clamp_(max=n - 1)
        room = n - 1 - b  # takes what is left, a row at a time in the end
        left = real - b.sum(-1, keepdim=True)
        b += left * room // room.sum(-1, keepdim=True)
        left = real - b.sum(-1, keepdim=True)
        b += (b.argsort(-1).argsort(-1) < left).long()
        out.append(b + 1)
    return torch.stack(out, 1)


def _keys(shape, gen):
    """Normal keys, a few channels eight times as large (as models' keys have)."""
    x = torch.randn(shape, generator=gen, device=DEV)
    big = torch.rand(shape[-1], generator=gen, device=DEV) < 0.05
    return x.mul_(torch.where(big, 8.0, 1.0))


def _values(shape, gen):
    """Student-t values with three degrees of freedom."""
    chi = torch.zeros(shape, device=DEV)
    for _ in range(3):
        chi += torch.randn(shape, generator=gen, device=DEV).square_()
    return torch.randn(shape, generator=gen, device=DEV).mul_(torch.rsqrt(chi / 3.0))


def _rows_of(rows, case, gen, make, fmt):
    """(values or codes, scale bytes) of `rows` rows in a format."""
    d = case["dim"]
    if fmt == "bf16":
        x = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV)
        for r in range(0, rows, 1 << 20):
            x[r:r + (1 << 20)] = make((min(rows - r, 1 << 20), d), gen)
        return x, None
    codes = torch.empty((rows, d if fmt == "mxfp8" else d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((rows, d // BLOCK), dtype=torch.uint8, device=DEV)
    for r in range(0, rows, 1 << 20):
        q, e = _round_blocks(make((min(rows - r, 1 << 20), d), gen), fmt)
        codes[r:r + len(q)] = _encode(q.flatten(-2), fmt)
        scales[r:r + len(q)] = (e.squeeze(-1) + 127).to(torch.uint8)
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


def _pool_shape(case, pages):
    """The pool's shape but for the last axis, and its strides in rows by layer, page, row and
    head."""
    L, H, page = case["layers"], case["heads"], case["page"]
    if case["lists"] == "head":
        return (pages, page), (0, page, 1, 0)
    if case["order"] == "token":
        return (L, pages, page, H), (pages * page * H, page * H, H, 1)
    return (L, pages, H, page), (pages * page * H, page * H, 1, page)


def _shuffled(x, gen):
    return x[torch.randperm(len(x), generator=gen, device=DEV)]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000003 + 31)
    L, H, G, d, page, fmt, B, tq = (case[x] for x in ("layers", "heads", "group", "dim", "page",
                                                      "format", "seqs", "tq"))
    st = dict(case=case)
    # rows of the lists now (had) and what changes
    if case["lists"] == "head":
        rows = _unit_rows(case, gen).reshape(-1)
    else:
        rows = _shuffled(torch.tensor(_seq_lens(case), device=DEV), gen)
    if case["kind"] == "plan":
        if case["step"] == "turn" and case["lists"] == "seq":
            both = _shuffled(torch.tensor(_roles(case), device=DEV), gen)
            had, change = both[:, 0].contiguous(), both[:, 1].contiguous()
        elif case["step"] == "fill":
            had, change = torch.zeros_like(rows), rows
        else:
            had, change = rows, torch.full_like(rows, tq)
        will = (had + change).clamp_(min=0)
    else:
        had = will = rows
        change = None
    U = len(rows)
    held = (had + page - 1) // page
    more = ((will + page - 1) // page - held).clamp_(min=0)
    # a list has at most a row for every token and one more, a pool a page for every `page` rows
    # and one for every list
    st["max_pages"] = (case["longest"] + 1 + (tq if case["kind"] == "plan" else 0)) // page + 1
    used = int(held.sum())
    N = st["num_pages"] = int(torch.maximum(had, will).sum()) // page + U + 1
    free = N - used
    if case["scarce"]:
        free = min(free, int(more.sum()) * 2 // 3)
    ids = torch.randperm(N, generator=gen, device=DEV).int()
    first = held.cumsum(0) - held
    at = torch.arange(st["max_pages"], device=DEV)
    st["table"] = torch.where(at < held[:, None], ids[(first[:, None] + at).clamp_(max=N - 1)],
                              torch.full((), -1, dtype=torch.int32, device=DEV))
    head = int(torch.randint(N, (), generator=gen, device=DEV))
    st["ring"] = torch.zeros(N, dtype=torch.int32, device=DEV)
    st["ring"][(head + torch.arange(N - used, device=DEV)) % N] = ids[used:]
    st["free"] = torch.tensor([head, free], device=DEV)
    st["offsets"] = torch.zeros(U + 1, dtype=torch.int64, device=DEV)
    st["offsets"][1:] = had.cumsum(0)
    st["rows"] = int(st["offsets"][-1])
    st["longest"] = int(had.max())
    if case["kind"] == "plan":
        st["change"] = change.int()
        st["new_rows"] = int(change.clamp(min=0).sum())
        st["freed"] = int((held - (will + page - 1) // page).clamp_(min=0).sum())
    else:
        _fill_pool(st, gen)
    if own:
        _plan(st)
    return st


def _fill_pool(st, gen):
    """The pool's rows, and what is written to it or attends it."""
    case = st["case"]
    L, H, G, d, page, fmt, B, tq = (case[x] for x in ("layers", "heads", "group", "dim", "page",
                                                      "format", "seqs", "tq"))
    N, U = st["num_pages"], len(st["table"])
    shape, st["strides"] = _pool_shape(case, N)
    total = math.prod(shape)
    written = case["kind"] in ("append", "store", "adopt")
    for x, make in (("k", _keys), ("v", _values)):
        if written:  # old rows: of no matter here
            wide = {"bf16": d, "mxfp8": d, "mxfp4": d // 2}[fmt]
            dt = torch.bfloat16 if fmt == "bf16" else torch.uint8
            st[x] = torch.zeros((total, wide), dtype=dt, device=DEV)
            st[x + "s"] = None if fmt == "bf16" else torch.full((total, d // BLOCK), 127,
                                                                dtype=torch.uint8, device=DEV)
        else:
            st[x], st[x + "s"] = _rows_of(total, case, gen, make, fmt)
    if not written:  # what no list holds may be anything
        mine = torch.zeros(total, dtype=torch.bool, device=DEV)
        idx, valid = _all_rows(st)
        mine[idx[valid]] = True
        if fmt == "bf16":
            st["k"][~mine] = math.nan
            st["v"][~mine] = math.nan
        else:
            st["ks"][~mine] = 255
            st["vs"][~mine] = 255
    lens = st["offsets"].diff()
    if case["kind"] in ("append", "store", "adopt"):
        # the lists' last rows (append) or all of them are new
        n = lens if case["kind"] != "append" else lens.clamp(max=tq)
        st["slot_offsets"] = torch.zeros(U + 1, dtype=torch.int64, device=DEV)
        st["slot_offsets"][1:] = n.cumsum(0)
        total_new = int(st["slot_offsets"][-1])
        unit = torch.repeat_interleave(torch.arange(U, device=DEV), n, output_size=total_new)
        row = (lens - n - st["slot_offsets"][:-1])[unit] + torch.arange(total_new, device=DEV)
        st["slots"] = (st["table"][unit, row // page].long() * page + row % page).int()
        if case["kind"] == "adopt":
            src = (total_new, d)
        else:
            src = (L, B * tq if case["kind"] == "append" else total_new, H, d)
        for x, make in (("k_src", _keys), ("v_src", _values)):
            t = torch.empty(src, dtype=torch.bfloat16, device=DEV)
            flat = t.view(-1, d)
            for r in range(0, len(flat), 1 << 20):
                flat[r:r + (1 << 20)] = make((min(len(flat) - r, 1 << 20), d), gen)
            st[x] = t
    if case["kind"] == "decode":
        st["q"] = torch.randn((L, B * tq, H * G, d), generator=gen, device=DEV).bfloat16()
        st["q_lens"] = None
        if tq > 1:  # drafts have their own lengths
            n = torch.randint(1, tq + 1, (B,), generator=gen, device=DEV)
            n[0] = tq
            st["q_lens"] = n.int()


def _plan(st):
    """What a program keeps between calls: the problem, the cache, outputs and workspace."""
    import paper_2608_21541_amd as ck
    case, dev = st["case"], torch.device(DEV)
    L, H, d, page, fmt = (case[x] for x in ("layers", "heads", "dim", "page", "format"))
    N, U = st["num_pages"], len(st["table"])
    spec = ck.ProblemSpec(L if case["kind"] != "plan" or case["lists"] == "head" else 1, H,
                          case["group"], d, 1, [1] * case["seqs"])
    st["spec"] = spec
    k = v = ks = vs = None
    if case["kind"] != "plan":
        shape, _ = _pool_shape(case, N)
        k, v = st["k"].view(*shape, -1), st["v"].view(*shape, -1)
        if fmt != "bf16":
            ks, vs = st["ks"].view(*shape, -1), st["vs"].view(*shape, -1)
        if case["lists"] == "seq" and case["order"] == "head":  # axes [L][pages][page][H]
            k, v, ks, vs = (t if t is None else t.transpose(2, 3) for t in (k, v, ks, vs))
    st["cache"] = ck.PagedCache(format=fmt, page=page, k=k, v=v, k_scales=ks, v_scales=vs,
                                table=st["table"], offsets=st["offsets"], ring=st["ring"],
                                free=st["free"], per_head=case["lists"] == "head")
    if case["kind"] == "plan":
        st["bufs"] = ck.ResizeBuffers(st["cache"], st["new_rows"], dev)
        st["into"] = (torch.empty_like(st["offsets"]), torch.empty_like(st["free"]))
    elif case["kind"] in ("store", "read"):
        shape = (st["rows"], d) if case["lists"] == "head" else (L, st["rows"], H, d)
        st["out"] = [torch.empty(shape, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    elif case["kind"] == "decode":
        st["bufs"] = ck.DecodeBuffers(spec, case["tq"], dev, with_lse=True,
                                      max_rows=st["longest"], pages=st["cache"])


def _run_own(st):
    import paper_2608_21541_amd as ck
    if "spec" not in st:
        _plan(st)
    case, spec, cache = st["case"], st["spec"], st["cache"]
    kind = case["kind"]
    if kind == "plan":
        slots, slot_offsets = ck.page_resize(spec, cache, st["change"], bufs=st["bufs"],
                                             into=st["into"])
        return dict(slots=slots, slot_offsets=slot_offsets, offsets=st["into"][0],
                    free=st["into"][1], table=st["table"], ring=st["ring"])
    if kind == "append":
        ck.page_write(spec, cache, st["k_src"], st["v_src"], st["slots"], st["slot_offsets"],
                      tn=case["tq"])
        return dict(k=st["k"], v=st["v"])
    if kind == "adopt":
        ck.page_adopt(spec, cache, (st["k_src"], st["v_src"], st["slot_offsets"]), st["slots"],
                      st["slot_offsets"])
        return dict(k=st["k"], v=st["v"])
    if kind == "store":
        ck.page_write(spec, cache, st["k_src"], st["v_src"], st["slots"], st["slot_offsets"])
    if kind in ("store", "read"):
        k, v = ck.page_read(spec, cache, out=st["out"])
        return dict(k=k, v=v)
    out, lse = ck.decode_paged(spec, st["q"], cache, case["tq"], q_lens=st["q_lens"],
                               with_lse=True, bufs=st["bufs"])
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


def _table_of_codes(fmt):
    """Values of all codes of a format, by code."""
    _, _, low, bits, _, _ = FORMATS[fmt]
    c = torch.arange(8 if fmt == "mxfp4" else 128, device=DEV)
    field, frac = c >> bits, c & ((1 << bits) - 1)
    mag = torch.where(field > 0, torch.ldexp((frac + (1 << bits)).float(), field + low - 1 - bits),
                      torch.ldexp(frac.float(), torch.full_like(field, low - bits)))
    return torch.cat([mag, -mag])


def _decoded(codes, scales, fmt):
    """fp32 values of rows as they are held."""
    if fmt == "bf16":
        return codes.float()
    if fmt == "mxfp4":
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    x = _table_of_codes(fmt)[codes.int()].unflatten(-1, (-1, BLOCK))
    return torch.ldexp(x, (scales.int() - 127).unsqueeze(-1)).flatten(-2)


def _all_rows(st):
    """The pool's rows of every list's, padded to the longest: indices and which are there, of
    shape [L][B][H][longest]."""
    case = st["case"]
    L, H, B, page = case["layers"], case["heads"], case["seqs"], case["page"]
    sl, sp, sr, sh = st["strides"]
    j = torch.arange(max(st["longest"], 1), device=DEV)
    lens = st["offsets"].diff()
    row = st["table"][:, j // page].long() * sp + (j % page) * sr
    valid = j < lens[:, None]
    row = torch.where(valid, row, torch.zeros_like(row))
    if case["lists"] == "head":
        return row.view(L, B, H, -1), valid.view(L, B, H, -1)
    l = torch.arange(L, device=DEV).view(L, 1, 1, 1) * sl
    h = torch.arange(H, device=DEV).view(1, 1, H, 1) * sh
    return row.view(1, B, 1, -1) + l + h, valid.view(1, B, 1, -1).expand(L, B, H, -1)


def _plan_plain(st):
    page, N, most = st["case"]["page"], st["num_pages"], st["max_pages"]
    table, ring, change = st["table"], st["ring"], st["change"].long()
    had = st["offsets"].diff()
    R, total, freed = len(had), st["new_rows"], st["freed"]
    head, count = st["free"].unbind()
    will = (had + change).clamp(min=0)
    held, want = (had + page - 1) // page, (will + page - 1) // page
    fits = want <= most
    need = torch.where(fits, want - held, 0).clamp(min=0)
    ok = fits & ((need == 0) | (need.cumsum(0) <= count))
    will, need = torch.where(ok, will, had), torch.where(ok, need, 0)
    add, gone = change.clamp(min=0), (held - want).clamp(min=0)
    slot_offsets = torch.cat([add.new_zeros(1), add.cumsum(0)])
    r = torch.arange(R, device=DEV)
    # given back: the pages behind what is left, in list order
    of = torch.repeat_interleave(r, gone, output_size=freed)
    i = torch.arange(freed, device=DEV)
    ring[(head + count + i) % N] = table[of, want[of] + i - (gone.cumsum(0) - gone)[of]]
    # taken: a page for every `page` rows, in list order
    of = torch.repeat_interleave(r, add, output_size=total)
    row = had[of] + torch.arange(total, device=DEV) - slot_offsets[of]
    p = (row // page).clamp(max=most - 1)
    fresh = ok[of] & (p >= held[of])
    taken = ring[(head + (need.cumsum(0) - need)[of] + p - held[of]) % N]
    ids = torch.where(fresh, taken, table[of, p])
    table[of, p] = ids
    slots = torch.where(ok[of], ids.long() * page + row % page, -1).int()
    offsets = torch.cat([will.new_zeros(1), will.cumsum(0)])
    free = torch.stack([(head + need.sum()) % N, count - need.sum() + gone.sum()])
    return dict(slots=slots, slot_offsets=slot_offsets, offsets=offsets, free=free, table=table,
                ring=ring)


def _targets(st):
    """The pool's rows of the new rows' slots: [L][rows][H], or [rows] where lists are heads."""
    case = st["case"]
    sl, sp, sr, sh = st["strides"]
    s = st["slots"].long()
    row = s // case["page"] * sp + s % case["page"] * sr
    if case["lists"] == "head":
        return row
    l = torch.arange(case["layers"], device=DEV).view(-1, 1, 1) * sl
    return row.view(1, -1, 1) + l + torch.arange(case["heads"], device=DEV) * sh


def _write_plain(st):
    case = st["case"]
    to, n = _targets(st), len(st["slots"])
    pick = Ellipsis
    if case["kind"] == "append":  # the sequences' rows are tq apart in the source
        B, L, H, tq = case["seqs"], case["layers"], case["heads"], case["tq"]
        add = st["slot_offsets"].diff()
        of = torch.repeat_interleave(torch.arange(len(add), device=DEV), add, output_size=n)
        i = torch.arange(n, device=DEV) - st["slot_offsets"][of]
        if case["lists"] == "head":
            pick = (of // (B * H), of // H % B * tq + i, of % H)
        else:
            pick = (slice(None), of * tq + i)
    st["k"][to] = st["k_src"][pick]
    st["v"][to] = st["v_src"][pick]
    return dict(k=st["k"], v=st["v"])


def _store_plain(st):
    """Rows to codes in their slots, and the slots' codes to rows."""
    case, to = st["case"], _targets(st)
    out = {}
    for x in ("k", "v"):
        if case["format"] == "bf16":
            st[x][to] = st[x + "_src"]
        else:
            q, e = _round_blocks(st[x + "_src"], case["format"])
            st[x][to] = _encode(q.flatten(-2), case["format"])
            st[x + "s"][to] = (e.squeeze(-1) + 127).to(torch.uint8)
    return _read_plain(st)


def _read_plain(st):
    case = st["case"]
    L, H, fmt, n = case["layers"], case["heads"], case["format"], st["rows"]
    sl, sp, sr, sh = st["strides"]
    lens = st["offsets"].diff()
    of = torch.repeat_interleave(torch.arange(len(lens), device=DEV), lens, output_size=n)
    j = torch.arange(n, device=DEV) - st["offsets"][of]
    row = st["table"][of, j // case["page"]].long() * sp + j % case["page"] * sr
    if case["lists"] == "seq":
        l = torch.arange(L, device=DEV).view(-1, 1, 1) * sl
        row = row.view(1, -1, 1) + l + torch.arange(H, device=DEV) * sh
    k = _decoded(st["k"][row], st["ks"][row] if fmt != "bf16" else None, fmt).bfloat16()
    v = _decoded(st["v"][row], st["vs"][row] if fmt != "bf16" else None, fmt).bfloat16()
    return dict(k=k, v=v)


def _attend_plain(st):
    case = st["case"]
    L, H, G, d, B, tq, fmt = (case[x] for x in ("layers", "heads", "group", "dim", "seqs", "tq",
                                                "format"))
    idx, valid = _all_rows(st)
    k = _decoded(st["k"][idx], st["ks"][idx] if fmt != "bf16" else None, fmt)
    k = k.masked_fill_(~valid.unsqueeze(-1), 0.0)
    # queries [L][B][H][tq G][d]
    q = st["q"].view(L, B, tq, H, G, d).permute(0, 1, 3, 2, 4, 5).reshape(L, B, H, tq * G, d)
    z = torch.matmul(q.float(), k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    del k
    # query t of n sees rows j <= len - n + t
    lens = st["offsets"].diff()
    lens = lens.view(L, B, H, 1) if case["lists"] == "head" else lens.view(1, B, 1, 1)
    t = torch.arange(tq, device=DEV)
    n = torch.full((B,), tq, device=DEV) if st["q_lens"] is None else st["q_lens"].long()
    n = n.view(1, B, 1, 1)
    last = torch.where(t < n, lens - n + t, -1)
    j = torch.arange(idx.shape[-1], device=DEV)
    seen = (j <= last.unsqueeze(-1)).unsqueeze(-2)  # [.][B][.][tq][1][rows]
    z.view(L, B, H, tq, G, -1).masked_fill_(~seen, -math.inf)
    m = z.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = z.sub_(m).exp_()
    s = p.sum(-1, keepdim=True)
    v = _decoded(st["v"][idx], st["vs"][idx] if fmt != "bf16" else None, fmt)
    v = v.masked_fill_(~valid.unsqueeze(-1), 0.0)
    out = torch.matmul(p, v) / s.clamp(min=1e-30)
    lse = torch.where(s > 0, m + s.log(), -math.inf).squeeze(-1)
    out = out.view(L, B, H, tq, G, d).permute(0, 1, 3, 2, 4, 5).reshape(L, B * tq, H * G, d)
    lse = lse.view(L, B, H, tq, G).permute(0, 1, 3, 2, 4).reshape(L, B * tq, H * G)
    return dict(out=out, lse=lse)


def run(st):
    if own:
        return _run_own(st)
    kind = st["case"]["kind"]
    if kind == "plan":
        return _plan_plain(st)
    if kind in ("append", "adopt"):
        return _write_plain(st)
    if kind == "store":
        return _store_plain(st)
    if kind == "read":
        return _read_plain(st)
    return _attend_plain(st)


def work(case):
    L, H, G, d, tq, B, page = (case[x] for x in ("layers", "heads", "group", "dim", "tq", "seqs",
                                                 "page"))
    lens = _seq_lens(case)
    if case["lists"] == "head":
        R = L * B * H
        rows = L * H * sum(int(math.floor(case["keep"] * n)) + 1 for n in lens)  # of all units
        lists = rows  # and of the lists
    else:
        R = B
        lists = sum(lens)
        rows = L * H * lists
    coded = {"bf16": 2 * d, "mxfp8": d + d // BLOCK, "mxfp4": d // 2 + d // BLOCK}[case["format"]]
    kind = case["kind"]
    if kind == "plan":
        if case["step"] == "fill":
            new = lists
        elif case["step"] == "turn" and case["lists"] == "seq":
            new = sum(max(0, c) for _, c in _roles(case))
        else:
            new = tq * R
        # a slot for every row, a page number read and one written for every page
        return dict(bytes=4 * new + 8 * new // page + (8 + 4 + 8 + 8) * R, flops=2.0 * new + 8 * R)
    if kind == "append":
        new = sum(min(n, tq) for n in lens) * L * H if case["lists"] == "seq" else tq * R
        return dict(bytes=2 * new * 4 * d + 4 * new, flops=2.0 * new * d)
    if kind == "adopt":
        return dict(bytes=rows * (2 * 4 * d + 4), flops=2.0 * rows * d)
    if kind == "store":  # the source in, the codes out and in, the values out
        return dict(bytes=rows * (4 * d + 4 * coded + 4 * d) + 8 * lists, flops=8.0 * rows * d)
    if kind == "read":
        return dict(bytes=rows * (2 * coded + 4 * d) + 4 * lists // page, flops=2.0 * rows * d)
    M = tq * G
    return dict(bytes=2 * rows * coded + L * B * H * M * (6 * d + 4) + 4 * lists // page + 8 * R,
                flops=4.0 * rows * M * d)


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


def _exact_plan(st):
    """List by list, on the host."""
    page, N, most = st["case"]["page"], st["num_pages"], st["max_pages"]
    had, change = st["offsets"].diff().tolist(), st["change"].tolist()
    table, ring = st["table"].cpu(), st["ring"].cpu()
    head, count = st["free"].tolist()
    slots, slot_offsets, offsets = [], [0], [0]
    taken = asked = 0
    back = []
    for r, (n, c) in enumerate(zip(had, change)):
        new = max(0, n + c)
        a, b = -(-n // page), -(-new // page)
        ok = True
        if b > a:
            ok = b <= most
            asked += b - a if ok else 0
            ok = ok and asked <= count
            if ok:
                at = (head + taken + torch.arange(b - a)) % N
                table[r, a:b] = ring[at]
                taken += b - a
        elif b < a:
            back.append(table[r, b:a].clone())
        if c > 0:
            if ok:
                row = torch.arange(n, new)
                slots.append(table[r, row // page].long() * page + row % page)
            else:
                slots.append(torch.full((c,), -1))
        slot_offsets.append(slot_offsets[-1] + max(0, c))
        offsets.append(offsets[-1] + (new if ok else n))
    back = torch.cat(back) if back else torch.empty(0, dtype=torch.int32)
    ring[(head + count + torch.arange(len(back))) % N] = back
    slots = torch.cat(slots) if slots else torch.empty(0)
    return dict(slots=slots.int().to(DEV), slot_offsets=torch.tensor(slot_offsets, device=DEV),
                offsets=torch.tensor(offsets, device=DEV),
                free=torch.tensor([(head + taken) % N, count - taken + len(back)], device=DEV),
                table=table.to(DEV), ring=ring.to(DEV))


def _exact_copies(st):
    """The pool with the new rows in their slots, list by list."""
    case = st["case"]
    L, H, B, tq, page = (case[x] for x in ("layers", "heads", "seqs", "tq", "page"))
    sl, sp, sr, sh = st["strides"]
    out, so, slots = {}, st["slot_offsets"].tolist(), st["slots"].long()
    to = torch.div(slots, page, rounding_mode="floor") * sp + torch.remainder(slots, page) * sr
    for x in ("k", "v"):
        pool, src = st[x].double(), st[x + "_src"]
        for r in range(len(so) - 1):
            at, n = to[so[r]:so[r + 1]], so[r + 1] - so[r]
            l, b, h = r // (B * H), r // H % B, r % H
            if case["kind"] == "adopt":
                pool[at] = src[so[r]:so[r + 1]].double()
            elif case["lists"] == "head":
                pool[at] = src[l, b * tq:b * tq + n, h].double()
            else:
                for l in range(L):
                    for h in range(H):
                        pool[at + l * sl + h * sh] = src[l, r * tq:r * tq + n, h].double()
        out[x] = pool
    return out


def exact(case, seed):
    st = prepare(case, seed)
    L, H, G, d, tq, B, page, fmt = (case[x] for x in ("layers", "heads", "group", "dim", "tq",
                                                      "seqs", "page", "format"))
    kind = case["kind"]
    if kind == "plan":
        return _exact_plan(st)
    if kind in ("append", "adopt"):
        return _exact_copies(st)
    if kind == "store":
        return dict((x, _exact_nearest(st[x + "_src"].reshape(-1, d), fmt).view(
            st[x + "_src"].shape) if fmt != "bf16" else st[x + "_src"].double()) for x in ("k", "v"))
    off = st["offsets"].tolist()
    sl, sp, sr, sh = st["strides"]

    def rows_of(l, b, h):
        r = (l * B + b) * H + h if case["lists"] == "head" else b
        n = off[r + 1] - off[r]
        first = st["table"][r, :-(-n // page)].long() * sp + l * sl + h * sh
        return (first[:, None] + torch.arange(page, device=DEV) * sr).flatten()[:n]

    def values(x, rows):
        s = st[x + "s"]
        return _exact_values(st[x][rows], None if s is None else s[rows], fmt)

    if kind == "read":
        out = {}
        for x in ("k", "v"):
            if case["lists"] == "head":
                parts = [values(x, rows_of(l, b, h)) for l in range(L) for b in range(B)
                         for h in range(H)]
                out[x] = torch.cat(parts)
            else:
                out[x] = torch.stack([torch.cat([torch.stack(
                    [values(x, rows_of(l, b, h)) for h in range(H)], 1) for b in range(B)])
                    for l in range(L)])
        return out
    out = torch.zeros((L, B, tq, H, G, d), dtype=torch.float64, device=DEV)
    lse = torch.full((L, B, tq, H, G), -math.inf, dtype=torch.float64, device=DEV)
    q = st["q"].double().view(L, B, tq, H, G, d)
    many = [tq] * B if st["q_lens"] is None else st["q_lens"].tolist()
    for l in range(L):
        for b in range(B):
            for h in range(H):
                rows = rows_of(l, b, h)
                k, v = values("k", rows), values("v", rows)
                for t in range(many[b]):
                    n = len(rows) - many[b] + t + 1
                    if n <= 0:
                        continue
                    z = torch.mv(k[:n], q[l, b, t, h, 0]).unsqueeze(0) if G == 1 else \
                        torch.tensordot(q[l, b, t, h], k[:n], dims=([1], [1]))
                    z = z / math.sqrt(d)
                    total = torch.logsumexp(z, -1)
                    lse[l, b, t, h] = total
                    w = torch.exp(z - total.unsqueeze(-1))
                    out[l, b, t, h] = torch.tensordot(w, v[:n], dims=([1], [0]))
    return dict(out=out.view(L, B * tq, H * G, d), lse=lse.view(L, B * tq, H * G))

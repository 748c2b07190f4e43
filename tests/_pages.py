"""Plain forms of the paged cache (CPU): its lists as Python keeps them, and where their rows are."""
import torch

import paper_2608_21541_amd as ck


class Lists:
    """Block table, offsets and ring of free pages, list by list."""

    def __init__(self, lists, num_pages, page, max_pages, ring=None, head=0):
        self.page, self.most, self.n = page, max_pages, num_pages
        self.table = [[-1] * max_pages for _ in range(lists)]
        self.rows = [0] * lists
        self.ring = list(range(num_pages)) if ring is None else list(ring)
        self.head, self.count = head, num_pages

    def resize(self, change, capacity):
        """(slots, slot_offsets, whether a list was refused) of a step; the lists after it."""
        slots, offsets, refused = [], [0], False
        asked = taken = 0
        back = []
        for r, c in enumerate(change):
            had = self.rows[r]
            will = max(0, had + c)
            a, b = -(-had // self.page), -(-will // self.page)
            offsets.append(offsets[-1] + max(0, c))
            ok = b <= self.most and (c <= 0 or offsets[-1] <= capacity)
            if b > a and b <= self.most:
                asked += b - a
                ok = ok and asked <= self.count
            if ok and b > a:
                for i in range(a, b):
                    self.table[r][i] = self.ring[(self.head + taken) % self.n]
                    taken += 1
            if b < a:
                back += self.table[r][b:a]
            if c > 0:
                slots += [self.table[r][i // self.page] * self.page + i % self.page if ok else -1
                          for i in range(had, had + c)]
            refused |= not ok
            if ok:
                self.rows[r] = will
        for i, x in enumerate(back):
            self.ring[(self.head + self.count + i) % self.n] = x
        self.head = (self.head + taken) % self.n
        self.count += len(back) - taken
        return slots, offsets, refused

    def offsets(self):
        out = [0]
        for n in self.rows:
            out.append(out[-1] + n)
        return out


def rows_of(cache, r, layer=0, head=0):
    """A list's rows as an index into the flat pool rows of (layer, head), on the CPU: pages and
    rows of pages."""
    n = int(cache.offsets[r + 1] - cache.offsets[r])
    i = torch.arange(n)
    return cache.table[r].cpu().long()[i // cache.page], i % cache.page


def values(cache, x, r, layer, head):
    """The rows of list r for (layer, head) in fp64: x "k" or "v"."""
    import _mx
    page, row = rows_of(cache, r)
    at = (page, row) if cache.per_head else (layer, page, row, head)
    t = getattr(cache, x).cpu()[at]
    if cache.format == "bf16":
        return t.double()
    return _mx.decode_codes(t, getattr(cache, x + "_scales").cpu()[at], cache.format)


def make_cache(spec, lens, page, fmt, dev, gen, per_head=False, head_major=False, spare=3,
               garbage=True, max_pages=None):
    """A cache whose lists hold lens rows of normal values in pages of a random order; everything
    else of its pool is not a number (garbage) or zero."""
    import _mx
    need = [-(-n // page) for n in lens]
    num = sum(need) + spare
    cache = ck.PagedCache.empty(spec, num, page, max_pages or max(need + [1]) + 1, "cpu", fmt,
                                per_head=per_head, head_major=head_major)
    ids = torch.randperm(num, generator=gen)
    at = 0
    for r, n in enumerate(need):
        cache.table[r, :n] = ids[at:at + n].int()
        cache.table[r, n:] = 2 ** 30  # (not read)
        at += n
    cache.offsets[1:] = torch.tensor(lens).cumsum(0)
    cache.ring[:num - at] = ids[at:].int()
    cache.free[1] = num - at
    mine = torch.zeros(cache.k.shape[:-1], dtype=torch.bool)
    for r in range(len(lens)):
        page_, row = rows_of(cache, r)
        mine[(page_, row) if per_head else (slice(None), page_, row)] = True
    for x in ("k", "v"):
        t = getattr(cache, x)
        val = torch.randn(tuple(t.shape[:-1]) + (spec.head_dim,), generator=gen)
        if fmt == "bf16":
            val[~mine] = float("nan") if garbage else 0.0
            t.copy_(val)
        else:
            codes, scales = encode(val, fmt)
            scales[~mine] = 255 if garbage else 127
            codes[~mine] = 0
            t.copy_(codes)
            getattr(cache, x + "_scales").copy_(scales)
    return to(cache, dev)


def encode(x, fmt):
    """Codes and scale bytes of x [..., d], by the plain quantiser."""
    import _mx
    v, scales = _mx.quantise(x, fmt)
    grid = torch.tensor(_mx.GRID[fmt], dtype=torch.float64)
    y = v.unflatten(-1, (-1, 32)) / torch.exp2(scales.double() - 127).unsqueeze(-1)
    code = torch.searchsorted(grid, y.abs().contiguous()).to(torch.uint8)
    code = (code + (torch.signbit(y).to(torch.uint8) << (7 if fmt == "mxfp8" else 3))).flatten(-2)
    if fmt == "mxfp4":
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code, scales


def to(cache, dev):
    """The cache on a device, its strides kept."""
    def move(t):
        if t is None:
            return None
        out = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=dev)
        return out.copy_(t)
    names = ("k", "v", "table", "offsets", "k_scales", "v_scales", "ring", "free")
    return ck.PagedCache(cache.format, cache.page, per_head=cache.per_head,
                         **{n: move(getattr(cache, n)) for n in names})


def attend(spec, cache, q, tq, q_lens=None):
    """(out, lse, bound of out, bound of lse) [L][B][tq][Hq].. in fp64 of certkv_decode_paged."""
    import _mx
    L, B, H, G, d = spec.layers, spec.batch, spec.kv_heads, spec.group, spec.head_dim
    q = q.cpu().double().view(L, B, tq, H, G, d)
    out, lse = torch.zeros_like(q), torch.full((L, B, tq, H, G), -float("inf"), dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(q), torch.zeros_like(lse)
    scale = spec.softmax_scale or d ** -0.5
    for l in range(L):
        for b in range(B):
            own = tq if q_lens is None else int(q_lens[b])
            for h in range(H):
                r = (l * B + b) * H + h if cache.per_head else b
                k, v = values(cache, "k", r, l, h), values(cache, "v", r, l, h)
                n = k.shape[0]
                t = torch.arange(tq)
                seen = (torch.arange(n)[None] <= (n - own + t)[:, None]) & (t < own)[:, None]
                o, s, size, dz = _mx.attend(q[l, b, :, h].reshape(tq * G, d), k, v, scale,
                                            seen.repeat_interleave(G, 0))
                e, es = _mx.bound(size, dz, n, d)
                out[l, b, :, h], lse[l, b, :, h] = o.view(tq, G, d), s.view(tq, G)
                tol[l, b, :, h], tol_lse[l, b, :, h] = e.view(tq, G, d), es.view(tq, G)
    flat = lambda x: x.reshape((L, B * tq, H * G) + x.shape[5:])  # noqa: E731
    return flat(out), flat(lse), flat(tol), flat(tol_lse)

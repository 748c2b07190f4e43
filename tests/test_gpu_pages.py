"""Tables and slots of the paged cache, and rows written to, copied to and read from its pages,
against plain forms (integers and rows exactly)."""
import random

import pytest
import torch

import _mx
import _pages
import paper_2608_21541_amd as ck

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DROP = -2 ** 31


def spec_of(L=1, B=2, H=2, G=1, d=64, dtype=torch.bfloat16):
    s = ck.ProblemSpec(L, H, G, d, 1, [1] * B, dtype)
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def tables(lists, num, page, most, ring=None, head=0, count=None, k=None):
    ring = list(range(num)) if ring is None else ring
    return ck.PagedCache("bf16", page, None, None,
                         torch.full((lists, most), -1, dtype=torch.int32, device=DEV),
                         torch.zeros(lists + 1, dtype=torch.int64, device=DEV),
                         ring=torch.tensor(ring, dtype=torch.int32, device=DEV),
                         free=torch.tensor([head, num if count is None else count], device=DEV))


def check_lists(cache, ref, table_too=True):
    assert cache.offsets.tolist() == ref.offsets()
    assert cache.free.tolist() == [ref.head, ref.count]
    assert cache.ring.tolist() == ref.ring
    if table_too:
        assert cache.table.tolist() == ref.table
    # every page has one owner
    held = [p for r, n in enumerate(ref.rows) for p in ref.table[r][:-(-n // ref.page)]]
    free = [ref.ring[(ref.head + i) % ref.n] for i in range(ref.count)]
    assert len(set(held + free)) == len(held) + len(free)


# filled in by the scan's workgroup, of one wave, four or sixteen, or by many
@pytest.mark.parametrize("room", [200, 3000, 10_000, 60_000])
@pytest.mark.parametrize("lists,page", [(1, 16), (2, 1024), (5, 16), (63, 32), (64, 16), (65, 64),
                                        (1023, 16), (1024, 128), (1025, 16), (3000, 32), (7169, 16)])
def test_steps_in_place(lists, page, room):
    rng = random.Random(lists * 7 + page)
    most = 9 if page < 1024 else 3
    num = max(4, lists * 2)
    spec = spec_of(B=lists)
    ring = rng.sample(range(num), num)
    head = rng.randrange(num)
    ref = _pages.Lists(lists, num, page, most, ring=ring, head=head)
    cache = tables(lists, num, page, most, ring=ring, head=head)
    bufs = ck.ResizeBuffers(cache, room, DEV)
    refused = 0
    for step in range(8):
        kind = [lambda: 1, lambda: rng.randint(-2 * page, 3 * page),
                lambda: rng.choice([0, 0, DROP, 1, page, -1, 5 * page]),
                lambda: rng.choice([-page, 0, 2]), lambda: rng.choice([DROP, most * page + 1, 3]),
                lambda: rng.randint(0, 2 * page), lambda: 0, lambda: rng.choice([DROP, 1, 16])][step]
        change = [kind() for _ in range(lists)]
        spec.status.zero_()
        bufs.slots.fill_(-7)
        slots, so = ck.page_resize(spec, cache, torch.tensor(change, dtype=torch.int32, device=DEV),
                                   bufs=bufs)
        want, want_so, bad = ref.resize(change, room)
        assert so.tolist() == want_so
        n = min(len(want), room)
        got = slots.tolist()
        assert got[:n] == want[:n] and set(got[n:]) <= {-7}
        assert (int(spec.status) == ck.CERTKV_ERANGE) == bad and int(spec.status) in (0, ck.CERTKV_ERANGE)
        refused += bad
        check_lists(cache, ref)
    assert refused or lists < 60


@pytest.mark.parametrize("lists,room", [(40, 200), (40, 500), (40, 20_000), (300, 5000), (300, 9000),
                                        (1500, 20_000)])
def test_a_step_beside_the_present_one(lists, room):
    # other offsets and free are written, the cache's own left; the same call gives the same again
    spec = spec_of(B=lists)
    rng = random.Random(lists)
    ref = _pages.Lists(lists, 4 * lists, 16, 4)
    cache = tables(lists, 4 * lists, 16, 4)
    bufs = ck.ResizeBuffers(cache, room, DEV)
    first = [rng.randint(0, 30) for _ in range(lists)]
    ck.page_resize(spec, cache, torch.tensor(first, dtype=torch.int32, device=DEV), bufs=bufs)
    ref.resize(first, room)
    check_lists(cache, ref)
    change = torch.tensor([rng.randint(-20, 20) for _ in range(lists)], dtype=torch.int32, device=DEV)
    offsets, free = cache.offsets.clone(), cache.free.clone()
    into = (torch.empty_like(offsets), torch.empty_like(free))
    want, want_so, _ = ref.resize(change.tolist(), room)
    for _ in range(3):
        slots, so = ck.page_resize(spec, cache, change, bufs=bufs, into=into)
        assert slots[:len(want)].tolist() == want and so.tolist() == want_so
        assert torch.equal(cache.offsets, offsets) and torch.equal(cache.free, free)
    cache.offsets, cache.free = into
    check_lists(cache, ref)


@pytest.mark.parametrize("lists", [1025, 300_000])
def test_many_lists(lists):
    # of numbers of rows that repeat, the last ones refused
    page, most, per = 16, 3, torch.tensor([1, 17, 0, 33, 48, 16], device=DEV)
    spec = spec_of(B=lists)
    change = per.repeat(lists // 6 + 1)[:lists].int()
    need = (change.long() + 15) // 16
    have = int(need.sum()) - 5
    cache = tables(lists, have, page, most)
    cache.ring.copy_(torch.randperm(have, device=DEV))
    cache.free[0] = 77
    bufs = ck.ResizeBuffers(cache, int(change.sum()), DEV)
    taken = need.cumsum(0)
    fits = (need == 0) | (taken <= have)
    slots, so = ck.page_resize(spec, cache, change, bufs=bufs)
    assert int(spec.status) == ck.CERTKV_ERANGE
    kept = torch.where(fits, change.long(), 0)
    assert torch.equal(cache.offsets[1:], kept.cumsum(0)) and int(cache.offsets[0]) == 0
    assert torch.equal(so[1:], change.long().cumsum(0)) and int(so[0]) == 0
    last = int(taken[fits].max())
    assert cache.free.tolist() == [(77 + last) % have, have - last]
    r = torch.repeat_interleave(torch.arange(lists, device=DEV), change.long())
    row = torch.arange(len(slots), device=DEV) - so[:-1][r]
    place = (taken - need)[r] + row // page
    want = cache.ring[(77 + place) % have].long() * page + row % page
    assert torch.equal(slots.long(), torch.where(fits[r], want, -1))
    # and all dropped again: pages go back in the lists' order
    ring = cache.ring.clone()
    held = cache.table[(torch.arange(most, device=DEV) < (need * fits)[:, None])]
    spec.status.zero_()
    ck.page_resize(spec, cache, torch.full_like(change, DROP), bufs=bufs)
    assert int(spec.status) == 0 and not bool(cache.offsets.any())
    at = (77 + have + torch.arange(last, device=DEV)) % have
    ring[at] = held
    assert torch.equal(cache.ring, ring) and cache.free.tolist() == [(77 + last) % have, have]


def test_room_for_no_slot_and_for_some():
    spec = spec_of(B=3)
    cache, ref = tables(3, 8, 16, 4), _pages.Lists(3, 8, 16, 4)
    change = [4, 5, 6]
    dev = lambda c: torch.tensor(c, dtype=torch.int32, device=DEV)  # noqa: E731
    slots, so = ck.page_resize(spec, cache, dev(change))  # room as needed
    assert slots.tolist() == ref.resize(change, 15)[0]
    bufs = ck.ResizeBuffers(cache, 0, DEV)
    assert bufs.slots.numel() == 0
    ck.page_resize(spec, cache, dev([-1, DROP, 0]), bufs=bufs)
    ref.resize([-1, DROP, 0], 0)
    assert int(spec.status) == 0
    check_lists(cache, ref)
    ck.page_resize(spec, cache, dev([1, 0, -6]), bufs=bufs)
    ref.resize([1, 0, -6], 0)
    assert int(spec.status) == ck.CERTKV_ERANGE
    check_lists(cache, ref)
    bufs = ck.ResizeBuffers(cache, 8, DEV)
    slots, _ = ck.page_resize(spec, cache, dev([4, 5, 0]), bufs=bufs)  # the second ends behind 8
    want = ref.resize([4, 5, 0], 8)[0]
    assert slots.tolist() == want[:8] and want[4:] == [-1] * 5
    check_lists(cache, ref)


@pytest.mark.parametrize("room", [100, 20_000])
def test_numbers_that_are_none(room):
    # The caller's numbers on the device: nothing outside the buffers is touched.
    spec = spec_of(B=4)
    dev = lambda c, t=torch.int32: torch.tensor(c, dtype=t, device=DEV)  # noqa: E731
    cache = tables(4, 6, 16, 2, ring=[9, -3, 5, 2 ** 30, 0, 1], head=-5, count=600)
    bufs = ck.ResizeBuffers(cache, room, DEV)
    slots, _ = ck.page_resize(spec, cache, dev([1, 1, 1, 1]), bufs=bufs)
    assert int(spec.status) == ck.CERTKV_ERANGE
    head = (2 ** 64 - 5) % 6
    ids = [[9, -3, 5, 2 ** 30, 0, 1][(head + i) % 6] for i in range(4)]
    assert slots[:4].tolist() == [16 * i if 0 <= i < 6 else -1 for i in ids]
    # lengths that fall, or are more than a list can have
    cache = tables(4, 6, 16, 2)
    cache.offsets.copy_(dev([0, 50, 20, 21, 10 ** 12], torch.int64))
    spec.status.zero_()
    ck.page_resize(spec, cache, dev([-1, 0, 3, DROP]), bufs=bufs)
    off = cache.offsets.tolist()
    assert all(0 <= b - a <= 32 for a, b in zip(off, off[1:]))


@pytest.mark.parametrize("room", [100, 20_000])
@pytest.mark.parametrize("offsets", [[0, 5, 3], [0, 5, 38]])
def test_lengths_that_are_none(room, offsets):
    # such a list holds none, or all that it can, and the call says so
    spec = spec_of(B=2)
    cache = tables(2, 6, 16, 2)
    cache.offsets.copy_(torch.tensor(offsets, dtype=torch.int64, device=DEV))
    change = torch.zeros(2, dtype=torch.int32, device=DEV)
    ck.page_resize(spec, cache, change, bufs=ck.ResizeBuffers(cache, room, DEV))
    assert int(spec.status) == ck.CERTKV_ERANGE
    assert cache.offsets.tolist() == [0, 5, 5 if offsets[2] < 5 else 37]
    spec.status.zero_()
    ck.page_resize(spec, cache, change, bufs=ck.ResizeBuffers(cache, room, DEV))
    assert int(spec.status) == 0


def test_offsets_of_a_part():
    # lists whose first row is not row 0 (a layer's of many)
    spec = spec_of(B=3)
    cache = tables(3, 12, 16, 4)
    cache.offsets.fill_(1000)
    ck.page_resize(spec, cache, torch.tensor([20, 0, 16], dtype=torch.int32, device=DEV))
    assert cache.offsets.tolist() == [1000, 1020, 1020, 1036]


# ---- rows ---------------------------------------------------------------------------


def bits(t):
    return t.contiguous().view(torch.uint8)


def sources(spec, shape, gen, strided=False):
    out = []
    for _ in range(2):
        x = torch.randn(shape, generator=gen) * 3
        if strided:  # heads before tokens, and a gap behind every row
            big = torch.zeros((shape[0], shape[2], shape[1], shape[3] + 8), dtype=spec.dtype, device=DEV)
            v = big[..., :shape[3]].transpose(1, 2)
            v.copy_(x)
            out.append(v)
        else:
            out.append(x.to(device=DEV, dtype=spec.dtype))
    return out


def as_held(x, fmt):
    """Rows as pages hold them, in fp64."""
    if fmt == "bf16":
        return x.bfloat16().double()
    return _mx.quantise(x.float(), fmt)[0]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d,page,head_major,strided", [(64, 16, False, True), (128, 64, True, False)])
def test_prompts_written_and_read(fmt, dtype, d, page, head_major, strided):
    spec = spec_of(L=3, B=4, H=5, d=d, dtype=dtype)
    gen = torch.Generator().manual_seed(d + page)
    lens = [37, 0, 1, 3 * page]
    cache = ck.PagedCache.empty(spec, 12, page, 5, DEV, fmt, head_major=head_major)
    for t in (cache.k, cache.v):
        t.fill_(7)
    n = sum(lens)
    slots, so = ck.page_resize(spec, cache, torch.tensor(lens, dtype=torch.int32, device=DEV))
    k, v = sources(spec, (3, n, 5, d), gen, strided)
    before = bits(cache.k).clone(), bits(cache.v).clone()
    ck.page_write(spec, cache, k, v, slots, so)
    for dt in (torch.bfloat16, torch.float32):
        got = ck.page_read(spec, cache, dtype=dt)
        for x, src in zip(got, (k, v)):
            assert x.shape == (3, n, 5, d) and x.dtype == dt
            assert torch.equal(x.double().cpu(), as_held(src.cpu(), fmt))
    # rows of no list are as they were
    mine = torch.zeros(cache.k.shape[:-1], dtype=torch.bool)
    for r in range(4):
        p, row = _pages.rows_of(cache, r)
        mine[:, p, row] = True
    for t, old in zip((cache.k, cache.v), before):
        wide = t.element_size() * t.shape[-1]
        same = (bits(t) == old).view(t.shape[:-1] + (wide,)).all(-1).cpu()
        assert bool(same[~mine].all()) and not bool(same[mine].all())
    assert int(spec.status) == 0


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("per_head", [False, True])
def test_tokens_appended(fmt, per_head):
    # three tokens of room for each sequence, of which lists take 0 to 3
    L, B, H, d, tn = 2, 3, 4, 64, 3
    spec = spec_of(L, B, H, d=d)
    gen = torch.Generator().manual_seed(11)
    lists = spec.units if per_head else B
    cache = ck.PagedCache.empty(spec, 3 * lists, 16, 3, DEV, fmt, per_head=per_head)
    dev = lambda c: torch.tensor(c, dtype=torch.int32, device=DEV)  # noqa: E731
    kept = {(l, b, h): [] for l in range(L) for b in range(B) for h in range(H)}
    for step in range(12):
        take = [(r * 5 + step) % 4 for r in range(B)]
        per = [take[r // H % B] if per_head else take[r] for r in range(lists)]
        k, v = sources(spec, (L, B * tn, H, d), gen, strided=step % 2 == 1)
        slots, so = ck.page_resize(spec, cache, dev(per))
        ck.page_write(spec, cache, k, v, slots, so, tn=tn)
        for (l, b, h), rows in kept.items():
            rows += [(k[l, b * tn + i, h].cpu(), v[l, b * tn + i, h].cpu()) for i in range(take[b])]
    assert int(spec.status) == 0
    for (l, b, h), rows in kept.items():
        r = (l * B + b) * H + h if per_head else b
        for x, name in ((0, "k"), (1, "v")):
            want = as_held(torch.stack([y[x] for y in rows]), fmt)
            assert torch.equal(_pages.values(cache, name, r, l, h), want)
    k, v = ck.page_read(spec, cache)
    off = cache.offsets.tolist()
    for (l, b, h), rows in kept.items():
        r = (l * B + b) * H + h if per_head else b
        got = k[off[r]:off[r + 1]] if per_head else k[l, off[r]:off[r + 1], h]
        assert torch.equal(got.double().cpu(), as_held(torch.stack([y[0] for y in rows]), fmt))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_packed_cache_adopted(fmt, d):
    spec = spec_of(2, 2, 3, d=d)
    gen = torch.Generator().manual_seed(d)
    rows = [int(x) for x in torch.randint(0, 70, (spec.units,), generator=gen)]
    rows[3], rows[4] = 0, 1
    n = sum(rows)
    off = torch.zeros(spec.units + 1, dtype=torch.int64, device=DEV)
    off[1:] = torch.tensor(rows, device=DEV).cumsum(0)
    if fmt == "bf16":
        packed = tuple(torch.randn((n, d), generator=gen).bfloat16().to(DEV) for _ in range(2)) + (off,)
        want = packed[:2]
    else:
        packed = ck.MxCache.empty(spec, n, fmt, DEV)
        packed.offsets.copy_(off)
        for t, s in ((packed.k, packed.k_scales), (packed.v, packed.v_scales)):
            c, e = _pages.encode(torch.randn((n, d), generator=gen), fmt)
            t.copy_(c), s.copy_(e)
        want = ck.read_mx(packed)
    cache = ck.PagedCache.empty(spec, 80, 16, 6, DEV, fmt, per_head=True)
    change = off.diff().int()
    slots, so = ck.page_resize(spec, cache, change)
    assert torch.equal(so, off)
    ck.page_adopt(spec, cache, packed, slots, so)
    for got, w in zip(ck.page_read(spec, cache), want):
        assert torch.equal(got, w)
    assert torch.equal(cache.offsets, off) and int(spec.status) == 0


def test_slots_that_are_none():
    # -1 leaves a row out; numbers past the pool are left out and reported, and nothing else is
    # written
    spec = spec_of(1, 2, 2, d=64)
    for per_head in (False, True):
        cache = ck.PagedCache.empty(spec, 4, 16, 2, DEV, per_head=per_head)
        cache.k.zero_(), cache.v.zero_()
        dev = lambda c, t=torch.int32: torch.tensor(c, dtype=t, device=DEV)  # noqa: E731
        slots = dev([-1, 3, 64, 2 ** 31 - 1, -2 ** 31, 40])
        if per_head:
            so = dev([0, 2, 3, 5, 6], torch.int64)
            rows = torch.ones((6, 64), dtype=torch.bfloat16, device=DEV)
            call = lambda s: ck.page_adopt(spec, cache, (rows, rows, so), s, so)  # noqa: E731
        else:
            so = dev([0, 4, 6], torch.int64)
            rows = torch.ones((1, 6, 2, 64), dtype=torch.bfloat16, device=DEV)
            call = lambda s: ck.page_write(spec, cache, rows, rows, s, so)  # noqa: E731
        spec.status.zero_()
        call(slots)
        assert int(spec.status) == ck.CERTKV_ERANGE
        hit = cache.k.view(-1, 64).any(-1).nonzero().flatten().tolist()
        assert hit == ([3, 40] if per_head else [6, 7, 80, 81])
        spec.status.zero_()
        call(dev([-1, 3, -1, -1, -1, 40]))
        assert int(spec.status) == 0
        # more slots by the offsets than there are
        spec.status.zero_()
        call(slots[:2].clone())
        assert int(spec.status) == ck.CERTKV_ERANGE


def test_read_into_other_room():
    spec = spec_of(2, 3, 2, d=64)
    gen = torch.Generator().manual_seed(3)
    cache = _pages.make_cache(spec, [20, 0, 33], 16, "bf16", DEV, gen)
    whole = ck.page_read(spec, cache)
    more = [torch.full((2, 60, 2, 64), 9.0, dtype=torch.float32, device=DEV) for _ in range(2)]
    ck.page_read(spec, cache, out=more)
    for m, w in zip(more, whole):
        assert torch.equal(m[:, :53], w.float()) and bool((m[:, 53:] == 9).all())
    assert int(spec.status) == 0
    less = [torch.zeros((2, 30, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ck.page_read(spec, cache, out=less)
    assert torch.equal(less[0], whole[0][:, :30]) and torch.equal(less[1], whole[1][:, :30])
    assert int(spec.status) == ck.CERTKV_ERANGE
    # a page that is none of the pool's
    spec.status.zero_()
    cache.table[2, 1] = 99
    out = [torch.full((2, 53, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ck.page_read(spec, cache, out=out)
    assert int(spec.status) == ck.CERTKV_ERANGE
    keep = torch.ones(53, dtype=torch.bool)
    keep[20 + 16:20 + 32] = False
    for o, w in zip(out, whole):
        assert torch.equal(o[:, keep], w[:, keep]) and bool((o[:, ~keep] == 9).all())


@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
def test_rows_that_are_not_numbers(fmt):
    spec = spec_of(1, 1, 1, d=64)
    cache = ck.PagedCache.empty(spec, 2, 16, 2, DEV, fmt)
    slots, so = ck.page_resize(spec, cache, torch.tensor([3], dtype=torch.int32, device=DEV))
    k = torch.ones((1, 3, 1, 64), dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    k[0, 1, 0, 40] = float("inf")
    ck.page_write(spec, cache, k, v, slots, so)
    assert int(spec.status) == ck.CERTKV_ENONFINITE
    got, _ = ck.page_read(spec, cache)
    assert bool(torch.isnan(got[0, 1, 0, 32:]).all()) and bool((got[0, 1, 0, :32] == 1).all())
    assert bool((got[0, [0, 2]] == 1).all())


def test_no_tokens():
    spec = spec_of(2, 2, 2, d=64)
    cache = ck.PagedCache.empty(spec, 4, 16, 2, DEV)
    none = torch.zeros((2, 0, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots, so = ck.page_resize(spec, cache, torch.zeros(2, dtype=torch.int32, device=DEV))
    assert slots.numel() == 0
    ck.page_write(spec, cache, none, none, slots, so)
    k, v = ck.page_read(spec, cache)
    assert k.shape == v.shape == (2, 0, 2, 64)


@pytest.mark.parametrize("lists", [200, 1000, 1200])
def test_sums_that_stop(lists):
    # far more pages asked for than there are, in lists before, in and behind those of one lane:
    # nothing behind the first refused list is given any
    spec = spec_of(B=lists)
    rng = random.Random(lists)
    for room in (10_000_000, 16_000):
        ref = _pages.Lists(lists, 20, 16, 64)
        cache = tables(lists, 20, 16, 64)
        change = [rng.choice([0, 1, 0, 900, 16, 1000]) if i > 3 else 1 for i in range(lists)]
        bufs = ck.ResizeBuffers(cache, room, DEV)
        slots, so = ck.page_resize(spec, cache, torch.tensor(change, dtype=torch.int32, device=DEV),
                                   bufs=bufs)
        want, want_so, refused = ref.resize(change, room)
        assert refused and so.tolist() == want_so
        n = min(room, len(want))
        assert slots[:n].tolist() == want[:n]
        check_lists(cache, ref)

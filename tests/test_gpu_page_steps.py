"""Steps of the paged cache's tables at the sizes where the way of a call changes: room for no slot,
and many pages given back beside few slots."""
import random

import pytest
import torch

import _pages
import paper_2608_21541_amd as ck
from test_gpu_pages import DEV, DROP, check_lists, spec_of, tables

pytestmark = pytest.mark.gpu


def step(spec, cache, change, bufs=None, into=None):
    return ck.page_resize(spec, cache, torch.tensor(change, dtype=torch.int32, device=DEV), bufs=bufs,
                          into=into)


@pytest.mark.parametrize("beside", [False, True])
@pytest.mark.parametrize("lists", [1, 64, 1024, 1025, 2048, 2049])
def test_lists_that_only_shrink(lists, beside):
    # rows dropped, requests ended, and a step that changes nothing, with room for no slot
    spec, rng = spec_of(B=lists), random.Random(lists)
    ref = _pages.Lists(lists, 4 * lists, 16, 4)
    cache = tables(lists, 4 * lists, 16, 4)
    first = [rng.randint(0, 60) for _ in range(lists)]
    step(spec, cache, first, ck.ResizeBuffers(cache, 60 * lists, DEV))
    ref.resize(first, 60 * lists)
    kinds = (lambda: rng.choice([0, -1, -16, -20]), lambda: 0, lambda: rng.choice([0, DROP]), lambda: DROP)
    for kind in kinds:
        change = [kind() for _ in range(lists)]
        into = (torch.empty_like(cache.offsets), torch.empty_like(cache.free)) if beside else None
        slots, so = step(spec, cache, change, into=into)  # (no list grows: buffers without a slot)
        assert slots.numel() == 0 and not bool(so.any())
        if beside:
            assert cache.offsets.tolist() == ref.offsets()
            cache.offsets, cache.free = into
        ref.resize(change, 0)
        check_lists(cache, ref)
    assert int(spec.status) == 0 and not bool(cache.offsets.any())
    # and grown without room: refused, nothing changes
    step(spec, cache, [1] * lists, ck.ResizeBuffers(cache, 0, DEV))
    ref.resize([1] * lists, 0)
    check_lists(cache, ref)
    assert int(spec.status) == ck.CERTKV_ERANGE


# pages given back by the workgroup of a short step, of one wave, four, eight or sixteen, and by many
@pytest.mark.parametrize("room", [0, 256, 4096, 40_000])
@pytest.mark.parametrize("lists,most", [(1, 3000), (1, 40_000), (3, 1500), (60, 500), (64, 700), (250, 90),
                                        (250, 140), (700, 30), (1500, 20), (2100, 20)])
def test_many_pages_given_back(lists, most, room):
    rng, page = random.Random(lists + most), 16
    spec, num = spec_of(B=lists), lists * most + 5
    ring = rng.sample(range(num), num)
    ref = _pages.Lists(lists, num, page, most, ring=ring, head=num - 3)
    cache = tables(lists, num, page, most, ring=ring, head=num - 3)
    full = [rng.choice([most * page, rng.randint(0, most * page), 0]) for _ in range(lists)]
    full[-1] = most * page
    step(spec, cache, full, ck.ResizeBuffers(cache, sum(full), DEV))
    ref.resize(full, sum(full))
    bufs = ck.ResizeBuffers(cache, room, DEV)
    for kind in (lambda r: rng.choice([0, 0, -1, -page * most // 3]), lambda r: 0 if r % 9 else DROP,
                 lambda r: DROP if r % 2 else -5, lambda r: DROP):
        change = [kind(r) for r in range(lists)]
        if room >= lists:  # (and a row for some)
            change = [c or 1 for c in change]
        step(spec, cache, change, bufs)
        ref.resize(change, room)
        check_lists(cache, ref)


def write(spec, cache, tokens, slots, so, tn=0):
    rows = torch.ones((spec.layers, tokens, spec.kv_heads, spec.head_dim), dtype=spec.dtype, device=DEV)
    spec.status.zero_()
    ck.page_write(spec, cache, rows, rows, slots, so, tn=tn)
    return int(spec.status)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_slots_that_no_token_fills(fmt):
    # rows that the lists count and nobody wrote are reported; the tokens that are there are written
    spec = spec_of(L=2, B=3, H=2, d=64)
    for given, tokens, tn, bad in (([3, 0, 4], 7, 0, False), ([3, 0, 4], 6, 0, True),
                                   ([3, 0, 4], 9, 0, False), ([3, 0, 4], 0, 0, True),
                                   ([0, 0, 0], 0, 0, False), ([3, 0, 4], 12, 4, False),
                                   ([3, 0, 4], 9, 3, True), ([2, 1, 1], 3, 1, True),
                                   ([1, 0, 1], 3, 1, False)):
        cache = ck.PagedCache.empty(spec, 8, 16, 2, DEV, fmt)
        cache.k.zero_()
        slots, so = step(spec, cache, given, ck.ResizeBuffers(cache, 20, DEV))
        got = write(spec, cache, tokens, slots, so, tn)
        assert (got == ck.CERTKV_ERANGE) == bad and got in (0, ck.CERTKV_ERANGE)
        rows = int(cache.k[0].any(-1).any(-1).sum())
        assert rows == (sum(min(n, tn) for n in given) if tn else min(tokens, sum(given)))


@pytest.mark.parametrize("lists", [1, 300, 5000])
def test_one_list_of_many_with_a_slot_too_many(lists):
    # the last list's, by tokens of a number for each sequence
    spec = spec_of(B=lists, H=1, d=64)
    cache = ck.PagedCache.empty(spec, lists + 4, 16, 2, DEV)
    change = torch.ones(lists, dtype=torch.int32, device=DEV)
    slots, so = ck.page_resize(spec, cache, change)
    assert write(spec, cache, lists, slots, so, tn=1) == 0
    change[-1] = 2
    slots, so = ck.page_resize(spec, cache, change)
    assert write(spec, cache, lists, slots, so, tn=1) == ck.CERTKV_ERANGE
    assert write(spec, cache, 2 * lists, slots, so, tn=2) == 0


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_calls_of_no_rows(fmt):
    # slots that a packed cache of no rows leaves, and lists that a read has no room for
    spec = spec_of(L=1, B=3, H=2, d=64)
    cache = ck.PagedCache.empty(spec, 8, 16, 2, DEV, fmt, per_head=True)
    for t in (cache.k, cache.v):
        t.fill_(3)
    packed = ck.MxCache.empty(spec, 0, fmt, DEV) if fmt != "bf16" else \
        tuple(torch.empty((0, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)) + (None,)
    none = [torch.empty((0, 64), dtype=torch.float32, device=DEV) for _ in range(2)]
    for change, bad in (([0] * 6, False), ([0, 3, 0, 0, 1, 0], True)):
        slots, so = step(spec, cache, change, ck.ResizeBuffers(cache, 20, DEV))
        spec.status.zero_()
        ck.page_adopt(spec, cache, packed, slots, so)
        assert int(spec.status) == (ck.CERTKV_ERANGE if bad else 0)
        spec.status.zero_()
        ck.page_read(spec, cache, out=none)
        assert int(spec.status) == (ck.CERTKV_ERANGE if bad else 0)
    assert bool((cache.k == 3).all()) and bool((cache.v == 3).all())
    cache = ck.PagedCache.empty(spec, 8, 16, 2, DEV, fmt)  # and of sequences' lists
    none = [torch.empty((1, 0, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for change, bad in (([0] * 3, False), ([0, 3, 0], True)):
        step(spec, cache, change)
        spec.status.zero_()
        ck.page_read(spec, cache, out=none)
        assert int(spec.status) == (ck.CERTKV_ERANGE if bad else 0)


@pytest.mark.parametrize("per_head", [False, True])
def test_a_read_of_offsets_that_are_none(per_head):
    # offsets that fall, or that say more than a table holds, are reported, also behind or between
    # the rows that are read; nothing outside the outputs is written
    spec = spec_of(L=1, B=2, H=2, d=64)
    cache = ck.PagedCache.empty(spec, 8, 16, 2, DEV, per_head=per_head)
    cache.k.fill_(1), cache.v.fill_(1), cache.table.zero_()
    lists = cache.lists
    room = [torch.full((80 * (1 if per_head else 2), 64), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    shape = (40, 64) if per_head else (1, 40, 2, 64)
    n = 40 * (1 if per_head else 2)
    out = [t[:n].view(shape) for t in room]
    for off in ([0, 20], [7, 39], [0, 20, 15], [0, -5, 20], [0, 33], [30, 20], [2 ** 40, 2 ** 40 + 9],
                [0, 10, 10 ** 12], [0, 30, 25]):
        full = (off + [off[-1]] * lists)[:lists + 1]
        cache.offsets.copy_(torch.tensor(full, device=DEV))
        for t in room:
            t.fill_(5)
        spec.status.zero_()
        ck.page_read(spec, cache, out=out)
        bad = any(not 0 <= b - a <= 32 for a, b in zip(full, full[1:]))
        assert int(spec.status) == (ck.CERTKV_ERANGE if bad else 0), full
        assert all(bool((t[n:] == 5).all()) for t in room)
        if not bad:
            m = (full[-1] - full[0]) * (1 if per_head else 2)
            assert all(bool((t[:m] == 1).all()) and bool((t[m:] == 5).all()) for t in room)

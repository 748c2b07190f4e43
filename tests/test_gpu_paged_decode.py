"""Attention over a paged cache against its definition in 64 bits, at lengths, pages, formats and
masks where it can go wrong."""
import pytest
import torch

import _pages
import paper_2608_21541_amd as ck

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LONG = 2000  # rows that lists have room for where a workgroup does not have a whole unit
EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]


def spec_of(L=1, lens=(), H=2, G=1, d=64, B=None):
    s = ck.ProblemSpec(L, H, G, d, 1, [1] * (B or len(lens)))
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def queries(spec, tq, gen):
    shape = (spec.layers, spec.batch * tq, spec.kv_heads * spec.group, spec.head_dim)
    return torch.randn(shape, generator=gen).bfloat16().to(DEV)


def check(spec, cache, q, tq, q_lens=None, status=0, **kw):
    spec.status.zero_()
    out, lse = ck.decode_paged(spec, q, cache, tq, q_lens=q_lens, with_lse=True, **kw)
    want, want_lse, tol, tol_lse = _pages.attend(spec, cache, q, tq,
                                                 None if q_lens is None else q_lens.tolist())
    got, got_lse = out.double().cpu(), lse.double().cpu()
    assert torch.equal(torch.isinf(want_lse), torch.isinf(got_lse))
    seen = ~torch.isinf(want_lse)
    assert bool((got[~seen] == 0).all()) and bool((got_lse[~seen] < 0).all())
    off = (got - want).abs() - tol
    assert bool((off[seen] <= 0).all()), float(off[seen].max())
    off = (got_lse - want_lse).abs()[seen] - tol_lse[seen]
    assert bool((off <= 0).all()), float(off.max())
    assert int(spec.status) == status
    return out


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,head_major", [(16, False), (32, True), (256, False)])
@pytest.mark.parametrize("H,room", [(3, 300), (3, LONG), (4, LONG)])
def test_one_token_of_every_length(fmt, d, page, head_major, H, room):
    # whole units, pieces of units, and of four heads' units
    spec = spec_of(2, EDGES, H=H, G=4, d=d)
    gen = torch.Generator().manual_seed(page + d)
    cache = _pages.make_cache(spec, EDGES, page, fmt, DEV, gen, head_major=head_major,
                              max_pages=-(-room // page))
    check(spec, cache, queries(spec, 1, gen), 1)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16)])
@pytest.mark.parametrize("room", [700, LONG])
def test_heads_of_their_own_lengths(fmt, d, page, room):
    spec = spec_of(2, B=3, H=3, G=2, d=d)
    gen = torch.Generator().manual_seed(page)
    lens = (EDGES + [700, 0, 90])[:spec.units]
    cache = _pages.make_cache(spec, lens, page, fmt, DEV, gen, per_head=True,
                              max_pages=-(-room // page))
    check(spec, cache, queries(spec, 1, gen), 1)


@pytest.mark.parametrize("G,tq", [(1, 2), (1, 16), (1, 17), (3, 5), (4, 8), (8, 5), (2, 33), (16, 1),
                                  (24, 1), (8, 64)])
@pytest.mark.parametrize("d,fmt,H,room", [(64, "bf16", 2, 250), (128, "bf16", 2, LONG),
                                          (64, "mxfp8", 4, LONG), (128, "mxfp4", 4, LONG)])
def test_drafts(d, fmt, H, room, G, tq):
    # lengths below, at and above the drafts' own
    lens = [0, 1, tq - 1, tq, tq + 1, 40, 200]
    spec = spec_of(1, lens, H=H, G=G, d=d)
    gen = torch.Generator().manual_seed(G * 100 + tq)
    cache = _pages.make_cache(spec, lens, 16, fmt, DEV, gen, max_pages=-(-room // 16))
    q = queries(spec, tq, gen)
    check(spec, cache, q, tq)
    q_lens = torch.tensor([0, tq, 1, tq // 2, tq, 1, tq], dtype=torch.int32, device=DEV)
    check(spec, cache, q, tq, q_lens)


@pytest.mark.parametrize("lists", [5, 300, 2100])
@pytest.mark.parametrize("H,per_head", [(1, False), (4, False), (2, True)])
def test_drafts_of_their_own_lengths(lists, H, per_head):
    # sequences with none, one, two or three groups of 32 query rows beside each other
    B, tq, G = lists // H if per_head else lists, 12, 8
    gen = torch.Generator().manual_seed(lists)
    spec = spec_of(1, B=B, H=H, G=G, d=64)
    n = B * H if per_head else B
    lens = torch.randint(0, 70, (n,), generator=gen).tolist()
    lens[n // 2] = 1500
    cache = _pages.make_cache(spec, lens, 16, "mxfp4", DEV, gen, per_head=per_head,
                              max_pages=LONG // 16)
    q = queries(spec, tq, gen)
    q_lens = torch.randint(0, tq + 1, (B,), generator=gen).int().to(DEV)
    check(spec, cache, q, tq, q_lens)
    assert bool((ck.decode_paged(spec, q, cache, tq, q_lens=torch.zeros_like(q_lens)) == 0).all())


@pytest.mark.parametrize("H,room", [(2, 100), (2, LONG), (4, LONG)])
def test_empty_lists(H, room):
    spec = spec_of(2, [0, 0, 0], H=H, G=2, d=64)
    gen = torch.Generator().manual_seed(1)
    cache = _pages.make_cache(spec, [0, 0, 0], 16, "bf16", DEV, gen, max_pages=room // 16)
    for tq in (1, 20):
        bufs = ck.DecodeBuffers(spec, tq, DEV, with_lse=True, pages=cache)
        bufs.out.fill_(7), bufs.lse.fill_(7)
        out, lse = ck.decode_paged(spec, queries(spec, tq, gen), cache, tq, with_lse=True, bufs=bufs)
        assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    assert int(spec.status) == 0


def test_numbers_of_queries_that_are_none():
    # fewer than none, more than there are
    lens = [40, 40]
    spec = spec_of(1, lens)
    gen = torch.Generator().manual_seed(1)
    cache = _pages.make_cache(spec, lens, 16, "bf16", DEV, gen)
    q = queries(spec, 3, gen)
    for given, meant in (([-5, 3], [0, 3]), ([2 ** 31 - 1, 2], [3, 2])):
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        a = ck.decode_paged(spec, q, cache, 3, q_lens=dev(given)).clone()
        assert torch.equal(a, ck.decode_paged(spec, q, cache, 3, q_lens=dev(meant)))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("d,G,H,room", [(64, 1, 2, 100), (128, 6, 2, LONG), (64, 8, 4, LONG),
                                        (128, 4, 1, 100)])
def test_rows_that_some_queries_do_not_see_may_hold_anything(fmt, d, G, H, room):
    tq, lens = 5, [5, 29, 33, 64, 70]
    spec = spec_of(1, lens, H=H, G=G, d=d)
    gen = torch.Generator().manual_seed(9)
    cache = _pages.make_cache(spec, lens, 16, fmt, DEV, gen, max_pages=-(-room // 16))
    q = queries(spec, tq, gen)
    good, lse = (x.clone() for x in ck.decode_paged(spec, q, cache, tq, with_lse=True))
    for b, n in enumerate(lens):  # the last two tokens' rows
        for row in (n - 1, n - 2):
            at = (0, int(cache.table[b, row // 16]), row % 16)
            if fmt == "bf16":
                cache.k[at] = float("nan")
                cache.v[at] = float("inf") if row % 2 else float("nan")
            else:
                cache.k_scales[at] = cache.v_scales[at] = 255
    out, lse2 = ck.decode_paged(spec, q, cache, tq, with_lse=True)
    t = torch.arange(len(lens) * tq, device=DEV) % tq
    assert torch.equal(out[:, t < tq - 2], good[:, t < tq - 2])
    assert torch.equal(lse2[:, t < tq - 2], lse[:, t < tq - 2])
    assert bool(torch.isnan(out[:, t >= tq - 2]).all())
    assert int(spec.status) == ck.CERTKV_ENONFINITE


@pytest.mark.parametrize("fmt,per_head,d,H", [("bf16", False, 128, 2), ("bf16", True, 64, 3),
                                              ("mxfp8", True, 128, 3), ("mxfp4", False, 64, 4),
                                              ("bf16", False, 128, 8)])
def test_long_lists_are_cut_and_joined(fmt, per_head, d, H):
    # pieces of a list in many workgroups, and many lists' beside them
    gen = torch.Generator().manual_seed(d)
    if per_head:
        spec = spec_of(2, B=1, H=H, G=2, d=d)
        lens = [40_000, 3, 900, 0, 12_345, 5000]
    else:
        lens = [30_011, 1, 4097, 0, 64]
        spec = spec_of(1, lens, H=H, G=4, d=d)
    cache = _pages.make_cache(spec, lens, 64, fmt, DEV, gen, per_head=per_head)
    q = queries(spec, 1, gen)
    a = check(spec, cache, q, 1).clone()
    for _ in range(3):  # no order of the workgroups in the sums
        assert torch.equal(a, ck.decode_paged(spec, q, cache, 1))
    check(spec, cache, queries(spec, 3, gen), 3)
    # a tight bound; a bound that is too short
    most = max(lens)
    check(spec, cache, q, 1, max_rows=most)
    spec.status.zero_()
    ck.decode_paged(spec, q, cache, 1, max_rows=1000)
    assert int(spec.status) == ck.CERTKV_ERANGE


@pytest.mark.parametrize("lists", [65, 400])
def test_many_lists(lists):
    gen = torch.Generator().manual_seed(lists)
    lens = torch.randint(0, 90, (lists,), generator=gen).tolist()
    spec = spec_of(1, lens, H=1, G=2, d=64)
    cache = _pages.make_cache(spec, lens, 16, "bf16", DEV, gen)
    check(spec, cache, queries(spec, 1, gen), 1)
    spec = spec_of(1, B=lists, H=2, G=1, d=64)
    lens = torch.randint(0, 60, (2 * lists,), generator=gen).tolist()
    cache = _pages.make_cache(spec, lens, 16, "bf16", DEV, gen, per_head=True)
    check(spec, cache, queries(spec, 1, gen), 1)


@pytest.mark.parametrize("bound", [100, 1100])
def test_rows_as_a_shorter_bound_leaves_them(bound):
    # the rows within the bound are attended, as if the list ended there
    spec = spec_of(1, [1500], H=2, G=2, d=64)
    gen = torch.Generator().manual_seed(4)
    cache = _pages.make_cache(spec, [1500], 16, "bf16", DEV, gen)
    q = queries(spec, 1, gen)
    out = ck.decode_paged(spec, q, cache, 1, max_rows=bound).clone()
    assert int(spec.status) == ck.CERTKV_ERANGE
    cache.offsets[1] = bound
    want, _, tol, _ = _pages.attend(spec, cache, q, 1)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())


@pytest.mark.parametrize("room", [100, LONG])
def test_pages_that_are_none(room):
    # a page number that is none of the pool's leaves its rows out and is reported
    spec = spec_of(1, [100, 50], H=2, G=2, d=128)
    gen = torch.Generator().manual_seed(6)
    cache = _pages.make_cache(spec, [100, 50], 16, "bf16", DEV, gen, max_pages=-(-room // 16))
    q = queries(spec, 1, gen)
    good = ck.decode_paged(spec, q, cache, 1).clone()
    for bad in (-1, cache.num_pages, 2 ** 31 - 1, -2 ** 31):
        was = cache.table[0, 3].clone()
        cache.table[0, 3] = bad
        spec.status.zero_()
        out = ck.decode_paged(spec, q, cache, 1)
        assert int(spec.status) == ck.CERTKV_ERANGE and bool(torch.isfinite(out).all())
        assert torch.equal(out[:, 1], good[:, 1]) and not torch.equal(out[:, 0], good[:, 0])
        cache.table[0, 3] = was
        # as without these rows
        import _mx
        for h in range(2):
            k, v = (_pages.values(cache, x, 0, 0, h) for x in "kv")
            keep = torch.ones(100, dtype=torch.bool)
            keep[48:64] = False
            o, _, size, dz = _mx.attend(q[0, 0, 2 * h:2 * h + 2].cpu(), k[keep], v[keep], 128 ** -0.5)
            tol, _ = _mx.bound(size, dz, 100, 128)
            assert bool(((out[0, 0, 2 * h:2 * h + 2].double().cpu() - o).abs() <= tol).all())


@pytest.mark.parametrize("H,G,tq", [(1, 1, 1), (4, 1, 1), (2, 8, 9)])
@pytest.mark.parametrize("room", [64, LONG])
def test_offsets_of_any_kind(H, G, tq, room):
    # lengths that fall or are beyond the table: no access outside it
    spec = spec_of(1, B=4, H=H, G=G, d=64)
    gen = torch.Generator().manual_seed(8)
    cache = _pages.make_cache(spec, [30, 40, 50, 20], 16, "bf16", DEV, gen, max_pages=room // 16)
    cache.table.clamp_(max=2)
    q_lens = torch.tensor([tq, 0, 1, tq], dtype=torch.int32, device=DEV)
    for off in ([0, 50, 20, 21, 10 ** 10], [5, 4, 3, 2, 1], [0, 0, 0, 0, 0], [7, 7, 10 ** 6, 7, 7]):
        cache.offsets.copy_(torch.tensor(off, device=DEV))
        for n in (None, q_lens):
            ck.decode_paged(spec, queries(spec, tq, gen), cache, tq, q_lens=n)
            torch.cuda.synchronize()


def test_strided_queries_and_large_scores():
    spec = spec_of(2, [70, 33], H=2, G=3, d=64)
    gen = torch.Generator().manual_seed(12)
    cache = _pages.make_cache(spec, [70, 33], 32, "bf16", DEV, gen, max_pages=LONG // 32)
    tq = 2
    q = queries(spec, tq, gen)
    big = torch.zeros((2, 6, 4, 72), dtype=torch.bfloat16, device=DEV)
    view = big[..., :64].transpose(1, 2)
    view.copy_(q)
    assert torch.equal(ck.decode_paged(spec, view, cache, tq).clone(),
                       ck.decode_paged(spec, q, cache, tq))
    # one key far above the others
    cache.k[:, int(cache.table[0, 0]), 5] *= 3000
    check(spec, cache, q, tq)
    spec.softmax_scale = 0.01
    check(spec, cache, q, tq)


def test_pools_past_32_bits():
    # a pool of more than 4 GiB for K, the lists' pages at its end
    spec = spec_of(1, [200, 77], H=8, G=1, d=128)
    gen = torch.Generator().manual_seed(2)
    small = _pages.make_cache(spec, [200, 77], 128, "bf16", DEV, gen)
    pages = (5 << 30) // (128 * 8 * 256)
    big = ck.PagedCache("bf16", 128, *[torch.empty((1, pages, 128, 8, 128), dtype=torch.bfloat16,
                                                   device=DEV) for _ in range(2)],
                        small.table.clone(), small.offsets)
    first = pages - small.num_pages
    for r, n in ((0, 2), (1, 1)):
        big.table[r, :n] += first
    big.k[:, first:], big.v[:, first:] = small.k, small.v
    q = queries(spec, 1, gen)
    assert torch.equal(ck.decode_paged(spec, q, big, 1).clone(), ck.decode_paged(spec, q, small, 1))
    a, b = ck.page_read(spec, big), ck.page_read(spec, small)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    slot = torch.tensor([pages * 128 - 1], dtype=torch.int32, device=DEV)
    row = torch.full((1, 1, 8, 128), 5.0, dtype=torch.bfloat16, device=DEV)
    ck.page_write(spec, big, row, row, slot, torch.tensor([0, 1, 1], device=DEV))
    assert bool((big.k[0, -1, -1] == 5).all()) and bool((big.v[0, -1, -1] == 5).all())
    assert int(spec.status) == 0


def test_one_layer_of_many():
    for per_head in (False, True):
        spec = spec_of(3, B=2, H=2, G=2, d=64)
        lens = list(range(20, 20 + 12 * 5, 5)) if per_head else [50, 21]
        gen = torch.Generator().manual_seed(7)
        cache = _pages.make_cache(spec, lens, 16, "mxfp8", DEV, gen, per_head=per_head)
        q = queries(spec, 1, gen)
        whole = ck.decode_paged(spec, q, cache, 1).clone()
        one = spec_of(1, B=2, H=2, G=2, d=64)
        for l in range(3):
            part = cache.layer(l, 3)
            got = ck.decode_paged(one, q[l:l + 1], part, 1)
            assert torch.allclose(got, whole[l:l + 1], rtol=0, atol=1e-5)
            check(one, part, q[l:l + 1], 1)
            k, v = ck.page_read(one, part)
            allk, _ = ck.page_read(spec, cache)
            at = slice(int(part.offsets[0]), int(part.offsets[-1]))
            assert torch.equal(k, allk[at] if per_head else allk[l:l + 1])


def test_other_streams_and_buffers():
    spec = spec_of(1, [3000, 100], H=2, G=2, d=64)
    gen = torch.Generator().manual_seed(3)
    cache = _pages.make_cache(spec, [3000, 100], 16, "bf16", DEV, gen)
    qs = [queries(spec, 1, gen) for _ in range(2)]
    want = [ck.decode_paged(spec, q, cache, 1).clone() for q in qs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = [ck.DecodeBuffers(spec, 1, DEV, pages=cache) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):  # two calls at once, each with buffers of its own
        for s, q, b in zip(streams, qs, bufs):
            with torch.cuda.stream(s):
                ck.decode_paged(spec, q, cache, 1, bufs=b)
    torch.cuda.synchronize()
    for b, w in zip(bufs, want):
        assert torch.equal(b.out, w)
    with pytest.raises(AssertionError):  # buffers of another call
        ck.decode_paged(spec, qs[0], cache, 1, bufs=ck.DecodeBuffers(spec, 2, DEV, pages=cache))
    with pytest.raises(AssertionError):
        ck.decode_paged(spec, qs[0], cache, 1, bufs=ck.DecodeBuffers(spec, 1, DEV))
    small = ck.DecodeBuffers(spec, 1, DEV, pages=cache, max_rows=64)
    small.max_rows = 0
    with pytest.raises(ck.CertKVError):
        ck.decode_paged(spec, qs[0], cache, 1, bufs=small)

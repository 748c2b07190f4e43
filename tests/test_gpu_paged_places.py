"""Attention over a paged cache whose lists share pages, or whose offsets are no lists'."""
import pytest
import torch

import _pages
import paper_2608_21541_amd as ck
from test_gpu_paged_decode import DEV, LONG, check, queries, spec_of

pytestmark = pytest.mark.gpu


def nothing(spec, q, cache, tq, q_lens=None):
    """The call sees nothing, says so, and writes nothing behind its buffers' ends."""
    bufs = ck.DecodeBuffers(spec, tq, DEV, with_lse=True, pages=cache)
    bufs.out.fill_(7), bufs.lse.fill_(7)
    room = torch.full((bufs.ws_bytes + (1 << 20),), 91, dtype=torch.uint8, device=DEV)
    bufs.ws = room
    spec.status.zero_()
    out, lse = ck.decode_paged(spec, q, cache, tq, q_lens=q_lens, with_lse=True, bufs=bufs)
    assert int(spec.status) == ck.CERTKV_ERANGE
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    assert bool((room[bufs.ws_bytes:] == 91).all())


@pytest.mark.parametrize("H,G,tq", [(2, 2, 1), (4, 1, 1), (2, 8, 9)])
def test_lists_that_share_pages(H, G, tq):
    # 40 sequences of one prompt: more rows than the pool has
    B, n = 40, 3001
    one = spec_of(1, [n], H=H, G=G, d=64)
    gen = torch.Generator().manual_seed(H)
    own = _pages.make_cache(one, [n], 64, "bf16", DEV, gen)
    cache = ck.PagedCache("bf16", 64, own.k, own.v, own.table.repeat(B, 1),
                          torch.arange(B + 1, device=DEV) * n)
    spec = spec_of(1, B=B, H=H, G=G, d=64)
    q = queries(spec, tq, gen)
    check(spec, cache, q, tq)
    q_lens = torch.randint(0, tq + 1, (B,), generator=gen).int().to(DEV)
    check(spec, cache, q, tq, q_lens)


@pytest.mark.parametrize("L,H,G,tq,copies", [(8, 2, 1, 1, 16), (16, 4, 1, 1, 16), (1, 2, 8, 64, 2)])
def test_more_tiles_than_are_counted(L, H, G, tq, copies):
    # 64 sequences of the same 2^27 rows, 2^28 tiles for a copy: 2^32 for 16, or for 16 groups of
    # query rows with numbers of their own.  The pool has one page.
    B, page = 64, 1024
    spec = spec_of(L, B=B, H=H, G=G, d=64)
    gen = torch.Generator().manual_seed(1)
    pool = lambda: torch.ones((L, 1, page, H, 64), dtype=torch.bfloat16, device=DEV)  # noqa: E731
    table = torch.zeros((B, 2 ** 27 // page), dtype=torch.int32, device=DEV)
    cache = ck.PagedCache("bf16", page, pool(), pool(), table, torch.arange(B + 1, device=DEV) << 27)
    q = queries(spec, tq, gen)
    if copies == 16:
        nothing(spec, q, cache, tq)
    nothing(spec, q, cache, tq, torch.full((B,), tq, dtype=torch.int32, device=DEV))
    # and as many as there may be: shorter lists of the same table
    cache.offsets.copy_(torch.arange(B + 1, device=DEV) * LONG)
    spec.status.zero_()
    out = ck.decode_paged(spec, q, cache, tq)
    # (a sum of n weights is off by half a step for each of its n terms, and so is theirs)
    assert int(spec.status) == 0 and bool(((out - 1).abs() <= 2 * LONG * 2.0 ** -24).all())


@pytest.mark.parametrize("H,G,tq", [(1, 1, 1), (4, 1, 1), (2, 8, 9)])
def test_offsets_below_the_first(H, G, tq):
    # lists that begin before the first offset, or end behind the last: none has a row to see; and
    # lists of more rows than there are places for
    spec = spec_of(1, B=4, H=H, G=G, d=64)
    gen = torch.Generator().manual_seed(8)
    cache = _pages.make_cache(spec, [30, 40, 50, 20], 16, "bf16", DEV, gen, max_pages=LONG // 16)
    cache.table.clamp_(max=2)
    q = queries(spec, tq, gen)
    q_lens = torch.tensor([tq, tq, 1, tq], dtype=torch.int32, device=DEV)
    for off in ([1000, 488, 1088, 1088, 1088], [5, 4, 3, 2, 1], [10 ** 6, 10 ** 6 + 50, 0, 50, 20],
                [0, 2 ** 40, 2 ** 40 + 7, 2 ** 40, 0], [2 ** 62, -2 ** 62, 2 ** 62, -2 ** 62, 2 ** 62],
                [7, 7, 10 ** 6, 7, 7], [0, 2 ** 37, 2 ** 37 + 50, 2 ** 37 + 50, 2 ** 37 + 70],
                [9, 50, 50 + 2 ** 42, 2 ** 43, 2 ** 43]):
        cache.offsets.copy_(torch.tensor(off, device=DEV))
        nothing(spec, q, cache, tq)
        nothing(spec, q, cache, tq, q_lens)


@pytest.mark.parametrize("room", [300, LONG])
@pytest.mark.parametrize("H,G,tq", [(1, 1, 1), (4, 1, 1), (2, 8, 9)])
def test_a_list_that_is_longer_than_its_table(H, G, tq, room):
    # the rows that the table has room for are attended, the others reported; empty ones are neither
    spec = spec_of(1, B=4, H=H, G=G, d=64)
    gen = torch.Generator().manual_seed(8)
    lens = [50, 0, room // 16 * 16, 20]
    cache = _pages.make_cache(spec, lens, 16, "bf16", DEV, gen, max_pages=room // 16)
    q = queries(spec, tq, gen)
    q_lens = torch.tensor([tq, tq, tq, min(1, tq)], dtype=torch.int32, device=DEV)
    for lens_q in (None, q_lens):
        good, lse = (x.clone() for x in ck.decode_paged(spec, q, cache, tq, q_lens=lens_q, with_lse=True))
        assert int(spec.status) == 0
        was = cache.offsets.clone()
        cache.offsets.copy_(torch.tensor([9, 59, 59, 59 + 10 ** 9, 59 + 10 ** 9 + 20], device=DEV))
        spec.status.zero_()
        out, lse2 = ck.decode_paged(spec, q, cache, tq, q_lens=lens_q, with_lse=True)
        assert int(spec.status) == ck.CERTKV_ERANGE
        spec.status.zero_()
        cache.offsets.copy_(was)
        keep = torch.tensor([b != 2 for b in range(4) for _ in range(tq)], device=DEV)
        # (cut elsewhere: sums in another order)
        assert torch.allclose(out[:, keep], good[:, keep], rtol=0, atol=1e-5)
        fin = torch.isfinite(lse[:, keep])
        assert torch.equal(fin, torch.isfinite(lse2[:, keep]))
        assert torch.allclose(lse2[:, keep][fin], lse[:, keep][fin], rtol=0, atol=1e-5)

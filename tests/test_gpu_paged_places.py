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

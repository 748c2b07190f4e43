"""The paged cache as a server uses it: prompts into pages, compressed out of them, the packed
result adopted by lists of its own, tokens appended and attended, steps captured and replayed."""
import pytest
import torch

import _pages
import paper_2608_21541_amd as ck

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
def test_prompts_compressed_and_decoded(fmt):
    L, B, H, G, d, w = 2, 2, 4, 2, 64, 8
    lens, keep = [300, 219], [40, 31]
    spec = ck.ProblemSpec(L, H, G, d, w, lens)
    spec.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    gen = torch.Generator().manual_seed(21)
    rnd = lambda *s: torch.randn(s, generator=gen).bfloat16().to(DEV)  # noqa: E731
    k, v, qw = rnd(L, sum(lens), H, d), rnd(L, sum(lens), H, d), rnd(L, B * w, H * G, d)
    # a prefill's pages, and out of them what the pass takes
    full = ck.PagedCache.empty(spec, 40, 16, 24, DEV)
    slots, so = ck.page_resize(spec, full, ints(lens))
    ck.page_write(spec, full, k, v, slots, so)
    k2, v2 = ck.page_read(spec, full)
    assert torch.equal(k2, k) and torch.equal(v2, v)
    mx = None if fmt == "bf16" else fmt
    res = ck.compress(spec, qw, k2, v2, keep, fmt=mx)
    packed = (res.k_packed, res.v_packed, res.packed_offsets) if mx is None else res.mx
    # its heads' rows into lists of their own, the prompts' pages free again
    heads = ck.PagedCache.empty(spec, 200, 16, 20, DEV, fmt, per_head=True)
    slots, so = ck.page_resize(spec, heads, res.packed_offsets.diff().int())
    ck.page_adopt(spec, heads, packed, slots, so)
    ck.page_resize(spec, full, ints([-2 ** 31] * B))
    assert full.free.tolist()[1] == 40 and int(full.offsets[-1]) == 0
    q = rnd(L, B, H * G, d)
    one = ck.decode(spec, q, *packed, 1) if mx is None else ck.decode_mx(spec, q, packed, 1)
    one = one.clone()
    # (one token that sees the packed rows: no new row of its own)
    got = ck.decode_paged(spec, q, heads, 1)
    assert torch.allclose(got, one, rtol=0, atol=2e-5)
    # tokens appended one after another, attended as decode_tree attends them
    new_k, new_v = rnd(L, B * 3, H, d), rnd(L, B * 3, H, d)
    if mx:  # (as the pages hold them)
        spare = ck.PagedCache.empty(spec, 6, 16, 2, DEV, fmt)
        s, o = ck.page_resize(spec, spare, ints([3, 3]))
        ck.page_write(spec, spare, new_k, new_v, s, o)
        new_k, new_v = ck.page_read(spec, spare)
    for t in range(3):
        at = torch.tensor([t, 3 + t], device=DEV)
        slots, so = ck.page_resize(spec, heads, ints([1] * spec.units))
        ck.page_write(spec, heads, new_k[:, at].contiguous(), new_v[:, at].contiguous(), slots, so,
                      tn=1)
        q = rnd(L, B, H * G, d)
        rows = torch.tensor([b * 3 + i for b in range(B) for i in range(t + 1)], device=DEV)
        want = ck.decode_tree(spec, q, packed, 1, new_k[:, rows].contiguous(),
                              new_v[:, rows].contiguous())
        assert torch.allclose(ck.decode_paged(spec, q, heads, 1), want, rtol=0, atol=2e-5)
    # the last two rolled back, then a draft of two in their place
    before = heads.offsets.clone()
    ck.page_resize(spec, heads, ints([-2] * spec.units))
    slots, so = ck.page_resize(spec, heads, ints([2] * spec.units))
    assert torch.equal(heads.offsets, before)
    at = torch.tensor([1, 2, 4, 5], device=DEV)
    ck.page_write(spec, heads, new_k[:, at].contiguous(), new_v[:, at].contiguous(), slots, so, tn=2)
    q = rnd(L, B * 2, H * G, d)
    want = ck.decode_tree(spec, q, packed, 2, new_k, new_v)
    assert torch.allclose(ck.decode_paged(spec, q, heads, 2), want, rtol=0, atol=2e-5)
    assert int(spec.status) == 0


@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("room", [None, 20_000])  # slots by one launch, or by two
def test_steps_captured_and_replayed(per_head, room):
    L, B, H, G, d = 1, 3, 2, 2, 64
    spec = ck.ProblemSpec(L, H, G, d, 1, [1] * B)
    spec.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    gen = torch.Generator().manual_seed(5)
    lists = spec.units if per_head else B
    lens = [13, 40, 0, 5, 31, 16][:lists]

    def fresh():
        g = torch.Generator().manual_seed(6)
        return _pages.make_cache(spec, lens, 16, "bf16", DEV, g, per_head=per_head, spare=20,
                                 max_pages=8)
    caches = [fresh(), fresh()]
    for c in caches:
        c.table.clamp_(max=c.num_pages - 1)
    change = ints([1 + i % 2 for i in range(lists)] if not per_head else [1] * lists)
    tn = 2
    k, v = (torch.empty((L, B * tn, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = torch.empty((L, B, H * G, d), dtype=torch.bfloat16, device=DEV)
    bufs = [(ck.ResizeBuffers(c, room or 2 * lists, DEV), ck.DecodeBuffers(spec, 1, DEV, pages=c))
            for c in caches]

    def step(i):
        slots, so = ck.page_resize(spec, caches[i], change, bufs=bufs[i][0])
        ck.page_write(spec, caches[i], k, v, slots, so, tn=tn)
        return ck.decode_paged(spec, q, caches[i], 1, bufs=bufs[i][1])

    def draw():
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=gen).bfloat16())
    draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # both one step on, outside the graph
        step(0), step(1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(1)
    for i in range(20):
        draw()
        want = step(0).clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bufs[1][1].out, want), i
        assert torch.equal(caches[0].offsets, caches[1].offsets)
        assert torch.equal(caches[0].free, caches[1].free)
        assert bool(torch.isfinite(want).all())
    assert int(spec.status) == 0
    ref, _, tol, _ = _pages.attend(spec, caches[1], q, 1)
    assert bool(((bufs[1][1].out.double().cpu() - ref).abs() <= tol).all())

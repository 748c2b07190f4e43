"""Calls of the microscaled cache's and the drafted tokens' entry points that their
documentation allows and that are easy to get wrong: many units, the longest rows of new
tokens, padded queries, two streams, buffers of another call."""
import math

import pytest
import torch

import paper_2608_21541_amd as ck
from test_gpu_mx import check, dev, gen, make_cache, queries, tree_mask

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.init()


@pytest.mark.parametrize("fmt,L,H,tq,tn", [("mxfp8", 70, 64, 1, 0), ("mxfp4", 3, 32, 40, 0),
                                           ("bf16", 70, 64, 2, 3), ("mxfp8", 9, 13, 70, 5)])
def test_many_units(fmt, L, H, tq, tn):
    # more units than 64, than 64 x 64: the search for a chunk's first unit; short segments,
    # many of them empty, so that a chunk holds several
    g = gen(L + H + tq)
    lens = torch.randint(0, 60, (L * H,), generator=g)
    lens[torch.rand(L * H, generator=g) < 0.3] = 0
    lens[-1] = 400
    cache, k, v, off = make_cache(fmt, lens.tolist(), 64, g, first=3)
    spec = ck.ProblemSpec(L, H, 1, 64, 1, [500])
    q, qd = queries(L, 1, tq, H, 64, g)
    if tn:
        kn, knd = queries(L, 1, tn, H, 64, g)
        mask = tree_mask(1, tq, tn, g)
        out, lse = ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()), with_lse=True)
        check(spec, q, off, k, v, tq, out, lse, kn, kn, mask)
    else:
        out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
        check(spec, q, off, k, v, tq, out, lse)


def test_all_segments_empty_but_the_last():
    g = gen(3)
    lens = [0] * 299 + [77]
    cache, k, v, off = make_cache("mxfp8", lens, 128, g)
    spec = ck.ProblemSpec(3, 100 // 2, 2, 128, 1, [100, 100])
    q, qd = queries(3, 2, 2, 100, 128, g)
    out, lse = ck.decode_mx(spec, qd, cache, 2, with_lse=True)
    check(spec, q, off, k, v, 2, out, lse)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
@pytest.mark.parametrize("tq,G", [(3, 2), (40, 4)])
def test_the_most_new_rows(fmt, tq, G):
    tn, g = 65536, gen(tq)
    cache, k, v, off = make_cache(fmt, [70, 0], 64, g)
    spec = ck.ProblemSpec(1, 2, G, 64, 1, [100])
    q, qd = queries(1, 1, tq, 2 * G, 64, g)
    kn, knd = queries(1, 1, tn, 2, 64, g)
    vn, vnd = queries(1, 1, tn, 2, 64, g, strided=True)
    mask = (torch.rand((1, tq, tn), generator=g) < 0.5)
    out, lse = ck.decode_tree(spec, qd, cache, tq, knd, vnd, mask.to(dev()), with_lse=True)
    check(spec, q, off, k, v, tq, out, lse, kn, vn, mask)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8"])
@pytest.mark.parametrize("G,tq", [(2, 6), (4, 8), (8, 7), (4, 30), (8, 30)])
def test_padded_queries_hold_anything(fmt, G, tq):
    # queries of a padded batch may be NaN: the others' bits are as without them
    g = gen(41 + tq * G)
    cache, k, v, off = make_cache(fmt, [333, 40, 64, 5000], 128, g)
    spec = ck.ProblemSpec(1, 2, G, 128, 1, [6000, 6000])
    q, qd = queries(1, 2, tq, 2 * G, 128, g)
    kn, knd = queries(1, 2, tq, 2, 128, g)
    mask = tree_mask(2, tq, tq, g, empty=False)
    call = lambda: ck.decode_tree(spec, qd, cache, tq, knd, knd, mask.to(dev()))  # noqa: E731
    ref = call()
    pad = slice(tq + tq // 2, 2 * tq)  # the second sequence's last queries
    qd[:, pad] = math.nan
    got = call()
    keep = [i for i in range(2 * tq) if not pad.start <= i < pad.stop]
    assert torch.equal(got[:, keep], ref[:, keep])
    assert bool(torch.isnan(got[:, pad]).all())


def test_two_streams_at_once():
    g = gen(5)
    cache, k, v, off = make_cache("mxfp8", [9000, 12000, 30, 7000], 128, g)
    spec = ck.ProblemSpec(1, 4, 4, 128, 1, [20000])
    tq, tn = 8, 40
    q, qd = queries(1, 1, tq, 16, 128, g)
    kn, knd = queries(1, 1, tn, 4, 128, g)
    mask = tree_mask(1, tq, tn, g).to(dev())
    ref = [ck.decode_mx(spec, qd, cache, tq).clone(),
           ck.decode_tree(spec, qd, cache, tq, knd, knd, mask).clone()]
    streams = [torch.cuda.Stream() for _ in range(2)]
    bufs = [ck.DecodeBuffers(spec, tq, dev(), fmt="mxfp8"),
            ck.DecodeBuffers(spec, tq, dev(), tn=tn, fmt="mxfp8")]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            ck.decode_mx(spec, qd, cache, tq, bufs=bufs[0])
        with torch.cuda.stream(streams[1]):
            ck.decode_tree(spec, qd, cache, tq, knd, knd, mask, bufs=bufs[1])
    torch.cuda.synchronize()
    assert torch.equal(bufs[0].out, ref[0]) and torch.equal(bufs[1].out, ref[1])


def test_refused_from_python():
    g = gen(6)
    cache, k, v, off = make_cache("mxfp8", [50, 20], 128, g)
    spec = ck.ProblemSpec(1, 2, 2, 128, 1, [100])
    q, qd = queries(1, 1, 2, 4, 128, g)
    two = ck.ProblemSpec(2, 2, 2, 128, 1, [100])
    bad = [lambda: ck.decode_mx(spec, qd.float(), cache, 2),
           lambda: ck.decode_mx(spec, qd, cache, 3),
           lambda: ck.decode_mx(two, qd, cache, 2),
           lambda: ck.decode_mx(spec, qd, cache, 2, bufs=ck.DecodeBuffers(spec, 2, dev())),
           lambda: ck.decode_mx(spec, qd, cache, 2, with_lse=True,
                                bufs=ck.DecodeBuffers(spec, 2, dev(), fmt="mxfp8")),
           lambda: ck.decode_mx(spec, qd, cache, 2, bufs=ck.DecodeBuffers(two, 2, dev(), fmt="mxfp8")),
           lambda: ck.decode_mx(spec, qd.cpu(), cache, 2),
           lambda: ck.read_mx(cache, first_row=60, rows=11),
           lambda: ck.read_mx(cache, out=[torch.empty((70, 64), device=dev()) for _ in range(2)]),
           lambda: ck.decode_tree(spec, qd, cache, 2, qd, qd, None),
           lambda: ck.decode_tree(spec, qd, cache, 2, qd[:, :, :2], qd[:, :, :2],
                                  torch.ones((1, 2, 3), dtype=torch.bool, device=dev()))]
    for i, call in enumerate(bad):
        with pytest.raises((AssertionError, ValueError, ck.CertKVError)):
            call()
            print("not refused:", i)
    with pytest.raises(ValueError):
        ck.MxCache.empty(spec, 5, "bf16", dev())
    with pytest.raises(ck.CertKVError):  # a workspace of a shorter call
        b = ck.DecodeBuffers(spec, 2, dev(), fmt="mxfp8")
        b.ws_bytes -= 256
        ck.decode_mx(spec, qd, cache, 2, bufs=b)

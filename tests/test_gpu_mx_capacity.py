"""A microscaled cache that has no room for the kept rows, and kept positions that are fewer
than their offsets say: nothing is written or read past either, and the call says so."""
import ctypes

import pytest
import torch

import paper_2608_21541_amd as ck
from paper_2608_21541_amd import _lib
from test_abi import FAKE, problem, tensor


def test_negative_capacities_are_refused():
    L = _lib.lib()

    def call(kept=5, rows=9, fmt=1):
        return L.certkv_compact_mx_bounded(ctypes.byref(problem()), fmt, tensor(), tensor(), FAKE,
                                           FAKE, kept, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE,
                                           rows, FAKE, None)

    assert call() == _lib.CERTKV_OK and call(kept=0, rows=0) == _lib.CERTKV_OK
    assert call(kept=-1) == _lib.CERTKV_EINVAL and call(rows=-1) == _lib.CERTKV_EINVAL
    assert call(fmt=0) == _lib.CERTKV_EINVAL


def test_the_pass_refuses_a_cache_put_in_its_buffers():
    spec = ck.ProblemSpec(1, 2, 2, 64, 4, [40])
    bufs = ck.CompressBuffers(spec, [10], "meta", fmt="mxfp8")
    x = torch.zeros((1, 40, 2, 64), dtype=torch.bfloat16)
    q = torch.zeros((1, 4, 4, 64), dtype=torch.bfloat16)
    for other in (ck.MxCache.empty(spec, bufs.rows - 1, "mxfp8", "cpu"),
                  ck.MxCache.empty(ck.ProblemSpec(1, 2, 2, 128, 4, [40]), bufs.rows, "mxfp8", "cpu")):
        bufs.mx = other
        with pytest.raises(AssertionError):
            ck.compress(spec, q, x, x, [10], bufs=bufs)


GUARD = 0x5A


def carve(fmt, rows, d, U, room, dev):
    """(cache of `rows` rows, its tensors' whole allocations): `room` bytes of guard follow each."""
    wide = d if fmt == "mxfp8" else d // 2
    whole, parts = [], []
    for n in (wide, d // 32, wide, d // 32, 4):
        t = torch.full((rows * n + room,), GUARD, dtype=torch.uint8, device=dev)
        whole.append((t, rows * n))
        parts.append(t[:rows * n].view(rows, n))
    pos = parts.pop().view(torch.int32).view(-1)
    return ck.MxCache(fmt, *parts, offsets=torch.zeros(U + 1, dtype=torch.int64, device=dev),
                      pos=pos), whole


def made(fmt, lens, L, H, d, slot, g, dev, dtype=torch.bfloat16):
    from test_gpu_mx import kept_sets
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    spec = ck.ProblemSpec(L, H, 2, d, 1, lens, dtype, slot=slot, status=status)
    k, v = (torch.randn((L, sum(lens), H, d), generator=g).to(dtype).to(dev) for _ in range(2))
    off, idx = kept_sets(lens, L, H, g)
    U = L * len(lens) * H
    star = [torch.randn((U, d), generator=g).to(dev) for _ in range(2)]
    return spec, k, v, off, idx, star


@pytest.fixture
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("d,slot,lens,L,H,dtype", [
    (128, True, [700, 33, 1025], 2, 4, torch.bfloat16),
    (64, True, [40 + i for i in range(53)], 1, 3, torch.bfloat16),
    (64, False, [5000, 2000], 2, 2, torch.float32)])
def test_rows_past_the_room_are_left_out(dev, fmt, d, slot, lens, L, H, dtype):
    g = torch.Generator()
    g.manual_seed(d + L)
    spec, k, v, off, idx, star = made(fmt, lens, L, H, d, slot, g, dev, dtype)
    run = lambda c: ck.compact_mx(spec, k, v, off.to(dev), idx.to(dev), *star, fmt, cache=c)  # noqa: E731
    U, rows = spec.units, int(off[-1]) + (spec.units if slot else 0)
    ref, _ = carve(fmt, rows, d, U, 4096, dev)
    run(ref)
    assert int(spec.status.item()) == ck.CERTKV_OK
    for room in (rows - 1, rows - 2, rows // 2, 1, rows + 3):
        cache, whole = carve(fmt, room, d, U, max(rows - room, 0) * d * 2 + 4096, dev)
        spec.status.zero_()
        run(cache)
        n = min(room, rows)
        assert int(spec.status.item()) == (ck.CERTKV_OK if room >= rows else ck.CERTKV_ERANGE)
        for t, used in whole:
            assert bool((t[used:] == GUARD).all())
        for x in ("k", "k_scales", "v", "v_scales", "pos"):
            assert torch.equal(getattr(cache, x)[:n], getattr(ref, x)[:n])
        assert torch.equal(cache.offsets, ref.offsets.clamp(max=n))
        if room > rows:
            assert bool((cache.pos[rows:].view(torch.uint8) == GUARD).all())


@pytest.mark.gpu
@pytest.mark.parametrize("slot", [True, False])
def test_positions_past_the_given_ones_are_not_read(dev, slot):
    lens, L, H, d, fmt = [700, 301], 2, 3, 64, "mxfp8"
    g = torch.Generator()
    g.manual_seed(4)
    spec, k, v, off, idx, star = made(fmt, lens, L, H, d, slot, g, dev)
    U = spec.units
    for n in (int(off[-1]) - 1, int(off[-1]) // 3, 1):
        want = ck.compact_mx(spec, k, v, off.clamp(max=n).to(dev), idx[:n].to(dev), *star, fmt)
        assert int(spec.status.item()) == ck.CERTKV_OK
        cache = ck.MxCache.empty(spec, int(off[-1]) + U, fmt, dev)
        ck.compact_mx(spec, k, v, off.to(dev), idx[:n].to(dev), *star, fmt, cache=cache)
        assert int(spec.status.item()) == ck.CERTKV_ERANGE
        spec.status.zero_()
        assert torch.equal(cache.offsets, want.offsets)
        for x in ("k", "k_scales", "v", "v_scales", "pos"):
            assert torch.equal(getattr(cache, x)[:want.rows], getattr(want, x))


@pytest.mark.gpu
def test_attention_over_what_there_was_room_for(dev):
    from test_gpu_mx import check, queries
    lens, L, H, d, fmt, tq = [900, 400], 1, 2, 128, "mxfp4", 3
    g = torch.Generator()
    g.manual_seed(9)
    spec, k, v, off, idx, star = made(fmt, lens, L, H, d, True, g, dev)
    off = torch.tensor([0, 200, 320, 321, 421])
    idx = torch.cat([torch.arange(n) for n in off.diff().tolist()]).int()
    cache = ck.MxCache.empty(spec, 300, fmt, dev)
    ck.compact_mx(spec, k, v, off.to(dev), idx.to(dev), *star, fmt, cache=cache)
    assert cache.offsets.tolist() == [0, 201, 300, 300, 300]
    kk, vv = (t.cpu().double() for t in ck.read_mx(cache))
    q, qd = queries(1, 2, tq, 2 * H, d, g)
    out, lse = ck.decode_mx(spec, qd, cache, tq, with_lse=True)
    check(spec, q, cache.offsets.cpu(), kk, vv, tq, out, lse)

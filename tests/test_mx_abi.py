"""Host-side checks of the microscaled cache's entry points (dry runs, no GPU), and of the
plain forms that their GPU tests compare with."""
import ctypes

import pytest
import torch

import _mx
import paper_2608_21541_amd as ck
from paper_2608_21541_amd import _lib
from test_abi import FAKE, problem, tensor

OK, EINVAL, EUNS, EWS = (_lib.CERTKV_OK, _lib.CERTKV_EINVAL, _lib.CERTKV_EUNSUPPORTED,
                         _lib.CERTKV_EWORKSPACE)


def cache(fmt=1, **kw):
    f = dict(k=FAKE, v=FAKE, k_scales=FAKE, v_scales=FAKE, offsets=FAKE)
    f.update(kw)
    return _lib.Cache(fmt, f["k"], f["v"], f["k_scales"], f["v_scales"], f["offsets"])


def test_compact_mx_refusals():
    L = _lib.lib()

    def call(p=None, fmt=1, k=None, v=None, off=FAKE, idx=FAKE, ks=FAKE, vs=FAKE, kc=FAKE, ksc=FAKE,
             vc=FAKE, vsc=FAKE, pos=FAKE, po=FAKE):
        p = p or problem()
        return L.certkv_compact_mx(ctypes.byref(p), fmt, k or tensor(), v or tensor(), off, idx, ks,
                                   vs, kc, ksc, vc, vsc, pos, po, None)

    assert call() == OK and call(fmt=2) == OK
    assert call(problem(dtype=_lib.CERTKV_F32, w=1)) == OK
    for fmt in (0, 3, -1):
        assert call(fmt=fmt) == EINVAL
    for name in ("off", "idx", "ks", "vs", "kc", "ksc", "vc", "vsc", "pos", "po"):
        assert call(**{name: None}) == EINVAL, name
    for name in ("kc", "vc", "ks", "vs"):
        assert call(**{name: FAKE + 8}) == EINVAL, name
    for name in ("ksc", "vsc"):
        assert call(**{name: FAKE + 2}) == EINVAL, name
    assert call(k=tensor(ptr=FAKE + 2)) == EINVAL
    assert call(v=tensor(st=4 * 128 + 4)) == EINVAL
    assert call(problem(d=96)) == EUNS
    flags = _lib.CERTKV_DRY_RUN | _lib.CERTKV_NO_SLOT
    assert call(problem(flags=flags), ks=None, vs=None) == OK


def test_read_mx_refusals():
    L = _lib.lib()

    def call(c=None, first=0, rows=5, dt=_lib.CERTKV_BF16, k=FAKE, v=FAKE, p=None):
        p = p or problem()
        return L.certkv_read_mx(ctypes.byref(p), c or cache(), first, rows, dt, k, v, None)

    assert call() == OK and call(rows=0) == OK and call(dt=_lib.CERTKV_F32) == OK
    assert call(k=None) == OK and call(v=None) == OK
    assert call(k=None, v=None) == EINVAL
    assert call(cache(0)) == EINVAL and call(cache(5)) == EINVAL
    assert call(first=-1) == EINVAL and call(rows=-1) == EINVAL
    assert call(dt=7) == EUNS
    assert call(k=FAKE + 4) == EINVAL and call(cache(k=FAKE + 1)) == EINVAL
    assert call(cache(v_scales=None)) == EINVAL and call(cache(k_scales=FAKE + 1)) == EINVAL
    assert call(cache(offsets=None)) == OK  # not read


def attend_call(name, p=None, fmt=1, tq=2, tn=3, c=None, q=None, kn=None, vn=None, mask=FAKE, out=FAKE,
                lse=None, ws=FAKE, less=0, max_rows=0, size=None):
    L = _lib.lib()
    p = p or problem()
    c = c or cache(fmt)
    n = L.certkv_decode_cache_workspace_size(ctypes.byref(p), c.format, tq,
                                             tn if name == "tree" else 0, max_rows)
    n = size if size is not None else n - less
    if name == "mx":
        return L.certkv_decode_mx(ctypes.byref(p), q or tensor(), tq, max_rows, c, out, lse, ws, n,
                                  None)
    return L.certkv_decode_tree(ctypes.byref(p), q or tensor(), tq, max_rows, c, kn or tensor(),
                                vn or tensor(), tn, mask, out, lse, ws, n, None)


@pytest.mark.parametrize("name", ["mx", "tree"])
def test_attention_refusals(name):
    call = lambda **kw: attend_call(name, **kw)  # noqa: E731
    assert call() == OK and call(fmt=2) == OK
    assert call(fmt=0) == (OK if name == "tree" else EINVAL)
    assert call(fmt=3) == EINVAL
    assert call(tq=0) == EINVAL and call(max_rows=-1) == EINVAL
    assert call(tq=256) == OK and call(tq=257, mask=FAKE) == EUNS  # 2 query heads per KV head
    assert call(p=problem(dtype=_lib.CERTKV_F32, w=1)) == EUNS
    assert call(p=problem(d=32)) == EUNS
    assert call(q=tensor(ptr=FAKE + 8)) == EINVAL and call(q=tensor(sh=4)) == EINVAL
    assert call(out=None) == EINVAL
    assert call(c=cache(offsets=None)) == EINVAL
    assert call(c=cache(k=None)) == EINVAL and call(c=cache(v=FAKE + 8)) == EINVAL
    assert call(c=cache(k_scales=None)) == EINVAL
    assert call(ws=None) == EWS and call(less=1) == EWS and call(ws=FAKE + 16) == EINVAL


def test_tree_refusals():
    call = lambda **kw: attend_call("tree", **kw)  # noqa: E731
    assert call(fmt=0, c=cache(0, k_scales=None, v_scales=None)) == OK
    assert call(tn=0, size=1 << 30) == EINVAL and call(tn=-1, size=1 << 30) == EINVAL
    assert call(tn=65536) == OK and call(tn=65537, size=1 << 40) == EUNS
    assert call(mask=None) == OK and call(mask=None, tq=4) == EINVAL
    assert call(kn=tensor(ptr=FAKE + 2)) == EINVAL and call(vn=tensor(st=12)) == EINVAL


def test_workspace_size_of_invalid_calls_is_zero():
    L = _lib.lib()
    size = lambda p, *a: L.certkv_decode_cache_workspace_size(ctypes.byref(p), *a)  # noqa: E731
    assert size(problem(), 1, 1, 0, 0) > 0 and size(problem(), 0, 4, 9, 100) > 0
    for bad in ((3, 1, 0, 0), (-1, 1, 0, 0), (1, 0, 0, 0), (1, 1, -1, 0), (1, 1, 65537, 0),
                (1, 1, 0, -1)):
        assert size(problem(), *bad) == 0
    assert size(problem(d=96), 1, 1, 0, 0) == 0


def test_plain_quantiser():
    # hand-worked blocks: the largest magnitude picks the scale, ties go to the even code
    x = torch.zeros(6, 32)
    x[0, 0] = 448.0                       # exactly the largest e4m3 code: scale 1
    x[1, 0] = 449.0                       # beyond it: scale 2, 224.5 -> 224
    x[2, 0], x[2, 1] = 6.0, 2.5           # the largest e2m1 code; 2.5 ties to 2
    x[3, 0], x[3, 1] = 7.0, -5.0          # scale 2: 3.5 ties to 4, -2.5 ties to -2
    x[5, 0] = float("inf")
    v, s = _mx.quantise(x, "mxfp8")
    assert s[:, 0].tolist() == [127, 128, 127 - 6, 127 - 6, 27, 255]
    assert v[0, 0] == 448 and v[1, 0] == 448 and v[2, 1] == 2.5 and bool(torch.isnan(v[5]).all())
    v, s = _mx.quantise(x, "mxfp4")
    assert s[2:, 0].tolist() == [127, 128, 27, 255]
    assert v[2, 1] == 2.0 and v[3, 0] == 8.0 and v[3, 1] == -4.0


def _spec_and_cache(fmt="mxfp8", **other):
    spec = ck.ProblemSpec(1, 2, 2, 64, 4, [40], dtype=torch.bfloat16)
    cache = ck.MxCache.empty(spec, 30, fmt, "cpu")
    for name, device in other.items():
        setattr(cache, name, getattr(cache, name).to(device))
    return spec, cache


@pytest.mark.parametrize("name", ["v", "k_scales", "v_scales", "offsets", "pos"])
def test_a_cache_is_on_one_device(name):
    spec, cache = _spec_and_cache()
    cache.c_cache()
    spec, cache = _spec_and_cache(**{name: "meta"})
    with pytest.raises(AssertionError):
        cache.c_cache()


@pytest.mark.parametrize("name,wrong", [
    ("k", lambda t: t[:, :39]), ("v", lambda t: t[:, :, :1]), ("kept_idx", lambda t: t.long()),
    ("kept_idx", lambda t: t.to("meta")), ("kept_offsets", lambda t: t.to("meta")),
    ("kept_offsets", lambda t: t[:-1]), ("k_star", lambda t: t.double()),
    ("v_star", lambda t: t.to("meta")), ("v_star", lambda t: t[:1])])
def test_compact_mx_refuses_other_tensors(name, wrong):
    spec, cache = _spec_and_cache()
    rows = torch.zeros((1, 40, 2, 64), dtype=torch.bfloat16)
    star = torch.zeros((2, 64))
    a = dict(k=rows, v=rows, kept_offsets=torch.tensor([0, 14, 28]),
             kept_idx=torch.zeros(28, dtype=torch.int32), k_star=star, v_star=star)
    with pytest.raises(ValueError, match="expected tensors on a GPU"):  # (these would do)
        ck.compact_mx(spec, fmt="mxfp8", cache=cache, **a)
    a[name] = wrong(a[name])
    with pytest.raises(AssertionError):
        ck.compact_mx(spec, fmt="mxfp8", cache=cache, **a)


@pytest.mark.parametrize("name", ["k", "v", "offsets", "k_new", "v_new", "mask"])
def test_decode_tree_refuses_other_devices(name):
    spec, _ = _spec_and_cache()
    packed = torch.zeros((30, 64), dtype=torch.bfloat16)
    new = torch.zeros((1, 3, 2, 64), dtype=torch.bfloat16)
    a = dict(k=packed, v=packed, offsets=torch.tensor([0, 15, 30]), k_new=new, v_new=new,
             mask=torch.ones((1, 2, 3), dtype=torch.bool))
    a[name] = a[name].to("meta")
    with pytest.raises(AssertionError):
        ck.decode_tree(spec, torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16),
                       (a["k"], a["v"], a["offsets"]), 2, a["k_new"], a["v_new"], a["mask"])

"""Host-side checks of the paged cache's entry points (dry runs, no GPU), of the binding's, and of
the plain forms that their GPU tests compare with."""
import ctypes

import pytest
import torch

import _mx
import _pages
import paper_2608_21541_amd as ck
from paper_2608_21541_amd import _lib
from test_abi import FAKE, problem, tensor

OK, EINVAL, EUNS, EWS = (_lib.CERTKV_OK, _lib.CERTKV_EINVAL, _lib.CERTKV_EUNSUPPORTED,
                         _lib.CERTKV_EWORKSPACE)


def pages(**kw):
    f = dict(format=0, page=16, num_pages=100, max_pages=9, per_head=0, s_layer=6400, s_page=64,
             s_row=4, s_head=1, k=FAKE, v=FAKE, k_scales=FAKE, v_scales=FAKE, table=FAKE,
             offsets=FAKE, ring=FAKE, free=FAKE)
    f.update(kw)
    return _lib.Pages(*[f[n] for n, _ in _lib.Pages._fields_])


UNITS = dict(per_head=1, s_layer=0, s_head=0, s_row=1, s_page=16)


def resize(p=None, g=None, change=FAKE, off=FAKE, free=FAKE, slots=FAKE, cap=10, so=FAKE, ws=FAKE,
           size=None):
    L = _lib.lib()
    p, g = p or problem(), g or pages()
    if size is None:
        size = L.certkv_page_workspace_size(ctypes.byref(p), ctypes.byref(g))
    return L.certkv_page_resize(ctypes.byref(p), ctypes.byref(g), change, off, free, slots, cap, so,
                                ws, size, None)


def write(p=None, g=None, k=None, v=None, tokens=10, tn=0, slots=FAKE, n=10, so=FAKE):
    p, g = p or problem(), g or pages()
    return _lib.lib().certkv_page_write(ctypes.byref(p), ctypes.byref(g), k or tensor(),
                                        v or tensor(), tokens, tn, slots, n, so, None)


def adopt(p=None, g=None, c=None, rows=10, slots=FAKE, n=10, so=FAKE):
    p, g = p or problem(), g or pages(**UNITS)
    c = c or _lib.Cache(g.format, FAKE, FAKE, FAKE, FAKE, None)
    return _lib.lib().certkv_page_adopt(ctypes.byref(p), ctypes.byref(g), c, rows, slots, n, so, None)


def read(p=None, g=None, rows=10, dt=1, k=FAKE, v=FAKE):
    p, g = p or problem(), g or pages()
    return _lib.lib().certkv_page_read(ctypes.byref(p), ctypes.byref(g), rows, dt, k, v, None)


def decode(p=None, g=None, q=None, tq=2, lens=None, max_rows=0, out=FAKE, lse=None, ws=FAKE, less=0,
           size=None):
    L = _lib.lib()
    p, g = p or problem(), g or pages()
    if size is None:
        size = L.certkv_decode_paged_workspace_size(ctypes.byref(p), ctypes.byref(g), tq,
                                                    max_rows) - less
    return L.certkv_decode_paged(ctypes.byref(p), q or tensor(), tq, lens, max_rows,
                                 ctypes.byref(g), out, lse, ws, size, None)


def test_resize_refusals():
    assert resize() == OK and resize(g=pages(**UNITS)) == OK
    assert resize(g=pages(k=None, v=None, s_row=0, format=9)) == OK  # not read
    for name in ("change", "off", "free", "so"):
        assert resize(**{name: None}) == EINVAL, name
    assert resize(slots=None) == EINVAL and resize(slots=None, cap=0) == OK
    assert resize(cap=-1) == EINVAL
    assert resize(cap=2 ** 31 - 1024) == OK and resize(cap=2 ** 31 - 1023) == EUNS
    assert resize(ws=None) == EWS and resize(size=0) == EWS and resize(ws=FAKE + 4) == EINVAL
    for name in ("table", "offsets", "ring", "free"):
        assert resize(g=pages(**{name: None}), size=1 << 20) == EINVAL, name


GEOMETRY = [(dict(page=8), EINVAL), (dict(page=48), EINVAL), (dict(page=2048), EINVAL),
            (dict(page=0), EINVAL), (dict(page=-16), EINVAL), (dict(num_pages=0), EINVAL),
            (dict(max_pages=0), EINVAL), (dict(max_pages=-1), EINVAL), (dict(per_head=2), EINVAL),
            (dict(num_pages=1 << 27), EUNS), (dict(max_pages=1 << 27), EUNS)]


@pytest.mark.parametrize("kw,st", GEOMETRY)
def test_geometry_is_checked_by_every_call(kw, st):
    g = pages(**kw)
    assert resize(g=g, size=1 << 20) == st and write(g=g) == st and read(g=g) == st
    assert decode(g=g, size=1 << 40) == st
    u = dict(UNITS, **kw)
    assert adopt(g=pages(**u)) == st
    L = _lib.lib()
    assert L.certkv_page_workspace_size(ctypes.byref(problem()), ctypes.byref(g)) == 0
    assert L.certkv_decode_paged_workspace_size(ctypes.byref(problem()), ctypes.byref(g), 1, 0) == 0


@pytest.mark.parametrize("kw,st", [
    (dict(format=3), EINVAL), (dict(format=-1), EINVAL), (dict(k=None), EINVAL),
    (dict(v=FAKE + 8), EINVAL), (dict(format=1, k_scales=None), EINVAL),
    (dict(format=2, v_scales=FAKE + 2), EINVAL), (dict(s_row=0), EINVAL), (dict(s_page=-1), EINVAL),
    (dict(s_layer=-1), EINVAL), (dict(s_head=-1), EINVAL), (dict(s_row=1 << 20), EUNS),
    (dict(s_page=1 << 50), EUNS), (dict(s_layer=1 << 52), EUNS), (dict(s_head=1 << 52), EUNS),
    (dict(UNITS, s_layer=64), EINVAL), (dict(UNITS, s_head=1), EINVAL)])
def test_rows_of_the_pool_are_checked(kw, st):
    g = pages(**kw)
    assert write(g=g, tn=5) == st and read(g=g) == st and decode(g=g, size=1 << 40) == st
    assert resize(g=g) == OK


def test_write_refusals():
    assert write() == OK and write(tn=5) == OK and write(g=pages(**UNITS), tn=5) == OK
    assert write(tokens=0, n=0, slots=None) == OK
    assert write(problem(dtype=_lib.CERTKV_F32, w=1)) == OK
    assert write(g=pages(**UNITS)) == EINVAL  # units' lists take tokens of a number for each
    assert write(tn=4) == EINVAL and write(tn=-5) == EINVAL and write(tokens=-1) == EINVAL
    assert write(so=None) == EINVAL and write(slots=None) == EINVAL and write(n=-1) == EINVAL
    assert write(k=tensor(ptr=FAKE + 2)) == EINVAL and write(v=tensor(st=12)) == EINVAL
    assert write(tokens=1 << 30) == EUNS and write(problem(d=96)) == EUNS


def test_adopt_refusals():
    assert adopt() == OK and adopt(g=pages(format=1, **UNITS)) == OK
    assert adopt(rows=0) == OK
    assert adopt(g=pages()) == EINVAL  # sequences' lists
    assert adopt(c=_lib.Cache(1, FAKE, FAKE, FAKE, FAKE, None)) == EINVAL  # another format
    assert adopt(c=_lib.Cache(0, None, FAKE, None, None, None)) == EINVAL
    assert adopt(c=_lib.Cache(0, FAKE, FAKE + 8, None, None, None)) == EINVAL
    assert adopt(rows=-1) == EINVAL and adopt(so=None) == EINVAL and adopt(slots=None) == EINVAL


def test_read_refusals():
    assert read() == OK and read(dt=0) == OK and read(rows=0, k=None, v=None) == OK
    assert read(k=None) == OK and read(v=None) == OK and read(k=None, v=None) == EINVAL
    assert read(dt=5) == EUNS and read(rows=-1) == EINVAL and read(k=FAKE + 8) == EINVAL
    assert read(rows=1 << 45) == EUNS


def test_decode_refusals():
    assert decode() == OK and decode(lens=FAKE, lse=FAKE, max_rows=7) == OK
    assert decode(g=pages(format=1)) == OK and decode(g=pages(format=2, **UNITS)) == OK
    assert decode(tq=0) == EINVAL and decode(max_rows=-1) == EINVAL
    assert decode(tq=256) == OK and decode(tq=257, size=1 << 40) == EUNS  # 2 heads to a KV head
    assert decode(problem(dtype=_lib.CERTKV_F32, w=1), size=1 << 40) == EUNS
    assert decode(q=tensor(ptr=FAKE + 8)) == EINVAL and decode(q=tensor(sh=4)) == EINVAL
    assert decode(out=None) == EINVAL
    assert decode(ws=None) == EWS and decode(less=1) == EWS and decode(ws=FAKE + 16) == EINVAL


def test_problem_is_checked():
    bad = problem()
    bad.flags |= 1 << 12
    for p, st in ((problem(d=32), EUNS), (problem(H=65), EUNS), (bad, EINVAL)):
        assert resize(p, size=1 << 20) == st and write(p) == st and read(p) == st
        assert decode(p, size=1 << 40) == st
    # lengths of the problem's sequences are not read
    p = problem()
    p.cu_seqlens_host = None
    p.window = 0
    assert resize(p) == OK and write(p) == OK and decode(p) == OK and read(p) == OK


@pytest.mark.parametrize("L,B,num,page,most,tq,mib", [
    (1, 64, 1 << 16, 16, 8192, 1, 45),      # lists that may be longer than the pool is large
    (32, 8, 1 << 13, 128, 1024, 1, 80), (1, 1, 64, 16, 64, 1, 5), (1, 64, 1 << 16, 16, 8192, 8, 45)])
def test_decode_workspace(L, B, num, page, most, tq, mib):
    # Partials for the pieces that lists within the pool can have.
    lib = _lib.lib()
    p = problem(L=L, seqlens=(100,) * B, H=8, G=4, w=1)
    g = pages(num_pages=num, page=page, max_pages=most, s_row=8, s_page=8 * page,
              s_layer=8 * page * num)
    size = lib.certkv_decode_paged_workspace_size(ctypes.byref(p), ctypes.byref(g), tq, 0)
    assert 0 < size <= mib * 2 ** 20


def test_plain_lists():
    # by hand: two lists of pages of 16 from a ring of four
    x = _pages.Lists(2, 4, 16, 3, ring=[3, 1, 0, 2])
    assert x.resize([17, 1], 100) == ([48 + i for i in range(16)] + [16, 0], [0, 17, 18], False)
    assert x.table[0][:2] == [3, 1] and x.table[1][0] == 0 and (x.head, x.count) == (3, 1)
    # list 0 gives a page, free from the next step on; list 1 takes the last one
    assert x.resize([-1, 16], 100) == (list(range(1, 16)) + [32], [0, 0, 16], False)
    assert (x.head, x.count, x.ring) == (0, 1, [1, 1, 0, 2]) and x.rows == [16, 17]
    assert x.resize([1, 40], 100)[0] == [16] + [-1] * 40 and x.rows == [17, 17]
    assert x.resize([3, 3], 2) == ([-1] * 6, [0, 3, 6], True)


def test_plain_codes():
    gen = torch.Generator().manual_seed(5)
    for fmt in ("mxfp8", "mxfp4"):
        x = torch.randn((7, 64), generator=gen)
        v, _ = _mx.quantise(x, fmt)
        assert torch.equal(_mx.decode_codes(*_pages.encode(x, fmt), fmt), v)


def _cpu(fmt="bf16", per_head=False, **kw):
    spec = ck.ProblemSpec(2, 2, 2, 64, 1, [1, 1], **kw)
    return spec, ck.PagedCache.empty(spec, 9, 16, 4, "cpu", fmt, per_head=per_head)


GPU = pytest.raises(ValueError, match="expected tensors on a GPU")  # (the arguments would do)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("per_head", [False, True])
def test_strides_are_counted_in_rows(fmt, per_head):
    spec, cache = _cpu(fmt, per_head)
    c = cache._c_pages(spec)[1]
    got = (c.s_layer, c.s_page, c.s_row, c.s_head)
    assert got == ((0, 16, 1, 0) if per_head else (9 * 16 * 2, 32, 2, 1))
    if not per_head:
        other = ck.PagedCache.empty(spec, 9, 16, 4, "cpu", fmt, head_major=True)
        c = other._c_pages(spec)[1]
        assert (c.s_layer, c.s_page, c.s_row, c.s_head) == (9 * 32, 32, 1, 16)
        one = other.layer(1, 2)
        c = one._c_pages(ck.ProblemSpec(1, 2, 2, 64, 1, [1, 1]))[1]
        assert (c.s_layer, c.s_page, c.s_row, c.s_head) == (0, 32, 1, 16)
        assert c.k == other.k[1].data_ptr() and c.num_pages == 9


@pytest.mark.parametrize("name,wrong", [
    ("k", lambda t: t[:1]), ("v", lambda t: t.float()), ("table", lambda t: t.long()),
    ("table", lambda t: t[:1]), ("offsets", lambda t: t[:-1]), ("offsets", lambda t: t.to("meta")),
    ("v", lambda t: t.to("meta")), ("v", lambda t: t.transpose(2, 3).contiguous().transpose(2, 3)),
    ("ring", lambda t: t[:-1]), ("free", lambda t: t.int()), ("k", lambda t: t[..., :32])])
def test_the_caches_tensors_are_checked(name, wrong):
    spec, cache = _cpu()
    q = torch.zeros((2, 2, 4, 64), dtype=torch.bfloat16)
    with GPU:
        ck.decode_paged(spec, q, cache, 1, bufs=_bufs(spec, cache, q))
    bufs = _bufs(spec, cache, q)
    setattr(cache, name, wrong(getattr(cache, name)))
    with pytest.raises(AssertionError):
        ck.decode_paged(spec, q, cache, 1, bufs=bufs)


def _bufs(spec, cache, q, tq=1):
    b = ck.DecodeBuffers.__new__(ck.DecodeBuffers)
    b.tq, b.max_rows, b.tn, b.fmt, b.paged = tq, 0, 0, None, True
    b.out, b.lse, b.ws, b.ws_bytes = torch.zeros_like(q, dtype=torch.float32), None, q, 0
    return b


def test_decode_paged_refuses_other_tensors():
    spec, cache = _cpu()
    q = torch.zeros((2, 4, 4, 64), dtype=torch.bfloat16)
    lens = torch.tensor([1, 2], dtype=torch.int32)
    call = lambda **kw: ck.decode_paged(spec, kw.pop("q", q), cache, 2, bufs=kw.pop(  # noqa: E731
        "bufs", _bufs(spec, cache, q, 2)), **kw)
    with GPU:
        call(q_lens=lens)
    for kw in (dict(q=q[:, :2]), dict(q=q.float()), dict(q_lens=lens.long()),
               dict(q_lens=lens[:1]), dict(q_lens=lens.to("meta")), dict(with_lse=True),
               dict(bufs=_bufs(spec, cache, q, 1))):
        with pytest.raises(AssertionError):
            call(**kw)


def test_page_calls_refuse_other_tensors():
    spec, cache = _cpu()
    rows = torch.zeros((2, 5, 2, 64), dtype=torch.bfloat16)
    slots, so = torch.zeros(5, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    with GPU:
        ck.page_write(spec, cache, rows, rows, slots, so)
    for a in ((rows[:1], rows, slots, so), (rows, rows.float(), slots, so),
              (rows, rows.to("meta"), slots, so), (rows, rows, slots.long(), so),
              (rows, rows, slots, so[:-1]), (rows, rows, slots.to("meta"), so)):
        with pytest.raises(AssertionError):
            ck.page_write(spec, cache, *a)
    change = torch.zeros(2, dtype=torch.int32)
    bufs = ck.ResizeBuffers(cache, 5, "cpu")
    with GPU:
        ck.page_resize(spec, cache, change, bufs=bufs)
    for bad in (change.long(), change[:1], torch.zeros((2, 2), dtype=torch.int32)[:, 0]):
        with pytest.raises(AssertionError):
            ck.page_resize(spec, cache, bad, bufs=bufs)
    for into in ((cache.offsets[:-1], cache.free), (cache.offsets, cache.free.int())):
        with pytest.raises(AssertionError):
            ck.page_resize(spec, cache, change, bufs=bufs, into=into)
    with GPU:
        ck.page_read(spec, cache, rows=3)
    with pytest.raises(AssertionError):
        ck.page_read(spec, cache, out=[rows[..., :32], rows[..., :32]])
    spec, cache = _cpu(per_head=True)
    packed = torch.zeros((5, 64), dtype=torch.bfloat16)
    so = torch.zeros(9, dtype=torch.int64)
    with GPU:
        ck.page_adopt(spec, cache, (packed, packed, so), slots, so)
    for p in ((packed, packed[:3], so), (packed.float(), packed.float(), so),
              (packed[:, ::2], packed[:, ::2], so)):
        with pytest.raises(AssertionError):
            ck.page_adopt(spec, cache, p, slots, so)
    with pytest.raises(AssertionError):
        ck.page_adopt(spec, cache, ck.MxCache.empty(spec, 5, "mxfp8", "cpu"), slots, so)

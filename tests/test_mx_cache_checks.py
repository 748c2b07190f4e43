"""What the Python binding refuses of a microscaled cache's description before any call."""
import pytest
import torch

import paper_2608_21541_amd as ck


def spec_and_cache(fmt, d=128, rows=30):
    spec = ck.ProblemSpec(1, 2, 2, d, 4, [40])
    return spec, ck.MxCache.empty(spec, rows, fmt, "cpu")


@pytest.mark.parametrize("fmt", ["bf16", "fp8", None])
@pytest.mark.parametrize("made", [False, True])
def test_a_cache_of_another_format_is_refused(fmt, made):
    # codes of 4 bits with the scales of their rows: as bf16 rows they would be four times as long
    spec, c = spec_and_cache("mxfp4")
    if made:
        c = ck.MxCache(fmt, c.k, c.k_scales, c.v, c.v_scales, c.offsets, c.pos)
    else:
        c.format = fmt
    q = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    new = torch.zeros((1, 2, 2, 128), dtype=torch.bfloat16)
    for call in (c.c_cache, lambda: ck.decode_tree(spec, q, c, 2, new, new),
                 lambda: ck.decode_mx(spec, q, c, 2), lambda: ck.read_mx(c)):
        with pytest.raises((AssertionError, ValueError)) as e:
            call()
        assert "expected tensors on a GPU" not in str(e.value)  # (refused before that)


def test_a_problem_that_its_caller_changes_is_the_callers_own():
    spec, _ = spec_and_cache("mxfp8")
    size = lambda: ck.decode_cache_workspace_size(spec, "mxfp8", 1)  # noqa: E731
    want = size()
    for p in (spec.c_problem(), spec.c_problem(), ck.CompressBuffers(spec, [10], "meta")._p):
        p.head_dim, p.cu_seqlens_host[1] = 96, 7
        assert size() == want
        q = spec.c_problem()
        assert (q.head_dim, q.cu_seqlens_host[1]) == (128, 40)
    # and a changed field is seen
    spec.seqlens[0] = 70000
    assert size() > want
    spec.seqlens[0], spec.layers = 40, 3
    assert size() > want


@pytest.mark.parametrize("name", ["k", "k_scales", "v", "v_scales", "pos"])
@pytest.mark.parametrize("how", ["data", "set"])
def test_a_tensor_changed_in_place_is_checked_again(name, how):
    spec, c = spec_and_cache("mxfp8")
    c.c_cache()
    t = getattr(c, name)
    less = t[:29].clone()
    if how == "data":
        t.data = less
    else:
        t.set_(less.untyped_storage(), 0, less.shape, less.stride())
    assert len(getattr(c, name)) == 29
    with pytest.raises(AssertionError):
        c.c_cache()
    for other in ("k", "k_scales", "v", "v_scales"):  # and all of one size will do
        setattr(c, other, getattr(c, other)[:29])
    c.c_cache()


@pytest.mark.parametrize("rows", [29, 31, 3000])
def test_keys_resized_in_place_are_checked_again(rows):
    spec, c = spec_and_cache("mxfp4", rows=3000)  # (room for what it grows to)
    c = ck.MxCache("mxfp4", c.k[:30], c.k_scales[:30].clone(), c.v[:30].clone(),
                   c.v_scales[:30].clone(), c.offsets, c.pos[:30].clone())
    c.c_cache()
    c.k.resize_((rows, 64))
    with pytest.raises(AssertionError):
        c.c_cache()


def test_decode_refuses_outputs_of_fewer_queries():
    spec, _ = spec_and_cache("mxfp8")
    packed = torch.zeros((30, 128), dtype=torch.bfloat16)
    q = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    bufs = ck.DecodeBuffers(spec, 1, "meta")
    with pytest.raises(AssertionError):
        ck.decode(spec, q, packed, packed, torch.zeros(3, dtype=torch.int64), 2, bufs=bufs)

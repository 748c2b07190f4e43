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

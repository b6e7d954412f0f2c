"""Calls on a whole cache without a device: what they refuse before they touch one."""
import ctypes as C

import pytest

from paper_2506_15969_b200 import binding


@pytest.fixture
def handle():
    lib, h = binding.lib(), C.c_void_p()
    assert lib.lazyev_create(C.byref(h), 2, 8, 2, 128, 512, 128, 1e-3) == binding.OK
    yield h
    assert lib.lazyev_destroy(h) == binding.OK


def test_weights_are_asked_for_before_they_are_a_score(handle):
    lib, at, size = binding.lib(), C.c_size_t(), C.c_size_t()
    assert lib.lazyev_set_score_mode(handle, binding.SCORE_WEIGHT) == binding.EINVAL and b"weights" in lib.lazyev_last_error(handle)
    assert lib.lazyev_query_weights_layout(handle, C.byref(at)) == binding.ESTATE
    lib.lazyev_query_sizes(handle, None, C.byref(size), None)
    plain = size.value
    assert lib.lazyev_set_weights(handle, 1) == binding.OK
    assert lib.lazyev_set_score_mode(handle, binding.SCORE_WEIGHT) == binding.OK
    assert lib.lazyev_set_score_mode(handle, 5) == binding.EINVAL
    assert lib.lazyev_set_weights(handle, 0) == binding.EINVAL              # it is the score
    lib.lazyev_query_sizes(handle, None, C.byref(size), None)
    info = binding.Info()
    lib.lazyev_get_info(handle, C.byref(info))
    assert lib.lazyev_query_weights_layout(handle, C.byref(at)) == binding.OK
    assert at.value == plain and at.value % 256 == 0 and size.value >= plain + 4 * info.units * info.capacity
    assert lib.lazyev_set_score_mode(handle, 0) == binding.OK and lib.lazyev_set_weights(handle, 0) == binding.OK
    lib.lazyev_query_sizes(handle, None, C.byref(size), None)
    assert size.value == plain
    assert lib.lazyev_set_weights(None, 1) == binding.EINVAL and lib.lazyev_query_weights_layout(handle, None) == binding.EINVAL


def test_calls_that_need_a_bound_handle(handle):
    lib, n, evicted = binding.lib(), C.c_size_t(), C.c_int(7)
    assert lib.lazyev_query_chunk_workspace(handle, 4, 0, C.byref(n)) == binding.ESTATE
    assert lib.lazyev_attend_chunk(handle, 256, 4, 256, 0, 256) == binding.ESTATE
    assert lib.lazyev_set_block_workspace(handle, 256) == binding.ESTATE
    assert lib.lazyev_index_blocks(handle, 0) == binding.ESTATE
    assert lib.lazyev_attend_sparse(handle, 256, 2, 256, None) == binding.ESTATE
    assert lib.lazyev_evict_to(handle, 200, None, C.byref(evicted)) == binding.ESTATE and evicted.value == 0
    for call, args in (("query_chunk_workspace", (4, 0, C.byref(n))), ("attend_chunk", (256, 4, 256, 0, 256)), ("set_block_workspace", (256,)),
                       ("index_blocks", (0,)), ("attend_sparse", (256, 2, 256, None)), ("evict_to", (200, None, None)),
                       ("query_block_workspace", (C.byref(n), None))):
        assert getattr(lib, "lazyev_" + call)(None, *args) == binding.EINVAL
    assert lib.lazyev_query_chunk_workspace(handle, 4, 0, None) == binding.EINVAL
    assert lib.lazyev_query_block_workspace(handle, None, None) == binding.EINVAL


def test_block_workspace_holds_bounds_keys_and_pages(handle):
    lib, n, at, info = binding.lib(), C.c_size_t(), C.c_size_t(7), binding.Info()
    lib.lazyev_get_info(handle, C.byref(info))
    assert lib.lazyev_query_block_workspace(handle, C.byref(n), C.byref(at)) == binding.OK
    pages = info.units * info.pages_per_unit
    assert at.value == 0 and n.value >= pages * (512 + 8 + 4) + 4 * info.units * info.capacity


def test_a_chunks_plan_needs_a_bound_handle(handle):
    lib, plan = binding.lib(), (C.c_int * 5)()
    assert lib.lazyev_debug_chunk_plan(handle, 100, 4, plan) == binding.ESTATE and b"bind" in lib.lazyev_last_error(handle)
    assert lib.lazyev_debug_chunk_plan(None, 100, 4, plan) == binding.EINVAL
    assert lib.lazyev_debug_chunk_plan(handle, 100, 4, None) == binding.EINVAL

"""Operators on a cache kept in pages, without a GPU: what a plan refuses, and what the calls refuse before they touch the device."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2305_13484_amd as fl
from paper_2305_13484_amd.binding import _PagedShape


def plan_bytes(shape, new, lens, table):
    new, lens, table = (np.ascontiguousarray(x, np.int32) for x in (new, lens, table))
    n = C.c_uint64()
    lib = fl.load_library()
    rc = lib.flover_k_paged_plan_bytes(C.byref(shape), len(new), new.ctypes.data, lens.ctypes.data, table.ctypes.data,
                                       table.shape[1] if table.ndim == 2 else 0, C.byref(n))
    return rc, n.value, (lib.flover_last_error(None) or b"").decode()


def shape(**kw):
    s = dict(dtype=2, n_head=8, n_kv_head=2, head_dim=128, page_size=16, n_pages=10, window=0, sinks=0)
    s.update(kw)
    return _PagedShape(*[s[n] for n, _ in _PagedShape._fields_])


@pytest.mark.parametrize("bad,why", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(n_head=9), "n_head"), (dict(n_kv_head=0), "n_head"), (dict(n_head=0), "n_head"),
    (dict(head_dim=96), "head_dim"), (dict(page_size=0), "page_size"), (dict(n_pages=0), "n_pages"), (dict(window=-1), "window"),
    (dict(sinks=-1), "sinks"), (dict(n_pages=1 << 26, page_size=16), "2^31")])
def test_shapes_that_are_refused(bad, why):
    rc, _, text = plan_bytes(shape(**bad), [1], [5], [[0]])
    assert rc == -1 and why in text
    h = C.c_void_p()
    s = shape(**bad)
    assert fl.load_library().flover_k_paged_plan_create(C.byref(s), C.byref(h)) == -1 and not h.value


@pytest.mark.parametrize("new,lens,table,why", [
    ([1], [17], [[0]], "beyond the page table"), ([6], [5], [[0]], "new_len"), ([-1], [5], [[0]], "new_len"), ([0], [-1], [[0]], "new_len"),
    ([1], [5], [[10]], "out of range"), ([1], [5], [[-1]], "out of range"), ([1, 1], [5, 40], [[0, 99, 99], [1, 2, -3]], "out of range of sequence 1")])
def test_lists_that_are_refused(new, lens, table, why):
    rc, _, text = plan_bytes(shape(), new, lens, table)
    assert rc == -1 and why in text


def test_pages_of_any_size_only_where_no_sequence_has_a_second():
    assert plan_bytes(shape(page_size=100), [1], [100], [[3]])[0] == 0
    rc, _, text = plan_bytes(shape(page_size=100), [1], [101], [[3, 4]])
    assert rc == -1 and "multiple of 16" in text


def test_entries_behind_the_last_page_are_not_read_and_empty_lists_are_fine():
    rc, n, _ = plan_bytes(shape(), [0, 2, 0], [0, 20, 3], [[-5, -5], [1, 2], [4, 1000000]])
    assert rc == 0 and n >= 256
    assert plan_bytes(shape(), np.zeros(0), np.zeros(0), np.zeros((0, 0)))[0] == 0


def test_lists_that_no_launch_could_take():
    table = [list(range(1 << 15))]
    rc, _, text = plan_bytes(shape(page_size=1 << 15, n_pages=1 << 15, n_kv_head=1), [0], [1 << 30], table)
    assert rc == -1 and "2^30" in text
    rc, _, text = plan_bytes(shape(page_size=1 << 20, n_pages=1 << 10, n_kv_head=1), [1 << 29], [1 << 29], [list(range(1 << 9))])
    assert rc == -1 and "too many new tokens" in text


def test_room_grows_with_keys_shared_out():
    """One long sequence: partial results of 16 rows per part and key head; many even ones: none, a work item of 80 bytes and the lists."""
    long = plan_bytes(shape(n_pages=4096), [1], [16 * 4000], [list(range(4000))])[1]
    many = plan_bytes(shape(n_pages=4096), [1] * 2000, [16] * 2000, [[i] for i in range(2000)])[1]
    assert long > 2 * 16 * 130 * 4 * 8 and many < 2000 * 128


def test_binding_checks_lists_before_the_device():
    with pytest.raises(fl.FloverError, match="out of range"):
        fl.PagedPlan(torch.bfloat16, 8, 2, 128, 16, 10, [1], [5], [[10]])
    with pytest.raises(fl.FloverError, match="n_seq"):
        fl.PagedPlan(torch.bfloat16, 8, 2, 128, 16, 10, [1, 1], [5], [[1]])
    with pytest.raises(fl.FloverError, match="beyond"):
        fl.PagedPlan(torch.bfloat16, 8, 2, 128, 16, 10, [1, 1], [5, 20], [[1], [2]])
    with pytest.raises(fl.FloverError, match="float32, float16 or bfloat16"):
        fl.PagedPlan(torch.float64, 8, 2, 128, 16, 10, [1], [5], [[1]])


def test_calls_refuse_a_missing_or_unset_plan():
    lib = fl.load_library()
    h = C.c_void_p()
    s = shape()
    assert lib.flover_k_paged_plan_create(C.byref(s), C.byref(h)) == 0
    for plan, code in ((None, -1), (h, -4)):
        assert lib.flover_k_paged_append(plan, None, 0, None, 0, None, None, None) == code
        assert lib.flover_k_paged_attention(plan, None, 0, None, None, None, None, None) == code
        assert lib.flover_k_paged_weights(plan, None, 0, None, None, 1.0, None, 0, None) == code
        assert lib.flover_k_paged_evict(plan, None, None, None, 0, 1, 0, 0, None, 0, None, None) == code
    one = np.array([1], np.int32)
    assert lib.flover_k_paged_plan_set(h, 1, one.ctypes.data, one.ctypes.data, one.ctypes.data, 1, None, 0, None) == -1
    assert lib.flover_k_paged_plan_set(h, 1, one.ctypes.data, one.ctypes.data, one.ctypes.data, 1, 128, 1 << 20, None) == -1
    assert lib.flover_k_paged_plan_set(h, 1, one.ctypes.data, one.ctypes.data, one.ctypes.data, 1, 256, 16, None) == -3
    assert lib.flover_k_paged_plan_destroy(h) == 0 and lib.flover_k_paged_plan_destroy(None) == 0

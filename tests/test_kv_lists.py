"""Lists of cache rows and of page copies, and the copies that put a pool in order: what is built, and what is refused (CPU)."""

import ctypes
import os
import shutil

import numpy as np
import pytest

from paper_2404_00242_amd import binding, workloads as wl
from tests.test_sanitizers import ROOT, SAN, run

EINVAL = -1


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_lists_under_the_sanitizers(tmp_path):
    # the driver makes the copies of random lists chain by chain, in any order of the chains, and compares pages; see there
    exe = str(tmp_path / "lists_driver")
    csrc = os.path.join(ROOT, "paper_2404_00242_amd", "csrc")
    run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "deft_lists.cpp"),
         os.path.join(ROOT, "tests", "sanitize", "lists_driver.cpp"), "-o", exe])
    assert "lists ok" in run([exe])


@pytest.mark.parametrize("rows,pool,block", [([0, 4], 4, 1), ([-1], 4, 1), ([3, 1, 3], 4, 2), ([1, 1], 4, 64), ([0], 0, 1), ([0], 4, 0),
                                             ([0], 4, 3), ([0], 4, 128), ([0], -1, 1), ([1 << 32], 4, 1), ([-(1 << 32) + 1], 4, 1), ([0.5], 4, 1),
                                             (["0"], 4, 1)])
def test_row_lists_that_are_refused(rows, pool, block):
    with pytest.raises(binding.DeftError) as e:
        binding.deft_kv_rows(rows, pool, block)
    assert e.value.status == EINVAL


@pytest.mark.parametrize("src,dst,pool", [([0, 1], [2, 2], 4), ([4], [0], 4), ([0], [4], 4), ([-1], [0], 4), ([0], [-1], 4), ([0], [0], 0),
                                          ([1, 1], [1, 1], 4), ([0, 1], [2], 4), ([1 << 33], [0], 4), ([0], [(1 << 32) + 1], 4)])
def test_copies_that_are_refused(src, dst, pool):
    with pytest.raises(binding.DeftError) as e:
        binding.deft_kv_copies(src, dst, pool)
    assert e.value.status == EINVAL


def test_null_arguments_are_refused():
    lib = binding.load_library()
    out = ctypes.c_void_p(1)
    one = (ctypes.c_int32 * 1)(0)
    assert lib.deft_kv_rows(None, 1, 4, 1, ctypes.byref(out)) == EINVAL and not out.value
    assert lib.deft_kv_rows(one, -1, 4, 1, ctypes.byref(out)) == EINVAL
    assert lib.deft_kv_rows(one, 1, 4, 1, None) == EINVAL
    assert lib.deft_kv_copies(None, one, 1, 4, ctypes.byref(out)) == EINVAL
    assert lib.deft_kv_copies(one, None, 1, 4, ctypes.byref(out)) == EINVAL
    assert lib.deft_kv_copies(one, one, 1, 4, None) == EINVAL
    assert lib.deft_kv_list_device_bytes(None) == 0
    assert lib.deft_kv_list_upload(None, None, 0, None) == EINVAL
    lib.deft_kv_list_destroy(None)
    # empty lists are lists
    assert binding.deft_kv_rows([], 0, 1).n == 0 and binding.deft_kv_copies([], [], 0).n == 0


def _cache(k=1 << 12, v=1 << 13, ks=16, vs=16, n_rows=64, Hkv=2, d=64, block=16):
    return binding._pack_cache(k, v, ks, vs, n_rows, Hkv, d, block)


@pytest.mark.parametrize("bad", [dict(k=0), dict(v=0), dict(ks=0), dict(vs=0), dict(k=8), dict(v=24), dict(ks=17), dict(vs=18), dict(n_rows=63), dict(Hkv=0), dict(Hkv=65537), dict(d=96),
                                 dict(block=8), dict(block=48), dict(block=0), dict(n_rows=-1)])
def test_calls_refuse_a_cache_that_is_none_or_not_the_lists(bad):
    # all of these are refused before anything is launched: no address here is one
    lib = binding.load_library()
    rows = binding.deft_kv_rows([3, 63], 64, 16)
    x = ctypes.c_void_p(1 << 14)
    c = _cache(**bad)
    assert lib.deft_kv_store_q8(rows.handle, x, x, x, 128, 128, c, None) == EINVAL
    assert lib.deft_kv_load_q8(rows.handle, x, c, x, x, None) == EINVAL


def test_calls_refuse_other_arguments():
    lib = binding.load_library()
    rows, copies = binding.deft_kv_rows([3, 63], 64, 16), binding.deft_kv_copies([0], [1], 4)
    x, y, odd = ctypes.c_void_p(1 << 14), ctypes.c_void_p(1 << 15), ctypes.c_void_p((1 << 14) + 8)
    c = _cache(vs=32)
    for same in (dict(v=1 << 12, vs=32), dict()):  # K and V, or their scales, in one place
        assert lib.deft_kv_store_q8(rows.handle, x, x, x, 128, 128, _cache(**same), None) == EINVAL
    assert lib.deft_kv_load_q8(rows.handle, x, c, y, y, None) == EINVAL
    store = lambda *a: lib.deft_kv_store_q8(*a, c, None)  # noqa: E731
    for k_stride, v_stride in ((120, 128), (128, 120), (132, 128), (128, 130), (-128, 128)):
        assert store(rows.handle, x, x, x, k_stride, v_stride) == EINVAL
    for args in ((None, x, x, x), (copies.handle, x, x, x), (rows.handle, None, x, x), (rows.handle, odd, x, x), (rows.handle, x, None, x),
                 (rows.handle, x, x, None), (rows.handle, x, odd, x), (rows.handle, x, x, odd)):
        assert store(*args, 128, 128) == EINVAL
    for args in ((None, x, x, x), (copies.handle, x, x, x), (rows.handle, None, x, x), (rows.handle, x, odd, x), (rows.handle, x, x, odd)):
        assert lib.deft_kv_load_q8(args[0], args[1], c, args[2], args[3], None) == EINVAL
    assert lib.deft_kv_store_q8(rows.handle, x, x, x, 128, 128, None, None) == EINVAL

    def copy(lst, image, pools, sizes):
        n = len(pools)
        return lib.deft_kv_copy_pages(lst, image, (ctypes.c_void_p * max(1, n))(*pools), (ctypes.c_int64 * max(1, n))(*sizes), n, None)

    base = 1 << 20
    assert copy(rows.handle, x, [base], [16]) == EINVAL
    assert copy(None, x, [base], [16]) == EINVAL
    assert copy(copies.handle, None, [base], [16]) == EINVAL
    assert copy(copies.handle, odd, [base], [16]) == EINVAL
    assert copy(copies.handle, x, [0], [16]) == EINVAL
    assert copy(copies.handle, x, [base], [0]) == EINVAL
    assert copy(copies.handle, x, [base, base], [16, 16]) == EINVAL       # the same pool twice
    assert copy(copies.handle, x, [base + 63, base], [16, 16]) == EINVAL  # the second ends inside the first
    assert copy(copies.handle, x, [base], [1 << 62]) == EINVAL
    assert lib.deft_kv_copy_pages(copies.handle, x, None, None, 1, None) == EINVAL
    assert lib.deft_kv_copy_pages(copies.handle, x, None, None, -1, None) == EINVAL
    assert copy(copies.handle, x, [], []) == 0


def test_attention_refuses_a_cache_that_is_none_or_too_small():
    lib = binding.load_library()
    plan = binding.deft_plan([0], [60], [-1], [0], 60)
    x = ctypes.c_void_p(1 << 14)
    call = lambda c: lib.deft_tree_attn_decode_q8(plan.handle, x, x, c, x, 2, 0.0, 0, x, 1 << 20, None)  # noqa: E731
    assert call(None) == EINVAL
    for bad in (dict(k=0), dict(vs=0), dict(v=8), dict(block=24), dict(d=32), dict(n_rows=59), dict(Hkv=3)):
        assert call(_cache(**bad)) == EINVAL
    assert call(_cache()) == -5  # a cache that is one; the plan has no image yet
    assert lib.deft_tree_attn_decode_q8(None, x, x, _cache(), x, 2, 0.0, 0, x, 1 << 20, None) == EINVAL


def test_binding_refuses_host_tensors():
    import torch

    c = binding.alloc_kv_cache_q8(32, 2, 64, 16, device="cpu")
    assert c.k.shape == (32, 2, 64) and c.k_scale.shape == (2, 2) and bool((c.v_scale.view(torch.uint8) == 10).all())
    rows = binding.deft_kv_rows([1], 32, 16)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    plan = binding.deft_plan([0], [8], [-1], [0], 8)
    for call in (lambda: binding.deft_kv_store_q8(rows, x, x, c), lambda: binding.deft_kv_load_q8(rows, c),
                 lambda: binding.deft_tree_attn_decode_q8(plan, x, c), lambda: binding.deft_kv_copy_pages(binding.deft_kv_copies([0], [1], 2), [x])):
        with pytest.raises(binding.DeftError):
            call()
    for block in (0, 3, 128):
        with pytest.raises(binding.DeftError):
            binding.alloc_kv_cache_q8(32, 2, 64, block, device="cpu")


@pytest.mark.parametrize("seed", range(6))
def test_a_pool_in_order_has_every_nodes_pages_in_a_row_depth_first(seed):
    t = wl.random_tree(seed, n_nodes=17, max_len=60, nq=11, n_roots=1 + seed % 3)
    ptr, ids, n_pool, _ = wl.to_paged(t, 8, seed)
    new, src, dst = binding.deft_compact_pages(ptr, ids, n_pool, t.node_parent)
    pages = np.arange(n_pool)
    pages[dst] = src  # what each page holds afterwards
    assert (pages[new] == ids).all() and sorted(new) == list(range(len(ids)))
    assert (src != dst).all() and len(set(dst)) == len(dst)
    order, todo = [], sorted(np.nonzero(t.node_parent < 0)[0], reverse=True)
    while todo:
        u = todo.pop()
        order.append(u)
        todo += sorted(np.nonzero(t.node_parent == u)[0], reverse=True)
    assert [int(x) for u in order for x in new[ptr[u]:ptr[u + 1]]] == list(range(len(ids)))
    # the plan has one piece to a node and chunk then, as that of a contiguous cache
    before, after = (binding.deft_plan_paged(ptr, x, 8, n_pool, t.node_tok_len, t.node_parent, t.query_node, 64).view() for x in (ids, new))
    whole = binding.deft_plan(np.cumsum(np.r_[0, t.node_tok_len[:-1]]), t.node_tok_len, t.node_parent, t.query_node, t.ntok, 64).view()
    assert after["n_segs"] == whole["n_segs"] <= before["n_segs"]


@pytest.mark.parametrize("ptr,ids,pool,parent", [
    ([0, 1], [4], 4, [-1]), ([0, 1], [-1], 4, [-1]), ([0, 2], [1, 1], 4, [-1]), ([0, 1, 2], [0, 0], 4, [-1, 0]), ([0, 2, 1], [0], 4, [-1, 0]),
    ([1, 1], [0], 4, [-1]), ([0, 1], [0], 4, [0]), ([0, 1, 2], [0, 1], 4, [1, 0]), ([0, 1], [0], 4, [1]), ([0, 1], [0], 4, [-2]), ([0, 2], [0, 1], 1, [-1]), ([0, 1], [1 << 32], 4, [-1])])
def test_tables_that_are_refused(ptr, ids, pool, parent):
    with pytest.raises(binding.DeftError) as e:
        binding.deft_compact_pages(ptr, ids, pool, parent)
    assert e.value.status == EINVAL


def test_sizes_that_32_bits_do_not_hold():
    for call in (lambda: binding.deft_kv_rows([0], (1 << 32) + 4), lambda: binding.deft_kv_rows([0], 4, (1 << 32) + 32), lambda: binding.deft_kv_copies([0], [1], (1 << 32) + 4),
                 lambda: binding.deft_compact_pages([0, 1], [0], (1 << 32) + 4, [-1])):
        with pytest.raises(binding.DeftError) as e:
            call()
        assert e.value.status == EINVAL


@pytest.mark.parametrize("seed", range(3))
def test_the_new_table_may_be_the_old_one(seed):
    t = wl.random_tree(seed, n_nodes=9, max_len=60, nq=5)
    ptr, ids, n_pool, _ = wl.to_paged(t, 8, seed)
    ptr, ids, par = (np.ascontiguousarray(x, dtype=np.int32) for x in (ptr, ids, t.node_parent))
    want = binding.deft_compact_pages(ptr, ids, n_pool, par)
    table, src, dst, n = ids.copy(), np.zeros_like(ids), np.zeros_like(ids), ctypes.c_int32()
    at = lambda x: x.ctypes.data  # noqa: E731
    assert binding.load_library().deft_compact_pages(at(ptr), at(table), n_pool, at(par), par.size, at(table), at(src), at(dst), ctypes.byref(n)) == 0
    for got, x in zip((table, src[:n.value], dst[:n.value]), want):
        assert np.array_equal(got, x)
    assert n.value > 0

"""Whole calls on an 8-bit cache that are made in one launch: which are, and what becomes of rows that are late."""

import ctypes

import numpy as np
import pytest
import torch

from paper_2404_00242_amd import binding, workloads as wl

pytestmark = pytest.mark.gpu


def prepared(t, chunk, flags=0, block=16):
    q, k, v = (x.cuda() for x in wl.make_qkv(t))
    cache = binding.alloc_kv_cache_q8(t.ntok, t.Hkv, t.d, block, torch.device("cuda:0"))
    binding.deft_kv_store_q8(binding.deft_kv_rows(np.arange(t.ntok), t.ntok, block), k, v, cache)
    return binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, t.query_node, t.ntok, chunk, flags), q, cache, v


def star(root, leaves, length, Hq, Hkv, d, nq=1):
    return wl._finish("star", [root] + [length] * leaves, [-1] + [0] * leaves, list(range(1, leaves + 1)) if leaves else [0] * nq, Hq, Hkv, d, 7)


def two_launches(plan, t, q, cache):
    ws = torch.empty(plan.view()["n_slots"] * t.Hq * (t.d + 2) * 4 + 32, dtype=torch.uint8, device="cuda")
    return binding.deft_tree_attn_decode_q8(plan, q, cache, out_dtype=torch.float32, workspace=ws)


def close(a, b, v):
    # a mean of V, whose bytes times scales are at most 2 |V|; two fp32 sums of n <= 512 terms differ by 2 n 2^-24 of the largest
    assert (a - b).abs().max().item() <= 2 * 512 * 2.0**-24 * 2 * v.abs().max().item()


def marks(plan, t, ws):
    rows = plan.view()["n_slots"] * t.Hq
    return ws[4 * (rows * t.d + (2 * rows + 3) // 4 * 4):][: 16 * rows].view(torch.int64).view(-1, 2)[:, 1]


@pytest.mark.parametrize("t,chunk,one", [
    (star(256, 4, 32, 4, 4, 64), 0, True),
    (star(16383, 0, 0, 32, 8, 128), 512, True),        # 32 partial results, one token under 32 MiB of K and V
    (star(16400, 0, 0, 32, 8, 128), 544, False),       # 31, 32.03 MiB
    (star(8192, 0, 0, 32, 8, 128), 128, True),         # 64, 16 MiB
    (star(8200, 0, 0, 32, 8, 128), 160, False),        # 52, 16.02 MiB
    (star(16384, 0, 0, 32, 8, 64), 128, True),         # 128 at d = 64, 16 MiB
    (star(16400, 0, 0, 32, 8, 64), 160, False),        # 103
    (star(2080, 0, 0, 8, 1, 128), 32, False),          # 65
    (star(4096, 0, 0, 32, 8, 128, nq=2), 256, True),   # 64 rows of output, 16 partial results, 8 MiB
    (star(4100, 0, 0, 32, 8, 128, nq=2), 288, False),  # 15, 8.01 MiB
    (star(8192, 0, 0, 32, 8, 64, nq=2), 256, True),    # 32 at d = 64, 8 MiB
    (star(8200, 0, 0, 32, 8, 64, nq=2), 288, False),   # 29
    (star(1000, 9, 50, 4, 4, 128), 64, False),         # 36 rows, 17 partial results
    (star(200, 17, 20, 4, 4, 128), 64, False),         # 68 rows
])
def test_which_calls_take_one_launch(t, chunk, one):
    # one launch writes its ticket into the marks, two leave them as they were
    plan, q, cache, v = prepared(t, chunk)
    ws = torch.full((plan.workspace_bytes(t.Hq, t.Hkv, t.d),), 0xFF, dtype=torch.uint8, device="cuda")
    got = binding.deft_tree_attn_decode_q8(plan, q, cache, out_dtype=torch.float32, workspace=ws)
    assert bool((marks(plan, t, ws) != -1).any()) == one
    close(got, two_launches(plan, t, q, cache), v)


def call_with_polls(plan, t, q, cache, out, ws, polls):
    """the call with another limit to the wait inside the kernel (deft_internal.h)"""
    img, p = plan.image(t.Hq, t.Hkv, "cuda"), ctypes.c_void_p
    flags = binding.DEFT_OUT_F32 if out.dtype == torch.float32 else binding.DEFT_OUT_BF16
    assert binding.load_library().deft_decode_polls_q8(
        plan.handle, p(img.data_ptr()), p(q.data_ptr()), binding._cache_args(cache, "")[0], p(out.data_ptr()), t.Hq, ctypes.c_float(0.0), flags,
        p(ws.data_ptr()), ctypes.c_size_t(ws.numel()), p(torch.cuda.current_stream().cuda_stream), polls) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t,chunk", [
    (star(40, 0, 0, 4, 4, 128), 32),
    (star(29 * 32, 0, 0, 2, 2, 64), 32),
    (star(700, 3, 20, 7, 1, 128), 32),     # tasks of one tile, rows that do not fill it
    (star(2048, 0, 0, 4, 1, 128), 32),     # two batches
    (star(2000, 7, 40, 8, 2, 128), 256),   # 56 rows, tasks of two tiles
    (star(900, 1, 100, 64, 8, 128), 128),  # 64 rows
    (star(4000, 0, 0, 32, 4, 128), 1024),  # streaming tasks
    (star(6000, 0, 0, 28, 2, 64), 512),
])
def test_rows_that_are_late_are_merged_by_stage_1(t, chunk, dtype):
    plan, q, cache, _ = prepared(t, chunk)
    ws = torch.zeros(plan.workspace_bytes(t.Hq, t.Hkv, t.d), dtype=torch.uint8, device="cuda")
    want = binding.deft_tree_attn_decode_q8(plan, q, cache, out_dtype=dtype, workspace=ws)
    assert bool((marks(plan, t, ws) != 0).any())  # made in one launch
    for polls in (1, 1, 2, 3, 4, 6, 9, 14):  # from a wait that is given up at once to one that may just do
        out = torch.full_like(want, float("nan"))
        ws.zero_()
        call_with_polls(plan, t, q, cache, out, ws, polls)
        assert torch.equal(out, want), polls

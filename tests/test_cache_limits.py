"""Lists of rows that one launch does not hold: what is launched, against a stand-in for the HIP runtime (CPU), and what is stored
and read back (GPU)."""

import numpy as np
import pytest
import torch

from paper_2404_00242_amd import binding
from tests.test_upload_errors import fake, needs_gxx, run  # noqa: F401 (fake is a fixture)

THREADS = 1 << 28  # of a launch, kMaxThreads in deft_cache.hip

LISTS = """
class Fake(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in names] + [("grid", ctypes.c_int32 * 16), ("kernel", ctypes.c_void_p * 16)]
fake = Fake.in_dll(fake_lib, "fake")
def launched(call):
    fake.launches = 0
    assert call() == 0
    return list(fake.grid[:fake.launches])
def cache(n_rows, Hkv, d, block):
    return binding._pack_cache(1 << 20, 1 << 40, 1 << 21, 1 << 22, n_rows, Hkv, d, block)
def store(rows, n_rows, Hkv, d, block):
    lst = binding.deft_kv_rows(rows, n_rows, block)
    return launched(lambda: lib.deft_kv_store_q8(lst.handle, 4096, 1 << 50, 1 << 51, Hkv * d, Hkv * d, cache(n_rows, Hkv, d, block), 1 << 12))
def load(rows, n_rows, Hkv, d, block, k=1 << 50, v=1 << 51):
    lst = binding.deft_kv_rows(rows, n_rows, block)
    return launched(lambda: lib.deft_kv_load_q8(lst.handle, 4096, cache(n_rows, Hkv, d, block), k, v, 1 << 12))
"""


@needs_gxx
@pytest.mark.parametrize("Hkv,d,block", [(65536, 64, 1), (65536, 128, 1), (32768, 64, 2), (65536, 128, 4), (65536, 64, 64), (65521, 128, 16)])
def test_stores_of_any_length(fake, Hkv, d, block):  # noqa: F811
    lanes = min(d // 8 * block, 64)  # of a unit, one (block, KV head)
    most = THREADS // lanes // Hkv   # blocks of a launch
    run(fake, LISTS + f"""
grid = lambda blocks: -(-blocks * {Hkv * lanes} // 256)
for blocks, want in (({most}, [{most}]), ({most + 1}, [{most}, 1]), ({2 * most + 3}, [{most}, {most}, 3]), (1, [1])):
    rows = np.arange(blocks) * {block}
    assert store(rows, blocks * {block}, {Hkv}, {d}, {block}) == [grid(n) for n in want]
""")


@needs_gxx
@pytest.mark.parametrize("Hkv,d", [(65536, 64), (65536, 128), (40000, 128)])
def test_loads_of_any_length(fake, Hkv, d):  # noqa: F811
    per_row = Hkv * d // 16
    run(fake, LISTS + f"""
for both, k, v in ((2, 1 << 50, 1 << 51), (1, 1 << 50, None), (1, None, 1 << 51)):
    most = {THREADS} // both // {per_row}
    for n, want in ((most, [most]), (most + 1, [most, 1]), (2 * most + 5, [most, most, 5])):
        assert load(np.arange(n), n, {Hkv}, {d}, 1, k, v) == [-(-x * both * {per_row} // 256) for x in want]
""")


@needs_gxx
def test_a_million_rows_of_thirty_two_heads(fake):  # noqa: F811
    run(fake, LISTS + """
n = (1 << 20) + 1
# 32 * 16 threads a row on either way: (2^20 + 1) 2^9 of them are two launches of 2^28 and one more
assert len(store(np.arange(n), n, 32, 128, 1)) == 3 and len(load(np.arange(n), n, 32, 128, 1)) == 3
n = 9_000_000
assert len(load(np.arange(n), n, 32, 128, 1, v=None)) == 9
""")


@pytest.mark.gpu
@pytest.mark.parametrize("Hkv,d,block,extra", [(65536, 64, 1, 5), (32768, 128, 2, 3)])
def test_lists_of_two_launches(Hkv, d, block, extra):
    # beside the same tokens in lists of one launch each: the same bytes in the cache, the same values out of it
    dev = torch.device("cuda:0")
    most = THREADS // (d // 8 * block) // Hkv * block
    n = most + extra * block
    g = torch.Generator(device=dev).manual_seed(3)
    k, v = (torch.randn((n, Hkv, d), generator=g, device=dev, dtype=torch.bfloat16) for _ in range(2))
    whole, parts = (binding.alloc_kv_cache_q8(n, Hkv, d, block, dev) for _ in range(2))
    for c in (whole, parts):
        for x in c[:2]:
            x.view(torch.uint8).zero_()
    lst = binding.deft_kv_rows(np.arange(n), n, block)
    binding.deft_kv_store_q8(lst, k, v, whole)
    half = n // 2 // block * block
    for a, b in ((0, half), (half, n)):
        binding.deft_kv_store_q8(binding.deft_kv_rows(np.arange(a, b), n, block), k[a:b], v[a:b], parts)
    del k, v
    for x, y in zip(whole[:4], parts[:4]):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    del parts
    rows = np.random.default_rng(1).permutation(n)
    at = torch.from_numpy(rows).to(dev)
    for got, x, s in zip(binding.deft_kv_load_q8(binding.deft_kv_rows(rows, n, block), whole), (whole.k, whole.v), (whole.k_scale, whole.v_scale)):
        for a in range(0, n, 64):  # (values are bf16 numbers: 0 is what they may be off)
            r = at[a:a + 64]
            scale = torch.exp2(s.view(torch.uint8)[r // block].float() - 127)
            assert torch.equal(got[a:a + 64].float(), x.view(torch.uint8)[r].view(torch.float8_e4m3fn).float() * scale[..., None])
    torch.cuda.empty_cache()

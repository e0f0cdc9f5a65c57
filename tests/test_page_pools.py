"""Which pools a list of copies goes with."""

import numpy as np
import pytest
import torch

from paper_2404_00242_amd import binding


def cpu_cache(n_rows, block, Hkv=2, d=64):
    return binding.alloc_kv_cache_q8(n_rows, Hkv, d, block, device="cpu")


def refused(copies, pools, match, **kw):
    with pytest.raises(binding.DeftError, match=match) as e:
        binding.deft_kv_copy_pages(copies, pools, **kw)
    assert e.value.status == -1


# what is accepted here fails for being on the CPU, behind all checks of sizes
ACCEPTED, SIZES = "device", "whole number of blocks|first dimension|whole number of bytes"


@pytest.mark.parametrize("page,block,ok", [(16, 32, False), (32, 32, True), (64, 32, True), (48, 32, False), (16, 16, True), (1, 1, True), (1, 2, False)])
def test_pages_of_an_8_bit_cache_are_whole_blocks(page, block, ok):
    copies, c = binding.deft_kv_copies([0], [1], 6), cpu_cache(6 * page, block)
    for kw in ({}, {"page_size": page}):
        refused(copies, [c.k_scale], ACCEPTED if ok else SIZES, **kw)
        refused(copies, [c.v_scale, c.k], ACCEPTED if ok else SIZES, **kw)
        refused(copies, [c.k, c.v], ACCEPTED, **kw)
        refused(copies, [c], "one device", **kw)
        for bad in (page + 1, 2 * page, 0):
            refused(copies, [c.k], SIZES, page_size=bad)
    refused(copies, [torch.zeros((6, 3), dtype=torch.uint8)], ACCEPTED)
    refused(copies, [torch.zeros((7, 3), dtype=torch.uint8)], SIZES)


def test_a_pool_of_other_pages_than_the_lists():
    # twice the pages: half a page would be copied; with the rows of a page named it is refused
    copies = binding.deft_kv_copies([0], [1], 10)
    k = torch.zeros((20 * 16, 2, 64), dtype=torch.bfloat16)
    refused(copies, [k], SIZES, page_size=16)
    refused(copies, [k[:160], k], SIZES, page_size=16)
    refused(copies, [k[:160]], ACCEPTED, page_size=16)
    refused(copies, [torch.zeros(())], SIZES, page_size=16)
    for rows, ok in ((10, True), (5, False), (20, True), (160, True), (30, False), (15, False)):  # blocks of 16, 32, 8, 1, 5.3, 10.7 rows
        scales = torch.zeros((rows, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu)
        refused(copies, [scales], ACCEPTED if ok else SIZES, page_size=16)
    refused(binding.deft_kv_copies([], [], 0), [k], SIZES)


@pytest.mark.gpu
def test_whole_caches_beside_pools():
    dev, rng, pages, page = torch.device("cuda:0"), np.random.default_rng(2), 30, 32
    src, dst = rng.integers(0, pages, 20), rng.permutation(pages)[:20]
    copies = binding.deft_kv_copies(src, dst, pages)
    caches = [binding.alloc_kv_cache_q8(pages * page, 2, d, block, dev) for d, block in ((64, 32), (128, 8))]
    plain = torch.randn((pages * page, 2, 64), device=dev).to(torch.bfloat16)
    flat = [x for c in caches for x in c[:4]] + [plain]
    for x in flat[:-1]:
        x.view(torch.uint8).copy_(torch.randint(0, 127, x.shape, dtype=torch.uint8, device=dev))
    want = []
    for x in flat:
        y = x.view(torch.uint8).reshape(pages, -1).clone()
        y[torch.from_numpy(dst).to(dev)] = y[torch.from_numpy(src).to(dev)]
        want.append(y)
    binding.deft_kv_copy_pages(copies, [caches[0], plain, caches[1]], page_size=page)
    assert all(torch.equal(x.view(torch.uint8).reshape(pages, -1), y) for x, y in zip(flat, want))
    for bad, kw in ((caches, {"page_size": 16}), ([binding.alloc_kv_cache_q8(pages * 16, 2, 64, 32, dev)], {}), ([caches[0]._replace(k=plain)], {})):
        with pytest.raises(binding.DeftError):
            binding.deft_kv_copy_pages(copies, bad, **kw)
    assert all(torch.equal(x.view(torch.uint8).reshape(pages, -1), y) for x, y in zip(flat, want))

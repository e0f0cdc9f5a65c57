"""Norms of heads, rotary positions and rows stored into an 8-bit cache in one call: byte for byte what the two calls that it takes the
place of leave, and near the definition in 64 bits (oracle/heads.py)."""

import numpy as np
import pytest
import torch

from oracle import heads as heads_model
from paper_2404_00242_amd import binding, workloads as wl
from tests.test_cache_q8 import new_cache, tokens
from tests.test_heads import EINVAL, _part, dev, on_gpu, positions, values
from tests.test_upload_errors import fake, needs_gxx, run  # noqa: F401 (fake is a fixture)


# ---- refusals (CPU: addresses that nothing reads) ----

def test_calls_that_are_refused():
    lib, rope, pos = binding.load_library(), binding.deft_rope(64).packed, 1 << 12
    rows, larger, none = binding.deft_kv_rows([3, 1], 8, 4), binding.deft_kv_rows([3, 1], 9, 4), binding.deft_kv_rows([], 8, 4)
    copies = binding.deft_kv_copies([0], [1], 8)
    at = [1 << 24, 1 << 25, 1 << 26, 1 << 27]

    def cache(k=at[0], v=at[1], ks=at[2], vs=at[3], n=8, heads=4, d=64, block=4):
        return binding._pack_cache(k, v, ks, vs, n, heads, d, block)

    k, v = _part(out=0), _part(x=1 << 21, out=0)

    def store(lst=rows.handle, image=1 << 16, q=None, k=k, v=v, cache=cache(), eps=0.0, offset=0.0, positions=pos, rope=rope):
        return lib.deft_qkv_store_q8(lst, image, q, k, v, cache, eps, offset, positions, rope, None)

    bad_caches = [dict(k=0), dict(ks=0), dict(k=at[0] + 4), dict(vs=at[3] + 2), dict(n=7), dict(heads=3), dict(d=96), dict(block=8), dict(block=3),
                  dict(v=at[0]), dict(vs=at[2]),
                  # of the cache and the inputs, and the queries' result, one is the other's
                  dict(k=1 << 20), dict(v=(1 << 20) + 512), dict(ks=1 << 20), dict(vs=(1 << 21) + 64), dict(k=1 << 22), dict(v=(1 << 23) - 2032), dict(ks=(1 << 23) + 4),
                  dict(k=1 << 12), dict(vs=(1 << 12) + 4), dict(ks=1 << 13), dict(v=(1 << 13) + 64 - 16)]
    q = _part(x=1 << 22, out=1 << 23, weight=1 << 13)
    for bad in bad_caches:
        assert store(q=q, cache=cache(**bad)) == EINVAL, bad
    for bad in (dict(lst=None), dict(lst=copies.handle), dict(lst=larger.handle), dict(image=None),
                dict(image=24), dict(k=None), dict(v=None), dict(cache=None), dict(k=_part(out=0, heads=3)), dict(v=_part(x=1 << 21, heads=5)),
                dict(v=_part(x=1 << 21, weight=1 << 12)), dict(k=_part(x=0)), dict(k=_part(x=(1 << 20) + 8)), dict(v=_part(x=1 << 21, token=260)),
                dict(k=_part(head=-64)), dict(k=_part(weight=(1 << 14) + 4)), dict(k=_part(weight=1 << 14), eps=-1.0), dict(k=_part(weight=1 << 14), eps=float("nan")),
                dict(k=_part(weight=1 << 14), offset=float("inf")), dict(k=_part(weight=1 << 14, wide=1), q=q), dict(positions=None), dict(positions=pos + 2),
                dict(rope=binding.deft_rope(128).packed), dict(q=_part(x=1 << 22, out=0)), dict(q=_part(x=1 << 22, out=1 << 20)),
                dict(q=_part(x=1 << 22, out=(1 << 21) - 16)), dict(q=_part(x=1 << 22, out=at[0])), dict(q=_part(x=1 << 22, out=at[1] - 16)),
                dict(q=_part(x=at[1] + 16, out=1 << 23)), dict(q=_part(x=1 << 22, heads=-1)), dict(q=_part(x=1 << 22, out=1 << 22, head=0))):
        assert store(**bad) == EINVAL, bad
    assert store(lst=none.handle, rope=None, positions=None) == 0 and store(lst=none.handle, k=_part(x=0), v=_part(x=0)) == 0
    assert store(lst=none.handle, v=_part(heads=3)) == store(lst=none.handle, k=None) == EINVAL


def test_cpu_tensors_are_refused():
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    cache = binding.alloc_kv_cache_q8(8, 4, 64, 1, "cpu")
    with pytest.raises(binding.DeftError):
        binding.deft_qkv_store_q8(binding.deft_kv_rows([0, 1], 8, 1), x, x, x, cache)


WAVES = 1 << 22  # of queries that share a launch, kMaxWaves in deft_heads.hip


@needs_gxx
@pytest.mark.parametrize("heads,d,block,n", [(65536, 128, 64, 640), (65536, 128, 64, 4200), (65536, 64, 1, 4097), (8, 128, 32, 500), (3, 64, 2, 5), (1, 128, 8, 1), (5, 128, 16, 100), (65533, 64, 32, 1500)])
def test_calls_of_any_length(fake, heads, d, block, n):  # noqa: F811
    # a block's rows of one head have lanes of sixteen elements: waves of them, and then a workgroup has heads of one block, or a part
    # of a wave; a workgroup has four waves, or eight where one head's are that many; queries share the first launch, or have launches
    # of their own in front if they are too many for it
    run(fake, f"""
class Fake(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in names] + [("grid", ctypes.c_int32 * 16), ("kernel", ctypes.c_void_p * 16)]
fake = Fake.in_dll(fake_lib, "fake")
heads, d, block, n = {heads}, {d}, {block}, {n}
def part(at, heads, out=0):
    return binding._pack_heads(at, heads * d, d, out, 0, 0, 0, heads)
cache = binding._pack_cache(1 << 52, 1 << 53, 1 << 54, 1 << 55, n, heads, d, block)
lst = binding.deft_kv_rows(np.arange(n), n, block)
def launched(q):
    fake.launches = 0
    assert lib.deft_qkv_store_q8(lst.handle, 4096, q, part(1 << 50, heads), part(1 << 51, heads), cache, 0.0, 0.0, 4096, binding.deft_rope(64).packed, 1 << 12) == 0
    return list(fake.grid[:fake.launches])
lanes = d // 16 * block
whole = lanes >= 64
threads = max(lanes, 256)
parts = -(-heads // (threads // lanes)) if whole else 0
groups, most = -(-n // block), (1 << 28) // threads // parts if whole else (1 << 28) // lanes // heads
want = []
while groups:
    now = min(groups, most)
    want.append(now * parts if whole else -(-now * heads // (256 // lanes)))
    groups -= now
assert launched(None) == want, (launched(None), want)
for Hq in (8, 65536):
    chunks = -(-Hq // (64 // (d // 16)))
    waves, most = n * chunks, {WAVES} // chunks
    if waves <= {WAVES}:
        expected = [want[0] + -(-waves // (threads // 64))] + want[1:]
    else:
        expected = [-(-min(most, n - i) * chunks // 4) for i in range(0, n, most)] + want
    if len(expected) <= 16:
        assert launched(part(1 << 56, Hq, 1 << 57)) == expected, Hq
""")


# ---- on the GPU ----

def same(a, b):
    for x, y in zip(a[:4], b[:4]):
        x, y = x.view(torch.uint8), y.view(torch.uint8)
        assert torch.equal(x, y), torch.nonzero(x != y)[:5]


def twice(Hkv, d, block, rows, seed):
    """A cache with earlier contents, and another of the same bytes."""
    return [new_cache(rows, Hkv, d, block, seed)[0] for _ in range(2)]


def fresh(n, Hq, Hkv, d, seed, special=True):
    """q, k and v as slices of one tensor, with infinities, NaN, zeros and extremes among the keys and values."""
    x = torch.empty((n, Hq + 2 * Hkv, d), dtype=torch.bfloat16)
    x[:, :Hq] = values(n, Hq, d, seed) if Hq else x[:, :0]
    x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:] = tokens(n, Hkv, d, seed, special=special)
    x = x.to(dev())
    return x[:, :Hq] if Hq else None, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def by_two_calls(lst, q, k, v, cache, p, rope, wq, wk, eps=1e-6, offset=0.0):
    none = k[:, :0]
    out, keys = binding.deft_qk_norm_rotate(none if q is None else q, k, wq if q is not None else None, wk, p, rope, eps=eps, weight_offset=offset)
    binding.deft_kv_store_q8(lst, keys, v.contiguous(), cache)
    return None if q is None else out


@pytest.mark.gpu
@pytest.mark.parametrize("block", [1, 2, 4, 8, 16, 32, 64])
@pytest.mark.parametrize("Hq,Hkv,d", [(3, 1, 64), (0, 3, 64), (2, 2, 128), (40, 5, 128), (32, 8, 128)])
@pytest.mark.parametrize("layout,rot,norm", [("half", 1, "bf16"), ("interleaved", 1, None), ("half", 2, "f32"), ("interleaved", 4, "heads"), (None, 0, "bf16"), (None, 0, None)])
def test_a_store_is_the_two_calls_byte_for_byte(Hq, Hkv, d, block, layout, rot, norm):
    rows = 5 * 64 + 7  # the last block is short
    a, b = twice(Hkv, d, block, rows, 3)
    rope = binding.deft_rope(d // rot, layout=layout, factor=1.25) if layout else None
    g = torch.Generator().manual_seed(block)
    kind = torch.float32 if norm == "f32" else torch.bfloat16
    wq, wk = (None, None) if norm is None else (torch.randn((h, d) if norm == "heads" else (d,), generator=g).to(kind).to(dev()) for h in (max(Hq, 1), Hkv))
    rng = np.random.default_rng([Hkv, d, block])
    filled = [[int(x), 0] for x in rng.permutation(rows // 64) * 64] + [[320, 0]]
    first = np.concatenate([np.arange(x, x + 37) for x, _ in filled[:3]])
    for f in filled[:3]:
        f[1] = 37
    for step in range(6):  # a prompt, then tokens behind what is there, in any order, loud ones among them
        at = first
        if step:
            at = []
            for f, room in zip(filled, [64] * 5 + [7]):
                n = int(min(room - f[1], rng.integers(0, 5)))
                at += [f[0] + f[1] + i for i in range(n)]
                f[1] += n
            at = rng.permutation(np.array(at, dtype=np.int64))
        n = len(at)
        lst = binding.deft_kv_rows(at, rows, block)
        q, k, v = fresh(n, Hq, Hkv, d, 10 + step)
        p = on_gpu(positions(n, step))
        got = binding.deft_qkv_store_q8(lst, q, k, v, a, p, rope, q_weight=wq if Hq else None, k_weight=wk, weight_offset=float(step % 2))
        want = by_two_calls(lst, q, k, v, b, p, rope, wq, wk, offset=float(step % 2))
        same(a, b)
        assert (got is None) == (not Hq) and (not Hq or torch.equal(got.view(torch.int16), want.view(torch.int16)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,Hq,Hkv,d,block", [(1, 32, 8, 128, 32), (1024, 32, 8, 128, 32), (1025, 32, 8, 128, 32), (2100, 7, 1, 64, 64), (3000, 40, 3, 128, 16)])
def test_few_and_many_queries(n, Hq, Hkv, d, block):
    rows = -(-n // 64) * 64 + 64
    a, b = twice(Hkv, d, block, rows, 1)
    lst = binding.deft_kv_rows(np.random.default_rng(n).permutation(n), rows, block)
    rope, w = binding.deft_rope(d), torch.rand((2, d), device=dev())
    q, k, v = fresh(n, Hq, Hkv, d, 5)
    p = on_gpu(positions(n))
    mine = q._base.clone()
    got = binding.deft_qkv_store_q8(lst, q, k, v, a, p, rope, q_weight=w[0], k_weight=w[1])
    want = by_two_calls(lst, q, k, v, b, p, rope, w[0], w[1])
    same(a, b)
    assert torch.equal(got, want)
    # the queries where they are
    x, y, z = mine[:, :Hq], mine[:, Hq:Hq + Hkv], mine[:, Hq + Hkv:]
    back = mine.clone()
    assert binding.deft_qkv_store_q8(lst, x, y, z, a, p, rope, q_weight=w[0], k_weight=w[1], q_out=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, want) and torch.equal(mine[:, Hq:].view(torch.int16), back[:, Hq:].view(torch.int16))
    by_two_calls(lst, q, k, v, b, p, rope, w[0], w[1])
    same(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_what_is_stored_is_near_the_definition(layout):
    n, Hkv, d, block = 200, 3, 128, 16
    cache = binding.alloc_kv_cache_q8(256, Hkv, d, block, dev())
    x, p, w = values(n, 2 * Hkv, d, 9), positions(n), torch.rand(d) + 0.5
    rope, (f, factor) = binding.deft_rope(96, layout=layout), heads_model.frequencies(96)
    lst = binding.deft_kv_rows(np.arange(n), 256, block)
    gpu = x.to(dev())
    # heads one after the other, the tokens of each: neither tokens nor heads are contiguous
    k, v = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (gpu[:, :Hkv], gpu[:, Hkv:]))
    binding.deft_qkv_store_q8(lst, None, k, v, cache, on_gpu(p), rope, k_weight=w.to(dev()))
    K, V = (t.double().cpu().numpy() for t in binding.deft_kv_load_q8(lst, cache))
    want, mag = heads_model.heads(x[:, :Hkv].double().numpy(), p, f, factor, layout == "interleaved", w.double().numpy())
    scale = [np.exp2(s.view(torch.uint8).cpu().numpy().astype(np.float64) - 127)[np.arange(n) // block][..., None] for s in (cache.k_scale, cache.v_scale)]
    # e4m3's half step, 2^-4 of a value or, of small ones, 2^-10 of the scale; a key's half step of bf16 and its arithmetic (see close in
    # test_heads.py) in front of it, which it is then rounded with: a factor 1 + 2^-4
    assert (np.abs(K - want) <= (1 + 2.0 ** -4) * (2.0 ** -8 * (1 + 2.0 ** -10) * np.abs(want) + 2.0 ** -19 * mag) + np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale[0])).all()
    values_ = x[:, Hkv:].double().numpy()
    assert (np.abs(V - values_) <= np.maximum(2.0 ** -4 * np.abs(values_), 2.0 ** -10 * scale[1])).all()


@pytest.mark.gpu
def test_rows_behind_four_billion_elements():
    # beside the same tokens in the first rows of a small cache
    n, Hkv, d, block = 70, 64, 128, 32
    rows = (1 << 32) // (Hkv * d) + 2 * n
    first = rows // block * block - 3 * block
    big, small = (binding.alloc_kv_cache_q8(r, Hkv, d, block, dev()) for r in (rows, 96))
    at = np.random.default_rng(1).permutation(n)
    q, k, v = fresh(n, 4, Hkv, d, 3)
    p, rope, w = on_gpu(positions(n)), binding.deft_rope(d), torch.rand(d, device=dev())
    got = binding.deft_qkv_store_q8(binding.deft_kv_rows(at + first, rows, block), q, k, v, big, p, rope, k_weight=w)
    want = by_two_calls(binding.deft_kv_rows(at, 96, block), q, k, v, small, p, rope, None, w)
    assert torch.equal(got, want)
    for a, b in zip(big[:2], small[:2]):
        assert torch.equal(a[first:first + n].view(torch.uint8), b[:n].view(torch.uint8))
    for a, b in zip(big[2:4], small[2:4]):
        assert torch.equal(a.view(torch.uint8)[first // block:first // block + 3], b.view(torch.uint8))
    del big
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_nothing_to_do():
    cache, _ = new_cache(64, 2, 64, 8)
    before = [t.view(torch.uint8).clone() for t in cache[:4]]
    x = torch.zeros((0, 6, 64), dtype=torch.bfloat16, device=dev())
    rope, p = binding.deft_rope(64), torch.zeros(0, dtype=torch.int32, device=dev())
    q = binding.deft_qkv_store_q8(binding.deft_kv_rows([], 64, 8), x[:, :2], x[:, 2:4], x[:, 4:], cache, p, rope)
    assert q.shape == (0, 2, 64) and all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, cache[:4]))
    y = torch.ones((1, 4, 64), dtype=torch.bfloat16, device=dev())
    q = binding.deft_qkv_store_q8(binding.deft_kv_rows([0], 64, 8), y[:, :0], y[:, :2], y[:, 2:], cache)
    assert q.shape == (1, 0, 64) and (binding.deft_kv_load_q8(binding.deft_kv_rows([0], 64, 8), cache)[0] == 1).all()


@pytest.mark.gpu
def test_gpu_refusals():
    n, d = 4, 64
    x = torch.zeros((n, 6, d), dtype=torch.bfloat16, device=dev())
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    p, rope, w = torch.zeros(n, dtype=torch.int32, device=dev()), binding.deft_rope(64), torch.ones(d, dtype=torch.bfloat16, device=dev())
    cache, _ = new_cache(8, 2, d, 1)
    other = binding.alloc_kv_cache_q8(8, 2, d, 2)
    rows, store = binding.deft_kv_rows([0, 1, 2, 3], 8, 1), binding.deft_qkv_store_q8
    pools = [torch.zeros((8, 2, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    inside = cache.k.view(torch.uint8).view(-1)[:8 * 2 * d].view(torch.bfloat16).view(4, 2, d)
    bad = [
        lambda: store(rows, q, k, v, other, p, rope), lambda: store(rows, q, k, v, cache._replace(v=cache.k), p, rope), lambda: store(rows, q, k, v, cache._replace(v=cache.v[:7]), p, rope),
        lambda: store(binding.deft_kv_rows([0, 1, 2, 3], 9, 1), q, k, v, cache, p, rope), lambda: store(binding.deft_kv_copies([0], [1], 8), q, k, v, cache, p, rope),
        lambda: store(rows, q, k[:, :1], v[:, :1], cache, p, rope), lambda: store(rows, q, k, v[:, :1], cache, p, rope), lambda: store(rows, q, k[:3], v[:3], cache, p, rope),
        lambda: store(rows, q[:3], k, v, cache, p, rope), lambda: store(rows, q, k.float(), v, cache, p, rope), lambda: store(rows, q, k.cpu(), v.cpu(), cache, p, rope),
        lambda: store(rows, q, k, v, cache, p[:3], rope), lambda: store(rows, q, k, v, cache, None, rope), lambda: store(rows, q, k, v, cache, p.long(), rope),
        lambda: store(rows, None, k, v, cache, p, rope, q_weight=w), lambda: store(rows, q, k, v, cache, p, rope, q_weight=w, k_weight=w.float()),
        lambda: store(rows, q, k, v, cache, p, rope, k_weight=w, eps=-1.0), lambda: store(rows, q, k, v, cache, p, binding.deft_rope(128)),
        lambda: store(rows, q, k, v, cache, p, rope, q_out=k), lambda: store(rows, q, k, v, cache, p, rope, q_out=inside), lambda: store(rows, q, inside, v, cache, p, rope),
        lambda: store(rows, inside, k, v, cache, p, rope),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.DeftError):
            call()
            pytest.fail(f"call {i}")
    with pytest.raises((binding.DeftError, ValueError, AttributeError)):
        store(rows, q, k, v, pools, p, rope)
    torch.cuda.synchronize()
    assert not x.any() and not any(t.any() for t in pools)
    again, _ = new_cache(8, 2, d, 1)
    same(cache, again)


@pytest.mark.gpu
def test_captured_and_replayed_and_on_other_streams():
    n, Hq, Hkv, d, block = 40, 8, 2, 128, 16
    a, b = twice(Hkv, d, block, 208, 2)
    rope, w = binding.deft_rope(64, layout="interleaved"), torch.rand(d, device=dev())
    x, p = torch.zeros((n, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device=dev()), on_gpu(positions(n))
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    rows = binding.deft_kv_rows(np.random.default_rng(0).permutation(208)[:n], 208, block)  # first used inside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.deft_qkv_store_q8(rows, q, k, v, a, p, rope, q_weight=w, k_weight=w)
    side = torch.cuda.Stream()
    for i in range(4):
        x[:, :Hq] = values(n, Hq, d, i).to(dev())
        x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:] = (t.to(dev()) for t in tokens(n, Hkv, d, i))
        p.copy_(on_gpu(positions(n, i)))
        w.uniform_()
        graph.replay()
        want = by_two_calls(rows, q, k, v, b, p, rope, w, w)
        assert torch.equal(out, want)
        same(a, b)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        got = binding.deft_qkv_store_q8(rows, q, k, v, a, p, rope, q_weight=w, k_weight=w, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        by_two_calls(rows, q, k, v, b, p, rope, w, w)
        assert torch.equal(got, want)
        same(a, b)


@pytest.mark.gpu
def test_layers_of_an_iteration():
    t = wl.random_tree(31, n_nodes=12, max_len=200, nq=14, Hq=8, Hkv=2, d=128, zero_len_prob=0.0)
    plan = binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, t.query_node, t.ntok, 64)
    rope, w = binding.deft_rope(t.d), torch.rand((2, t.d), device=dev())
    caches = [binding.alloc_kv_cache_q8(t.ntok, t.Hkv, t.d, 1, dev()) for _ in range(2)]
    every = binding.deft_kv_rows(np.arange(t.ntok), t.ntok, 1)
    _, k, v = fresh(t.ntok, 0, t.Hkv, t.d, 1, special=False)
    k, v = k.clamp(-8, 8), v.clamp(-8, 8)
    p = on_gpu(np.arange(t.ntok, dtype=np.int32))
    # the prompt, and then what a layer does: new tokens' keys and values stored, queries turned, attention over them
    binding.deft_qkv_store_q8(every, None, k, v, caches[0], p, rope, k_weight=w[1])
    by_two_calls(every, None, k, v, caches[1], p, rope, None, w[1])
    node = np.unique(t.query_node)
    at = t.node_tok_begin[node] + t.node_tok_len[node] - 1
    new = binding.deft_kv_rows(at, t.ntok, 1)
    q, k, v = fresh(len(at), t.Hq, t.Hkv, t.d, 2, special=False)
    k, v = k.clamp(-8, 8), v.clamp(-8, 8)
    p = on_gpu(at.astype(np.int32))
    got = binding.deft_qkv_store_q8(new, q, k, v, caches[0], p, rope, q_weight=w[0], k_weight=w[1])
    want = by_two_calls(new, q, k, v, caches[1], p, rope, w[0], w[1])
    index = torch.from_numpy(np.searchsorted(node, t.query_node)).to(dev())
    o = [binding.deft_tree_attn_decode_q8(plan, x[index], c, out_dtype=torch.float32) for x, c in ((got, caches[0]), (want, caches[1]))]
    assert torch.equal(o[0], o[1]) and torch.isfinite(o[0]).all() and o[0].any()

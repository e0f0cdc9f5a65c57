"""Norms of heads, rotary positions and rows stored into a bf16 cache: against the definition in 64 bits (oracle/heads.py)."""

import ctypes
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import heads as model
from paper_2404_00242_amd import binding
from tests.test_upload_errors import fake, needs_gxx, run  # noqa: F401 (fake is a fixture)

EINVAL = -1
SCALINGS = [dict(), dict(scaling="linear", scale=4.0), dict(scaling="base", scale=8.0, base=500000.0),
            dict(scaling="dimension", scale=8.0, original=4096), dict(scaling="dimension", scale=0.5, original=100, low=2.0, high=16.0),
            dict(scaling="wavelength", scale=8.0, original=8192, base=500000.0), dict(scaling="wavelength", scale=3.0, original=50, low=0.5, high=3.0)]


# ---- frequencies (CPU) ----

@pytest.mark.parametrize("rot", [16, 32, 48, 128])
@pytest.mark.parametrize("how", SCALINGS, ids=lambda h: "-".join(map(str, h.values())) or "none")
def test_frequencies_are_the_formulas(rot, how):
    f, factor = binding.deft_rope_frequencies(rot, **how)
    want, want_factor = model.frequencies(rot, **how)
    # a few roundings of 64 bits in each of the powers, logarithms and quotients
    assert np.allclose(f, want, rtol=64 * 2.0 ** -53, atol=0) and math.isclose(factor, want_factor, rel_tol=2.0 ** -50)
    assert (np.diff(f) < 0).all()


def _pi():
    """pi to 60 digits by Machin's formula, as a fraction."""
    def arctan(inv):
        x, total, n = Fraction(1, inv), Fraction(0), 0
        term = x
        while abs(term) > Fraction(1, 10 ** 62):
            total += term / (2 * n + 1) * (-1) ** n
            term *= x * x
            n += 1
        return total
    return 4 * (4 * arctan(5) - arctan(239))


@pytest.mark.parametrize("rot", [1 << 62, 1 << 45, -(1 << 62), 1 << 30, 130])
def test_sizes_of_ropes_are_looked_at_before_memory_is_taken_for_them(rot):
    for call in (lambda: binding.deft_rope_frequencies(rot), lambda: binding.deft_rope(rot)):
        with pytest.raises(binding.DeftError):
            call()


def test_turns_are_the_frequencies_to_sixty_four_bits():
    rng = np.random.default_rng(1)
    f = np.concatenate([10000.0 ** (-np.arange(32) / 32), rng.uniform(-1e6, 1e6, 16), [0.0, -1e-9, 2 * math.pi, 1e6], rng.uniform(-7, 7, 12)])
    rope = binding.deft_rope(128, frequencies=f, layout="interleaved", factor=1.5)
    turns = np.frombuffer(rope.packed, dtype=np.uint64, count=64)
    two_pi = 2 * _pi()
    for x, t in zip(f, turns):
        want = Fraction(float(x)) / two_pi
        off = abs((want - Fraction(int(t), 1 << 64) + Fraction(1, 2)) % 1 - Fraction(1, 2))
        # half a step of 2^-64, and the quotient's rounding in 64 bits of mantissa
        assert off <= Fraction(1, 1 << 64) + abs(want) / (1 << 63)
    assert np.frombuffer(rope.packed, dtype=np.float32)[128] == 1.5 and list(np.frombuffer(rope.packed, dtype=np.int32)[129:131]) == [128, 1]


def test_ropes_that_are_refused():
    nan, inf = float("nan"), float("inf")
    for bad in (dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16), dict(rot=1 << 32), dict(rot=64, base=1.0), dict(rot=64, base=nan),
                dict(rot=64, base=inf), dict(rot=64, layout="quarter"), dict(rot=64, scaling="some"), dict(rot=64, scaling="linear", scale=0.0),
                dict(rot=64, scaling="base", scale=-1.0), dict(rot=64, scaling="linear", scale=nan), dict(rot=64, scaling="dimension", scale=2.0),
                dict(rot=64, scaling="wavelength", scale=2.0, original=inf), dict(rot=64, scaling="wavelength", scale=2.0, original=100, low=4.0, high=4.0),
                dict(rot=64, factor=nan), dict(rot=64, factor=1e300), dict(rot=64, frequencies=[1.0] * 31), dict(rot=32, frequencies=[1.0] * 15 + [nan]),
                dict(rot=32, frequencies=[1e7] * 16)):
        with pytest.raises(binding.DeftError):
            binding.deft_rope(**bad)
    lib, f = binding.load_library(), np.ones(64)
    at, one = f.ctypes.data, ctypes.byref(ctypes.c_double())
    assert lib.deft_rope(None, 64, 0, 1.0, b"x" * 528) == EINVAL and lib.deft_rope(at, 64, 0, 1.0, None) == EINVAL
    assert lib.deft_rope(at, 64, 2, 1.0, ctypes.create_string_buffer(528)) == EINVAL
    assert lib.deft_rope_frequencies(64, 1e4, 5, 1, 1, 1, 1, at, one) == EINVAL and lib.deft_rope_frequencies(64, 1e4, -1, 1, 1, 1, 1, at, one) == EINVAL
    assert lib.deft_rope_frequencies(64, 1e4, 0, 1, 1, 1, 1, None, one) == EINVAL


@pytest.mark.parametrize("bad", [
    dict(scaling="base", base=1e300, scale=1e30),  # the base leaves 64 bits: all pairs but the first would stand still
    dict(scaling="base", scale=1e-9), dict(scaling="base", base=2.0, scale=0.5),  # a base of one or less
    dict(scaling="linear", scale=5e-324), dict(scaling="linear", scale=1e-7),  # infinite, and more than a rope takes
    dict(scaling="dimension", scale=1e-300, original=4096), dict(scaling="wavelength", scale=1e-300, original=4096)], ids=str)
def test_scalings_that_lead_out_of_a_ropes_range_are_refused(bad):
    for rot in (16, 128):
        with pytest.raises(binding.DeftError):
            binding.deft_rope_frequencies(rot, **bad)
        with pytest.raises(binding.DeftError):
            binding.deft_rope(rot, **bad)


@pytest.mark.parametrize("good", [dict(scaling="linear", scale=1.1e-6), dict(scaling="base", scale=0.9, base=2.0), dict(scaling="base", base=1e200, scale=1e30),
                                  dict(base=1e300), dict(base=1 + 1e-9), dict(scaling="linear", scale=1e300)], ids=str)
def test_scalings_at_the_ends_of_a_ropes_range(good):
    for rot in (16, 128):
        f, factor = binding.deft_rope_frequencies(rot, **good)
        want, _ = model.frequencies(rot, **good)
        # the power's argument is off by a few roundings, times the base's logarithm: at most 1100 of them
        assert np.allclose(f, want, rtol=4096 * 2.0 ** -53, atol=0) and factor == 1 and np.isfinite(f).all()
        binding.deft_rope(rot, **good)


# ---- refusals (CPU: addresses that nothing reads) ----

def _part(x=1 << 20, token=256, head=64, out=1 << 24, weight=0, step=0, wide=0, heads=4):
    return binding._pack_heads(x, token, head, out, weight, step, wide, heads)


def test_calls_that_are_refused():
    lib = binding.load_library()
    rope = binding.deft_rope(64).packed
    pos = 1 << 12

    def rotate(part, n=8, d=64, positions=pos, rope=rope):
        return lib.deft_rotate(part, n, d, positions, rope, None)

    bad_parts = [dict(x=0), dict(out=0), dict(x=(1 << 20) + 8), dict(out=(1 << 24) + 2), dict(token=260), dict(head=68), dict(token=-256), dict(head=-64),
                 dict(heads=-1), dict(heads=65537), dict(token=1 << 41), dict(x=1 << 20, out=(1 << 20) + 512), dict(x=1 << 20, out=(1 << 20) - 512),
                 dict(out=1 << 20, token=192), dict(out=1 << 20, head=0), dict(out=1 << 20, head=32), dict(weight=1 << 12)]
    for bad in bad_parts:
        assert rotate(_part(**bad)) == EINVAL, bad
    assert rotate(None) == rotate(_part(), n=-1) == rotate(_part(), d=96) == rotate(_part(), positions=None) == rotate(_part(), rope=None) == EINVAL
    assert rotate(_part(), positions=pos + 2) == EINVAL
    assert rotate(_part(head=128, token=512), d=128, rope=binding.deft_rope(128).packed, n=-5) == EINVAL
    assert rotate(_part(), rope=binding.deft_rope(128).packed) == EINVAL  # more than a head of 64 has
    assert rotate(_part(token=1 << 40), n=1 << 30) == EINVAL  # the strides leave the address space
    assert rotate(_part(x=0, out=0), n=0) == 0 and rotate(_part(heads=0)) == 0

    def norm(q, k, n=8, d=64, eps=1e-6, offset=0.0, positions=pos, rope=rope):
        return lib.deft_qk_norm_rotate(q, k, n, d, eps, offset, positions, rope, None)

    q = _part(weight=1 << 12)
    for bad in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(offset=float("nan")), dict(positions=None), dict(d=32)):
        assert norm(q, None, **bad) == EINVAL, bad
    for bad in (dict(weight=(1 << 12) + 4), dict(weight=1 << 12, step=4), dict(weight=1 << 12, step=-64), dict(weight=1 << 12, step=8192),
                dict(weight=1 << 12, wide=1), dict(out=1 << 20), dict(out=(1 << 24) + 1024), dict(out=(1 << 20) + 1024)):
        assert norm(q, _part(x=1 << 21, **{"out": 1 << 25, **bad})) == EINVAL, bad
    # what is written meets a weight or the positions
    for out in ((1 << 12) - 1000, (1 << 12) - 4080):
        assert norm(_part(weight=1 << 16, out=out & ~15), None) == EINVAL
    assert norm(_part(weight=(1 << 24) + 2048), None) == norm(_part(), _part(x=1 << 21, out=1 << 25, weight=(1 << 24) - 16)) == EINVAL
    # one tensor twice, in place
    assert norm(_part(out=1 << 20), _part(out=1 << 20)) == EINVAL
    assert norm(None, None, n=0) == 0

    rows, none, copies = binding.deft_kv_rows([3, 1], 8, 4), binding.deft_kv_rows([], 8, 4), binding.deft_kv_copies([0], [1], 8)
    k, v = _part(), _part(x=1 << 21, out=1 << 25)

    def store(lst=rows.handle, image=1 << 16, q=None, k=k, v=v, n_rows=8, d=64, eps=0.0, positions=pos, rope=rope):
        return lib.deft_qkv_store(lst, image, q, k, v, n_rows, d, eps, 0.0, positions, rope, None)

    for bad in (dict(lst=None), dict(lst=copies.handle), dict(image=None), dict(image=24), dict(k=None), dict(v=None), dict(n_rows=7),
                dict(n_rows=-1), dict(v=_part(x=1 << 21, out=1 << 25, heads=3)), dict(k=_part(heads=0), v=_part(heads=0)),
                dict(v=_part(x=1 << 21, out=1 << 25, weight=1 << 12)), dict(v=_part(x=1 << 21)), dict(v=_part(x=1 << 21, out=(1 << 24) + 8 * 512 - 16)),
                dict(k=_part(out=1 << 20)), dict(q=_part(x=1 << 22, out=1 << 24)), dict(q=_part(x=(1 << 25) + 16, out=1 << 26)), dict(d=256)):
        assert store(**bad) == EINVAL, bad
    assert store(lst=none.handle, rope=None, positions=None) == 0


def test_keys_and_values_in_their_own_pool_are_refused():
    # token i goes to row rows[i]: where the heads are the pool's own rows another wave has yet to read that one
    lib, rope = binding.load_library(), binding.deft_rope(64).packed
    for at in ([7, 6, 5, 4, 3, 2, 1, 0], [1, 0], [0, 1, 2], [0]):
        n = len(at)
        rows = binding.deft_kv_rows(at, n, 4)

        def store(k, v, q=None):
            return lib.deft_qkv_store(rows.handle, 1 << 16, q, k, v, n, 64, 1e-6, 0.0, 1 << 12, rope, None)

        here, there = _part(out=1 << 20), _part(x=1 << 21, out=1 << 25)
        assert store(here, there) == store(there, here) == EINVAL, at
        assert store(here, _part(x=1 << 22, out=1 << 22)) == store(_part(x=1 << 20, weight=1 << 12, out=1 << 20), there) == EINVAL, at
        # nor is a pool the other's heads, or the queries
        assert store(_part(out=1 << 21), there) == store(there, _part(x=1 << 20, out=1 << 26), _part(x=1 << 26, out=1 << 27)) == EINVAL, at


def test_cpu_tensors_are_refused():
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    p, rope = torch.zeros(2, dtype=torch.int32), binding.deft_rope(64)
    rows = binding.deft_kv_rows([0, 1], 8, 1)
    for call in (lambda: binding.deft_rotate(x, p, rope), lambda: binding.deft_qk_norm_rotate(x, x), lambda: binding.deft_qkv_store(rows, x, x, x, (x, x))):
        with pytest.raises(binding.DeftError):
            call()


# ---- many heads: more than a launch holds ----

WAVES = 1 << 22  # of a launch, kMaxWaves in deft_heads.hip


@needs_gxx
@pytest.mark.parametrize("heads,d", [((65536, 65536, 65536), 128), ((65536, 1, 1), 64), ((40, 8, 8), 128)])
def test_calls_of_any_length(fake, heads, d):  # noqa: F811
    run(fake, f"""
class Fake(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in names] + [("grid", ctypes.c_int32 * 16), ("kernel", ctypes.c_void_p * 16)]
fake = Fake.in_dll(fake_lib, "fake")
H, d = {heads}, {d}
def part(i, out, heads):
    return binding._pack_heads(1 << 50 + i, heads * d, d, out, 0, 0, 0, heads)
def launched(n):
    fake.launches = 0
    pools = [part(i, (1 << 55) + (i << 53), H[i]) for i in range(3)]
    lst = binding.deft_kv_rows(np.arange(n), n, 1)
    assert lib.deft_qkv_store(lst.handle, 4096, *pools, n, d, 0.0, 0.0, 4096, binding.deft_rope(64).packed, 1 << 12) == 0
    return list(fake.grid[:fake.launches])
H = (H[0], H[1], H[1])
chunks = sum(-(-h // (64 // (d // 16))) for h in H)  # a wave has heads of one kind
most = {WAVES} // chunks
for n, want in ((1, [1]), (most, [most]), (most + 1, [most, 1]), (2 * most + 3, [most, most, 3])):
    if n < 1 << 20:
        assert launched(n) == [-(-x * chunks // 4) for x in want], n
""")


@pytest.mark.gpu
def test_heads_of_two_launches():
    # beside the same tokens in calls of one launch each
    n, H, d = 1100, 65536, 64
    x = torch.empty((n, H, d), dtype=torch.bfloat16, device=dev())
    x.view(torch.int16).random_(0, 0x4000)
    p, rope = on_gpu(positions(n)), binding.deft_rope(32)
    whole = binding.deft_rotate(x, p, rope)
    for a in range(0, n, 100):
        assert torch.equal(whole[a:a + 100], binding.deft_rotate(x[a:a + 100], p[a:a + 100], rope))
    del whole, x
    torch.cuda.empty_cache()


# ---- on the GPU ----

def dev():
    return torch.device("cuda:0")


def values(n, H, d, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, H, d), generator=g) * torch.exp(spread * torch.randn((n, H, 1), generator=g))
    return x.to(torch.bfloat16)


def laid_out(x, how):
    """The same values on the GPU in another layout."""
    n, H, d = x.shape
    if how == "dense":
        return x.to(dev())
    if how == "fused":  # a slice of a projection's output
        y = torch.zeros((n, H + 5, d), dtype=x.dtype, device=dev())[:, 2:2 + H]
    elif how == "between":  # q, k and v head by head
        y = torch.zeros((n, H, 3, d), dtype=x.dtype, device=dev())[:, :, 1]
    else:  # head by head, the tokens of each
        y = torch.zeros((H, n, d), dtype=x.dtype, device=dev()).transpose(0, 1)
    y.copy_(x)
    return y


def close(got, want, mag):
    """Half a step of bf16 of the value, and 2^-19 of the pair's magnitude for the arithmetic (19 additions of squares, 5.7e-7 behind
    the root; its reciprocal, two products and the weight's sum 2.4e-7; cosine and sine with the factor 2.1e-7; two products and a
    sum 1.8e-7: 1.2e-6 of 1.9e-6); below bf16's normal numbers their step."""
    got = got.double().cpu().numpy()
    finite = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all()
    assert (got[np.isinf(want)] == want[np.isinf(want)]).all()
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - (2.0 ** -8 * (1 + 2.0 ** -10) * np.abs(want) + 2.0 ** -19 * mag + 2.0 ** -133)
    assert (off[finite] <= 0).all(), (np.argwhere(finite & (off > 0))[:5], np.nanmax(off[finite]))


POSITIONS = [0, 1, -1, 2, 100000, 1 << 20, (1 << 31) - 1, -(1 << 31), 12345, 7]


def positions(n, seed=0):
    p = np.random.default_rng(seed).integers(0, 200000, n)
    p[:min(n, len(POSITIONS))] = POSITIONS[:n]
    return p.astype(np.int32)


def on_gpu(p):
    return torch.from_numpy(p).to(dev())


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 13, 300])
@pytest.mark.parametrize("H,d,rot", [(1, 64, 64), (5, 64, 16), (8, 128, 128), (3, 128, 48), (32, 128, 64), (17, 64, 48), (65, 128, 112)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotate_is_the_definition(n, H, d, rot, layout):
    how = SCALINGS[(n + H + rot) % len(SCALINGS)]
    rope, (f, factor) = binding.deft_rope(rot, layout=layout, **how), model.frequencies(rot, **how)
    p = positions(n, H)
    x = values(n, H, d, n + H)
    want, mag = model.heads(x.double().numpy(), p, f, factor, layout == "interleaved")
    for how in ("dense", "fused", "between", "by head"):
        y = laid_out(x, how)
        got = binding.deft_rotate(y, on_gpu(p), rope)
        assert got.is_contiguous() and got.shape == x.shape
        close(got, want, mag)
        assert torch.equal(got[..., rot:].cpu(), x[..., rot:])
        out = torch.empty_like(got)
        assert binding.deft_rotate(y, on_gpu(p), rope, out=out) is out and torch.equal(out, got)
        assert binding.deft_rotate(y, on_gpu(p), rope, out=y) is y and torch.equal(y, got)  # in place


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 3, 50])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 64), (32, 8, 128), (15, 5, 64), (6, 1, 128), (1, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("rot,layout", [(0, "half"), (16, "interleaved"), (64, "half"), (64, "interleaved")])
@pytest.mark.parametrize("wide,by_head,offset", [(True, False, 0.0), (False, True, 1.0)])
def test_norm_and_rotation_are_the_definition(n, Hq, Hkv, d, rot, layout, wide, by_head, offset):
    g = torch.Generator().manual_seed(n * Hq)
    base = torch.empty((n, Hq + 2 * Hkv, d), dtype=torch.bfloat16)
    base.copy_(values(n, Hq + 2 * Hkv, d, Hq, 3.0))
    gpu = base.to(dev())
    q, k = gpu[:, :Hq], gpu[:, Hq:Hq + Hkv]
    weights = [(1 - offset + 0.3 * torch.randn((H, d) if by_head else (d,), generator=g)).to(torch.float32 if wide else torch.bfloat16) for H in (Hq, Hkv)]
    rope = binding.deft_rope(rot, layout=layout) if rot else None
    f, factor = model.frequencies(rot) if rot else (None, 1.0)
    p = positions(n, 3)
    for both in (weights, [weights[0], None], [None, weights[1]], [None, None]):
        want = [model.heads(x.double().numpy(), p, f, factor, layout == "interleaved", None if w is None else w.double().numpy(), 1e-5, offset)
                for x, w in zip((base[:, :Hq], base[:, Hq:Hq + Hkv]), both)]
        w = [None if t is None else t.to(dev()) for t in both]
        got = binding.deft_qk_norm_rotate(q, k, *w, on_gpu(p) if rot else None, rope, eps=1e-5, weight_offset=offset)
        for x, (y, mag) in zip(got, want):
            close(x, y, mag)
        # in place in the projection's output, whose values stay as they are
        mine = gpu.clone()
        binding.deft_qk_norm_rotate(mine[:, :Hq], mine[:, Hq:Hq + Hkv], *w, on_gpu(p) if rot else None, rope, eps=1e-5, weight_offset=offset,
                                    q_out=mine[:, :Hq], k_out=mine[:, Hq:Hq + Hkv])
        assert torch.equal(mine[:, :Hq], got[0]) and torch.equal(mine[:, Hq:Hq + Hkv], got[1]) and torch.equal(mine[:, Hq + Hkv:], gpu[:, Hq + Hkv:])


@pytest.mark.gpu
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 128)])
def test_extreme_heads(d, rot):
    # zeros, one element, magnitudes whose squares leave fp32 on either side, infinities, NaN; each in a head of its own
    x = values(14, 2, d, 5, 0.0)
    x[0] = 0
    x[1] = 0
    x[1, :, 3] = 2.0
    x[2] = (x[2].float() * 1e25).to(torch.bfloat16)
    x[3] = (x[3].float() * 1e-25).to(torch.bfloat16)
    x[4] = torch.where(x[4] > 0, 1e38, -1e38)
    x[5] = torch.where(x[5] > 0, 2.0 ** -133, 0.0)
    x[6, 0, 5], x[6, 1, d - 1], x[7, 0, 0], x[7, 1, rot // 2] = math.inf, -math.inf, math.nan, math.inf
    x[8, :, 1] = 3e38
    w = values(1, 1, d, 6, 0.0)[0, 0]
    p = positions(14, 1)
    f, factor = model.frequencies(rot)
    rope = binding.deft_rope(rot)
    for eps in (1e-6, 0.0, 10.0, 1e30):
        if eps == 0.0:  # (0 / 0 by definition)
            x[0, :, 0] = 1e-38
        want, mag = model.heads(x.double().numpy(), p, f, factor, False, w.double().numpy(), eps)
        got, k = binding.deft_qk_norm_rotate(x.to(dev()), x[:, :1].to(dev()), w.to(dev()), w.to(dev()), on_gpu(p), rope, eps=eps)
        close(got, want, mag)
        close(k, want[:, :1], mag[:, :1])
    # without a norm infinities stay with their pair, NaN too, and elements that do not turn keep their bits
    keep = [i for i in range(14) if i not in (4, 8)]
    want, mag = model.heads(x[keep].double().numpy(), p[keep], f, factor, False)
    got = binding.deft_rotate(x[keep].to(dev()), on_gpu(p[keep]), rope)
    close(got, want, mag)
    assert torch.equal(got[..., rot:].cpu().view(torch.int16), x[keep][..., rot:].view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_weights_at_the_ends_of_their_range(d, eps):
    # heads of any magnitude with weights from 2^-60 to 2^80 and zeros: their product with the root's reciprocal stays within fp32
    scale = [2.0 ** 120, 2.0 ** 50, 2.0 ** 49, 1.0, 2.0 ** -39, 2.0 ** -40, 2.0 ** -120]
    x = values(len(scale), 3, d, 9, 0.0)
    x = (x.double() * torch.tensor(scale, dtype=torch.float64)[:, None, None]).to(torch.bfloat16)
    rng = np.random.default_rng(d)
    w = torch.from_numpy(rng.choice([2.0 ** -60, -(2.0 ** -60), 1.0, 0.0, 2.0 ** 80, -(2.0 ** 80)], (3, d)).astype(np.float32))
    p = positions(len(scale), 2)
    for rope, f in ((None, None), (binding.deft_rope(d), model.frequencies(d)[0])):
        for wide in (True, False):
            weight = w if wide else w.to(torch.bfloat16)
            want = model.heads(x.double().numpy(), p, f, 1.0, False, weight.double().numpy(), eps)
            got, _ = binding.deft_qk_norm_rotate(x.to(dev()), x[:, :0].to(dev()), weight.to(dev()), None, on_gpu(p), rope, eps=eps)
            close(got, *want)


@pytest.mark.gpu
@pytest.mark.parametrize("d,H", [(128, 9), (64, 17)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_every_pair_has_its_own_angle_in_every_wave(d, H, layout):
    # a lane makes one pair's angle and the others of its wave read it: frequencies and positions that are all different, waves of
    # several batches of heads, and the same tokens in other waves and workgroups
    n = 2000
    rng = np.random.default_rng(d)
    f = rng.uniform(-3, 3, d // 2)
    rope = binding.deft_rope(d, layout=layout, frequencies=f)
    p = rng.permutation(1 << 20)[:n].astype(np.int32)
    x = values(n, H, d, 3)
    got = binding.deft_rotate(x.to(dev()), on_gpu(p), rope)
    close(got, *model.heads(x.double().numpy(), p, f, 1.0, layout == "interleaved"))
    for _ in range(3):
        at = torch.from_numpy(rng.permutation(n)[:n - 7])
        assert torch.equal(binding.deft_rotate(x[at].to(dev()), on_gpu(p)[at.to(dev())], rope), got[at.to(dev())])
    # the waves of the queries in a store into an 8-bit cache
    cache = binding.alloc_kv_cache_q8(n, 2, d, 16, dev())
    q = binding.deft_qkv_store_q8(binding.deft_kv_rows(np.arange(n), n, 16), x.to(dev()), x[:, :2].to(dev()), x[:, 2:4].to(dev()), cache, on_gpu(p), rope)
    assert torch.equal(q, got)


@pytest.mark.gpu
def test_turning_back_and_relative_positions():
    rope = binding.deft_rope(128)
    x = values(64, 8, 128, 1, 0.0).to(dev())
    p = on_gpu(positions(64))
    p[7] = 5  # (the lowest number has no opposite)
    back = binding.deft_rotate(binding.deft_rotate(x, p, rope), -p, rope)
    # two roundings to bf16, of the first a share of either element of the pair
    mag = torch.hypot(x[..., :64].float(), x[..., 64:].float()).repeat(1, 1, 2)
    assert ((back.float() - x.float()).abs() <= 2.0 ** -8 * (2.0 ** 0.5 * mag + x.float().abs()) * (1 + 2.0 ** -6)).all()
    # turning by a sum is turning twice: products of turned queries and keys go by the distance
    one, two = on_gpu(np.full(64, 1000, np.int32)), p.clamp(0, 1 << 20)
    a = binding.deft_rotate(x, two, rope).float()
    b = binding.deft_rotate(x, two + one, rope).float()
    c = binding.deft_rotate(x, one, rope).float()
    x = x.float()
    err = ((a * b).sum(-1) - (x * c).sum(-1)).abs()
    assert (err <= 2.0 ** -8 * 4 * (x * x).sum(-1)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,Hq,Hkv,d,rows,block", [(1, 4, 4, 64, 5, 1), (20, 32, 8, 128, 333, 16), (77, 5, 5, 64, 100, 1), (300, 6, 1, 128, 640, 64), (1000, 0, 3, 64, 1000, 32)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("ascending", [False, True])
def test_store_puts_heads_into_their_rows(n, Hq, Hkv, d, rows, block, norm, ascending):
    rng = np.random.default_rng([n, rows])
    at = rng.permutation(rows)[:n]
    at = np.sort(at) if ascending else at
    lst = binding.deft_kv_rows(at, rows, block)
    x = values(n, Hq + 2 * Hkv, d, n)
    x[0, Hq + Hkv] = torch.tensor([0x7fa5, -1], dtype=torch.int16).repeat(d // 2).view(torch.bfloat16)  # NaN with bits of their own
    gpu = x.to(dev())
    q, k, v = gpu[:, :Hq], gpu[:, Hq:Hq + Hkv], gpu[:, Hq + Hkv:]
    pools = [values(rows, Hkv, d, 7 + i).to(dev()) for i in range(2)]
    before = [t.clone() for t in pools]
    w = torch.rand(d, device=dev()) if norm else None
    rope, (f, factor), p = binding.deft_rope(d // 2), model.frequencies(d // 2), positions(n)
    got = binding.deft_qkv_store(lst, q if Hq else None, k, v, pools, on_gpu(p), rope, q_weight=w if Hq else None, k_weight=w)
    if Hq:
        want, want_k = binding.deft_qk_norm_rotate(q, k, w, w, on_gpu(p), rope)
        assert torch.equal(got, want)
    else:
        assert got is None
        want_k = binding.deft_qk_norm_rotate(k, k, w, w, on_gpu(p), rope)[1]
    close(want_k, *model.heads(x[:, Hq:Hq + Hkv].double().numpy(), p, f, factor, False, w.double().cpu().numpy() if norm else None))
    i = torch.from_numpy(at).to(dev())
    before[0][i], before[1][i] = want_k, v
    for a, b in zip(pools, before):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    if Hq:  # the queries where they are
        mine = gpu.clone()
        assert torch.equal(binding.deft_qkv_store(lst, mine[:, :Hq], mine[:, Hq:Hq + Hkv], mine[:, Hq + Hkv:], pools, on_gpu(p), rope, q_weight=w, k_weight=w,
                                                  q_out=mine[:, :Hq]), want)
        assert torch.equal(mine[:, Hq:].view(torch.int16), gpu[:, Hq:].view(torch.int16))


@pytest.mark.gpu
def test_positions_say_nothing_without_a_rope():
    x, p = values(5, 6, 64, 1).to(dev()), on_gpu(positions(5))
    w = torch.rand(64, device=dev())
    for a, b in zip(binding.deft_qk_norm_rotate(x[:, :4], x[:, 4:], w, None, p), binding.deft_qk_norm_rotate(x[:, :4], x[:, 4:], w, None)):
        assert torch.equal(a, b)
    assert torch.equal(b, x[:, 4:])


@pytest.mark.gpu
def test_nothing_to_do():
    rope, x = binding.deft_rope(64), torch.zeros((0, 4, 64), dtype=torch.bfloat16, device=dev())
    p = torch.zeros(0, dtype=torch.int32, device=dev())
    assert binding.deft_rotate(x, p, rope).shape == (0, 4, 64)
    assert [t.shape[1] for t in binding.deft_qk_norm_rotate(x, x[:, :2], None, None, p, rope)] == [4, 2]
    y, p = torch.zeros((3, 0, 64), dtype=torch.bfloat16, device=dev()), torch.zeros(3, dtype=torch.int32, device=dev())
    assert binding.deft_rotate(y, p, rope).shape == (3, 0, 64)
    pools = [torch.ones((8, 2, 64), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    q = binding.deft_qkv_store(binding.deft_kv_rows([], 8, 1), x, x[:, :2], x[:, :2], pools)
    assert q.shape == (0, 4, 64) and all((t == 1).all() for t in pools)


@pytest.mark.gpu
def test_rows_behind_four_billion_elements():
    n_rows, Hkv, d = 4_300_000, 8, 128  # 4.4e9 elements a pool
    pools = [torch.empty((n_rows, Hkv, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    at = np.array([n_rows - 1, 0, 2_100_000, 4_194_304])
    x = values(4, 3 * Hkv, d, 1).to(dev())
    p = on_gpu(positions(4))
    rope = binding.deft_rope(d)
    binding.deft_qkv_store(binding.deft_kv_rows(at, n_rows, 64), x[:, :Hkv], x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:], pools, p, rope)
    i = torch.from_numpy(at).to(dev())
    assert torch.equal(pools[0][i], binding.deft_rotate(x[:, Hkv:2 * Hkv], p, rope)) and torch.equal(pools[1][i], x[:, 2 * Hkv:])
    # heads that lie as far apart
    far = pools[0].view(4, -1)[:, :Hkv * d].view(4, Hkv, d)
    far.copy_(x[:, :Hkv])
    assert torch.equal(binding.deft_rotate(far, p, rope), binding.deft_rotate(x[:, :Hkv], p, rope))
    del pools, far
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_gpu_refusals():
    n, d = 4, 64
    x = torch.zeros((n, 6, d), dtype=torch.bfloat16, device=dev())
    q, k, v = x[:, :2], x[:, 2:4], x[:, 4:]
    p, rope = torch.zeros(n, dtype=torch.int32, device=dev()), binding.deft_rope(64)
    w, wide = torch.ones(d, dtype=torch.bfloat16, device=dev()), torch.ones(d, device=dev())
    pools = [torch.zeros((8, 2, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    rows = binding.deft_kv_rows([0, 1, 2, 3], 8, 1)
    cache = binding.alloc_kv_cache_q8(8, 2, d, 1)
    store, norm, rotate = binding.deft_qkv_store, binding.deft_qk_norm_rotate, binding.deft_rotate
    dense = torch.zeros((n, 2, d), dtype=torch.bfloat16, device=dev())
    bad = [
        lambda: rotate(x.float(), p, rope), lambda: rotate(x[0], p, rope), lambda: rotate(x, p.long(), rope), lambda: rotate(x, p[:3], rope), lambda: rotate(x, p.cpu(), rope),
        lambda: rotate(x, None, rope), lambda: rotate(x, p, None), lambda: rotate(x[..., :32], p, rope), lambda: rotate(x[..., ::2], p, rope),
        lambda: rotate(x, p, binding.deft_rope(128)), lambda: rotate(x, p, rope, out=x[:, :5]), lambda: rotate(x, p, rope, out=x.float()),
        lambda: rotate(q, p, rope, out=k), lambda: rotate(q, p, rope, out=x.view(-1)[:n * 2 * d].view(n, 2, d)), lambda: rotate(q, p, rope, out=x.view(-1)[64:64 + n * 2 * d].view(n, 2, d)),
        lambda: rotate(x.view(-1)[4:4 + 2 * d].view(1, 2, d), p[:1], rope), lambda: rotate(x[:, :1].expand(n, 3, d), p, rope, out=x[:, :1].expand(n, 3, d)),
        lambda: norm(q, k, w, wide, p, rope), lambda: norm(q, k, w[:32], None, p, rope), lambda: norm(q, k, w.half(), None, p, rope), lambda: norm(q, k, w.cpu(), None, p, rope),
        lambda: norm(q, k, w, w, None, rope), lambda: norm(q, k, w, w, p, rope, eps=-1.0), lambda: norm(q, k, w.expand(3, d), w, p, rope),
        lambda: norm(q, k[:3], w, w, p, rope), lambda: norm(q, k.cpu(), w, w, p, rope), lambda: norm(q, q, w, w, p, rope, q_out=q, k_out=q),
        lambda: norm(q, k, w, w, p, rope, q_out=dense, k_out=dense), lambda: norm(dense, k, w, w, p, rope, k_out=dense),
        lambda: store(rows, q, k, v, cache, p, rope), lambda: store(rows, q, k, v, pools[:1], p, rope), lambda: store(rows, q, k, v, (pools[0], pools[0]), p, rope),
        lambda: store(rows, q, k, v[:, :1], pools, p, rope), lambda: store(rows, q, k[:3], v, pools, p, rope), lambda: store(rows, q, k, v, [t[:3] for t in pools], p, rope),
        lambda: store(rows, q, k, v, [t[:, :1] for t in pools], p, rope), lambda: store(rows, q, k, v, [t.float() for t in pools], p, rope),
        lambda: store(binding.deft_kv_copies([0], [1], 8), q, k, v, pools, p, rope), lambda: store(rows, None, k, v, pools, p, rope, q_weight=w),
        lambda: store(rows, pools[0][:4], k, v, pools, p, rope), lambda: store(rows, q, k, v, pools, p, rope, q_out=pools[1][:4]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.DeftError):
            call()
            pytest.fail(f"call {i}")
    torch.cuda.synchronize()
    assert not x.any() and not any(t.any() for t in pools)


@pytest.mark.gpu
def test_heads_longer_than_thirty_two_bits_say_are_refused():
    x = torch.empty((1, 1, (1 << 32) + 64), dtype=torch.bfloat16, device=dev())
    p, rope, rows = torch.zeros(1, dtype=torch.int32, device=dev()), binding.deft_rope(64), binding.deft_kv_rows([0], 1, 1)
    for call in (lambda: binding.deft_rotate(x, p, rope, out=x), lambda: binding.deft_qk_norm_rotate(x, x, None, None, p, rope, q_out=x, k_out=x),
                 lambda: binding.deft_qkv_store(rows, None, x, x, (x, x), p, rope)):
        with pytest.raises(binding.DeftError, match="must be"):
            call()
    del x
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_captured_and_replayed():
    n, Hq, Hkv, d = 40, 8, 2, 128
    rope, rng = binding.deft_rope(64, layout="interleaved"), np.random.default_rng(0)
    x, p = values(n, Hq + 2 * Hkv, d, 1).to(dev()), on_gpu(positions(n))
    w = torch.rand(d, device=dev())
    pools = [torch.zeros((200, Hkv, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    rows = binding.deft_kv_rows(rng.permutation(200)[:n], 200, 1)  # first used inside the capture

    def step():
        return binding.deft_qkv_store(rows, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pools, p, rope, q_weight=w, k_weight=w)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q = step()
        turned = binding.deft_rotate(q, p, rope)
    for i in range(4):
        x.copy_(values(n, Hq + 2 * Hkv, d, 10 + i))
        p.copy_(on_gpu(positions(n, i)))
        w.uniform_()
        graph.replay()
        got = [t.clone() for t in (q, turned, *pools)]
        for t in pools:
            t.zero_()
        want = step()
        assert torch.equal(got[0], want) and torch.equal(got[1], binding.deft_rotate(want, p, rope))
        assert all(torch.equal(a, b) for a, b in zip(got[2:], pools))
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_other_streams():
    n, Hq, Hkv, d = 4000, 16, 4, 128
    rope, side = binding.deft_rope(128), torch.cuda.Stream()
    x, p = values(n, Hq + 2 * Hkv, d, 1).to(dev()), on_gpu(positions(n))
    pools = [torch.zeros((n, Hkv, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    rows = binding.deft_kv_rows(np.random.default_rng(2).permutation(n), n, 1)
    args = rows, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pools, p, rope
    want = binding.deft_qkv_store(*args)
    want_k = pools[0].clone()
    pools[0].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        q = binding.deft_qkv_store(*args, stream=side)
        a, b = binding.deft_qk_norm_rotate(args[1], args[2], None, None, p, rope, stream=side)
        c = binding.deft_rotate(args[1], p, rope, stream=side.cuda_stream)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(q, want) and torch.equal(a, want) and torch.equal(c, want) and torch.equal(pools[0], want_k)
        assert torch.equal(b, binding.deft_rotate(args[2], p, rope))

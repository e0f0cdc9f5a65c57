"""Logits bent by the tokens of each query's path, by biases and by masks: against the definition in 64 bits (oracle/logits.py)."""

import math

import numpy as np
import pytest
import torch

from oracle import logits as model
from paper_2404_00242_amd import binding, workloads as wl

EINVAL, EWORKSPACE, ENOTREADY = -1, -3, -5
PROMPT = binding.DEFT_TOKEN_PROMPT


def plan_of(t, chunk=0, flags=0, page=0, seed=0):
    """(plan, pool row of every row of the contiguous cache, rows of the pool)"""
    if not page:
        return binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, t.query_node, t.ntok, chunk, flags), np.arange(t.ntok), t.ntok
    pp, pg, npool, row_of = wl.to_paged(t, page, seed=seed)
    return binding.deft_plan_paged(pp, pg, page, npool, t.node_tok_len, t.node_parent, t.query_node, chunk, flags), row_of, npool * page


# ---- refusals (CPU: addresses that nothing reads) ----

def test_calls_that_are_refused():
    lib = binding.load_library()
    t = wl.random_tree(3, n_nodes=5, nq=4)
    plan = plan_of(t)[0]
    rows = plan.limits()[1]

    def call(plan=plan.handle, image=0, group=1, logits=1 << 20, out=1 << 24, stride=1000, out_stride=1000, vocab=1000, wide=1, out_wide=1, n_bias=0, n_masks=0, reserved=0,
             tokens=0, n_tokens=0, repetition=0, frequency=0, presence=0, bias=0, bias_row=0, bias_stride=0, mask=0, mask_row=0, mask_stride=0):
        packed = binding._pack_logits(logits, out, stride, out_stride, vocab, wide, out_wide, n_bias, n_masks, reserved, tokens, n_tokens, repetition, frequency,
                                      presence, bias, bias_row, bias_stride, mask, mask_row, mask_stride)
        return lib.deft_adjust_logits(plan, image, group, packed, None, 0, None)

    at = 1 << 12
    for bad in (dict(plan=None), dict(logits=0), dict(out=0), dict(vocab=0), dict(vocab=-5), dict(vocab=(1 << 28) + 1, stride=1 << 29, out_stride=1 << 29),
                dict(out_stride=999), dict(stride=-1000), dict(stride=1 << 32), dict(out_stride=1 << 32), dict(logits=(1 << 20) + 2), dict(out=(1 << 24) + 2),
                dict(wide=0, logits=(1 << 20) + 1), dict(wide=0, out_wide=0, out=(1 << 24) + 1), dict(out_wide=0),
                dict(out=(1 << 20) + 4), dict(out=1 << 20, out_stride=1001), dict(out=1 << 20, wide=0), dict(out=(1 << 20) - 8000),
                dict(bias=at), dict(bias=at + 2, n_bias=1), dict(bias=at, n_bias=-1), dict(bias=at, n_bias=2, bias_stride=999), dict(bias_row=at),
                dict(bias=at, n_bias=1, bias_row=at + 1), dict(mask=at), dict(mask=at + 2, n_masks=1), dict(mask=at, n_masks=2, mask_stride=31), dict(mask_row=at),
                dict(mask=at, n_masks=1, mask_row=at + 2), dict(reserved=1), dict(bias=at, n_bias=2, bias_stride=1 << 32), dict(mask=at, n_masks=2, mask_stride=1 << 32),
                # what is written meets what is read
                dict(bias=(1 << 24) + 12000, n_bias=1), dict(bias=(1 << 24) - 4000, n_bias=3, bias_stride=1000), dict(bias=at, n_bias=1, bias_row=(1 << 24) + 4),
                dict(mask=(1 << 24) - 4, n_masks=1), dict(mask=at, n_masks=1, mask_row=(1 << 24) + 15996),
                dict(repetition=at), dict(frequency=at, tokens=at, n_tokens=rows - 1), dict(presence=at + 2, tokens=at, n_tokens=rows),
                dict(presence=at, tokens=at + 2, n_tokens=rows), dict(repetition=at, tokens=at, n_tokens=rows), dict(repetition=at, tokens=at, n_tokens=rows, image=at + 8),
                dict(repetition=at, tokens=at, n_tokens=rows, image=at, group=0)):
        assert call(**bad) == EINVAL, bad
    assert lib.deft_adjust_logits(plan.handle, None, 1, None, None, 0, None) == EINVAL
    history = dict(tokens=at, n_tokens=rows, image=1 << 16, group=3)
    assert call(repetition=at, **history) == ENOTREADY
    assert lib.deft_plan_upload(plan.handle, 3, 1, 1 << 16, 0, None) == EWORKSPACE  # (the schedule is made, nothing is copied)
    for bad in (dict(repetition=(1 << 24) + 8), dict(presence=(1 << 24) - 12), dict(frequency=1 << 24), dict(repetition=at, tokens=(1 << 24) - 4)):
        assert call(**{**history, **bad}) == EINVAL, bad
    nobody = binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, [], t.ntok)
    assert call(plan=nobody.handle, logits=0, out=0) == 0
    with pytest.raises(binding.DeftError):
        binding.deft_adjust_logits(plan, torch.zeros((4, 10)))


def test_more_workgroups_than_a_launch_holds_are_refused():
    plan = binding.deft_plan([0], [1], [-1], [0] * 300, 1)
    packed = binding._pack_logits(1 << 20, 1 << 52, 1 << 28, 1 << 28, 1 << 28, 1, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    assert binding.load_library().deft_adjust_logits(plan.handle, 0, 1, packed, None, 0, None) == EINVAL  # 2^18 * 38, not below 2^23


def test_an_image_is_looked_for_while_another_thread_adds_one():
    t = wl.random_tree(3, n_nodes=5, nq=4)
    plan = plan_of(t)[0]

    class Index(int):  # a device's number; while it is compared, another thread makes an image
        def __eq__(self, other):
            plan._images.of[(len(plan._images.of) + 10, 7)] = image
            return int(self) == other

        __hash__ = int.__hash__

    image = binding._Images._Image()
    image.tensor, image.event, image.first, image.streams = torch.zeros(1), None, 5, {5}
    plan._images.of.update({(4, Index(1)): image, (2, Index(1)): image, (3, Index(0)): image})
    assert plan._any_image(0, 5, 0) == (image.tensor.data_ptr(), 3)
    assert len(plan._images.of) > 3


def _tree(kind, **sizes):
    return getattr(wl, kind)(**sizes)


@pytest.mark.parametrize("sorts,vocab,tree,plan", [
    (False, 5003, ("random_tree", dict(seed=5003, n_nodes=14, max_len=90, nq=11, n_roots=2)), {}),
    (False, 777, ("random_tree", dict(seed=902, n_nodes=37, max_len=150, nq=40, n_roots=3)), dict(chunk=64, page=16)),
    (True, 777, ("random_tree", dict(seed=902, n_nodes=37, max_len=150, nq=40, n_roots=3)), dict(chunk=64, page=1)),
    (False, 777, ("random_tree", dict(seed=901, n_nodes=20, max_len=40, nq=9, n_roots=2)), dict(chunk=64, page=1)),
    (True, 777, ("random_tree", dict(seed=903, n_nodes=54, max_len=90, nq=100, n_roots=4)), dict(chunk=64, flags=binding.SPLIT_MODES["query"])),
    (True, 30011, ("random_tree", dict(seed=77, n_nodes=300, max_len=12, nq=1100, n_roots=3)), {}),
    (True, 2500, ("config5_longcontext", dict(root=6000, branches=9, lo=1, hi=700)), dict(flags=binding.DEFT_SPLIT_BALANCED | binding.rows_per_query(4))),
    (True, 2500, ("config5_longcontext", dict(root=6000, branches=9, lo=1, hi=700)), dict(page=1)),
    (True, 3000, ("config5_longcontext", dict(root=6000, branches=9, lo=1, hi=700)), dict(page=16)),
    (True, 5000, ("config2_fewshot", dict(prefix=290_000, branches=3, gen=20_000)), dict(chunk=1024)),
    (True, 2000, ("config2_fewshot", dict(prefix=70000, branches=3, gen=5)), {}),
    (False, 3001, ("random_tree", dict(seed=18, n_nodes=20, max_len=50, nq=30)), {}),
    (True, 20000, ("config5_longcontext", dict(root=3000, branches=16, lo=10, hi=300)), {}),
], ids=str)
def test_trees_of_the_tests_below_take_the_form_that_is_meant(sorts, vocab, tree, plan):
    # both forms are tested below, by these trees: where the line between them moves, they have to move with it
    plan = plan_of(_tree(tree[0], **tree[1]), **plan)[0]
    assert (binding.load_library().deft_logits_workspace_bytes(plan.handle, vocab) > 0) == sorts


@pytest.mark.parametrize("page,unsorted,sorted_", [(1, (1, 512, 513, 600, 1000, 1500), (2500, 8193)), (8, (4096, 4097, 7000), (8193, 12000)), (16, (8191,), (9500, 16000)),
                                                   (64, (8191, 8193, 10000), (12000, 32000))])
def test_the_line_from_which_tokens_are_sorted_goes_by_tokens_and_pieces(page, unsorted, sorted_):
    # pieces add to the cost as they are measured to; 512 of them, which are looked at together, are no limit by themselves
    room = binding.load_library().deft_logits_workspace_bytes

    def plan(n):
        t = wl.Tree("line", np.array([0]), np.array([n]), np.array([-1]), np.array([0]), n, 8, 2, 128)
        return plan_of(t, page=page)[0]

    for vocab in (32000, 128000):
        for n in unsorted:
            assert room(plan(n).handle, vocab) == 0, (n, vocab)
        for n in sorted_:
            assert room(plan(n).handle, vocab) > 0, (n, vocab)


# ---- on the GPU ----

def dev():
    return torch.device("cuda:0")


def gpu(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev())


class Inputs:
    """Everything that a call can be given, on the host, for a tree whose rows lie in a pool as row_of says."""

    def __init__(self, t, vocab, seed, wide, prompts=True):
        rng = np.random.default_rng(seed)
        self.t, self.vocab, self.rng = t, vocab, rng
        x = torch.from_numpy(4.0 * rng.standard_normal((t.nq, vocab)).astype(np.float32))
        self.x = x if wide else x.to(torch.bfloat16)
        # few tokens often; tokens that are none, in every way
        self.tokens = (vocab * rng.random(t.ntok) ** 4).astype(np.int32)
        if prompts:
            some = rng.random(t.ntok) < 0.4
            self.tokens[some] |= PROMPT
        odd = rng.random(t.ntok) < 0.05
        self.tokens[odd] = rng.choice([-1, -(1 << 31), vocab, (1 << 31) - 1, vocab | PROMPT, -PROMPT], int(odd.sum()))
        f32 = np.float32
        self.repetition, self.frequency, self.presence = (f32(1) + rng.random(t.nq).astype(f32), rng.standard_normal(t.nq).astype(f32), rng.standard_normal(t.nq).astype(f32))
        self.bias = np.where(rng.random((3, vocab)) < 0.1, 5 * rng.standard_normal((3, vocab)), 0).astype(f32)
        self.mask = rng.integers(-(1 << 31), 1 << 31, (5, -(-vocab // 32))).astype(np.int32)
        self.mask[3] = 0  # a state that allows nothing
        self.mask[4] = -1
        self.bias_row, self.mask_row = rng.integers(-1, 4, t.nq).astype(np.int32), rng.integers(-1, 6, t.nq).astype(np.int32)  # (3 and 5 are no rows)

    def call(self, plan, row_of, pool, out_dtype=None, stream=None, x=None, **which):
        tokens = None
        if any(which.get(k) for k in ("repetition", "frequency", "presence")):
            tokens = np.full(pool, 3, np.int32)  # (rows that no path holds)
            owned = row_of >= 0
            tokens[row_of[owned]] = self.tokens[owned]
        args = {k: gpu(getattr(self, k)) for k in which if which[k]}
        return binding.deft_adjust_logits(plan, self.x.to(dev()) if x is None else x, gpu(tokens), out_dtype=out_dtype, stream=stream, **args)

    def want(self, **which):
        return model.adjust(self.t, self.x.double().numpy(), self.tokens, **{k: getattr(self, k) for k in which if which[k]})


def close(got, want, mag):
    """Each of the at most six fp32 roundings (1 / repetition, the product; frequency * count + presence; two sums; 2^-24 each) is
    relative to no more than `mag`; bf16 results are rounded once more, 2^-8."""
    bf16 = got.dtype == torch.bfloat16
    got = got.double().cpu().numpy()
    assert (np.isnan(got) == np.isnan(want)).all()
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all()
    with np.errstate(invalid="ignore"):
        off = np.abs(got - want) - (6 * 2.0 ** -24 * mag * 1.001 + (2.0 ** -8 * 1.001 * np.abs(want) if bf16 else 0) + 2.0 ** -126)
    bad = np.isfinite(want) & ~(off <= 0)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


ALL = dict(repetition=True, frequency=True, presence=True, bias=True, bias_row=True, mask=True, mask_row=True)
SOME = [dict(repetition=True), dict(presence=True), dict(frequency=True), dict(repetition=True, presence=True, mask=True, mask_row=True), dict(bias=True, bias_row=True),
        dict(mask=True), dict(bias=True, mask=True, mask_row=True), ALL]


@pytest.mark.gpu
@pytest.mark.parametrize("which", SOME, ids=lambda w: "+".join(w))
@pytest.mark.parametrize("vocab", [1, 31, 1024, 1027, 5003])
@pytest.mark.parametrize("types", ["f32", "bf16", "bf16 f32"])
def test_every_part_of_the_formula(which, vocab, types):
    t = wl.random_tree(vocab, n_nodes=14, max_len=90, nq=11, n_roots=2)
    s = Inputs(t, vocab, vocab, types == "f32")
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    got = s.call(plan, row_of, pool, out_dtype=torch.float32 if types == "bf16 f32" else None, **which)
    assert got.dtype == (torch.bfloat16 if types == "bf16" else torch.float32)
    close(got, *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("mode", sorted(binding.SPLIT_MODES))
@pytest.mark.parametrize("page", [0, 1, 16])
@pytest.mark.parametrize("seed", range(4))
def test_trees_of_any_kind(mode, page, seed):
    t = wl.random_tree(900 + seed, n_nodes=3 + 17 * seed, max_len=[1, 40, 150, 90][seed], nq=[1, 9, 40, 100][seed], n_roots=1 + seed)
    s = Inputs(t, 777, seed, True)
    plan, row_of, pool = plan_of(t, 64, binding.SPLIT_MODES[mode], page, seed)
    plan.image(t.Hq, t.Hkv, dev())
    for which in (ALL, dict(repetition=True, presence=True)):
        close(s.call(plan, row_of, pool, **which), *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
def test_more_queries_than_a_workgroup_takes(counts):
    t = wl.random_tree(77, n_nodes=300, max_len=12, nq=1100, n_roots=3)
    s = Inputs(t, 30011, 5, True)
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    which = dict(repetition=True, presence=True, frequency=counts)
    got = s.call(plan, row_of, pool, **which).cpu()
    some = np.concatenate([np.arange(0, 1100, 13), [1099]])
    t.query_node = t.query_node[some]
    s.x = s.x[some]
    for k in ("repetition", "presence", "frequency"):
        setattr(s, k, getattr(s, k)[some])
    close(got[some], *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
@pytest.mark.parametrize("page", [0, 1, 16])
def test_paths_of_many_pieces(counts, page):
    # a long prompt, and branches behind it; of pages of one row every token is a piece
    t = wl.config5_longcontext(root=6000, branches=9, lo=1, hi=700)
    s = Inputs(t, 2500, page, False)
    plan, row_of, pool = plan_of(t, 0, binding.DEFT_SPLIT_BALANCED | binding.rows_per_query(4), page, 1)
    plan.image(t.Hq, t.Hkv, dev())
    which = dict(repetition=True, presence=True, frequency=counts, mask=True, mask_row=True)
    close(s.call(plan, row_of, pool, **which), *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
@pytest.mark.parametrize("page", [0, 16])
def test_without_a_workspace_and_with_a_large_vocabulary(counts, page):
    # the tokens are then looked through as they are
    t = wl.config5_longcontext(root=6000, branches=9, lo=1, hi=700)
    s = Inputs(t, 3000, 1, True)
    plan, row_of, pool = plan_of(t, 0, 0, page, 1)
    plan.image(t.Hq, t.Hkv, dev())
    which = dict(repetition=True, presence=True, frequency=counts)
    want = s.call(plan, row_of, pool, **which)
    plan._logits_workspace = lambda *args: (0, 0)
    assert torch.equal(s.call(plan, row_of, pool, **which), want)
    s = Inputs(t, 2_200_000, 1, False)
    plan, row_of, pool = plan_of(t, 0, 0, page, 1)
    plan.image(t.Hq, t.Hkv, dev())
    room = binding.load_library().deft_logits_workspace_bytes
    assert room(plan.handle, 2_200_000) == 0 < room(plan.handle, 2_000_000)
    close(s.call(plan, row_of, pool, **which), *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
@pytest.mark.parametrize("page", [0, 64])
def test_more_tokens_than_are_taken_at_a_time(counts, page):
    # sorted tokens come in groups of 1024, of which 256 are looked at together; unsorted pieces 512 together
    t = wl.config2_fewshot(prefix=290_000, branches=3, gen=20_000)
    s = Inputs(t, 5000, page, True)
    plan, row_of, pool = plan_of(t, 1024, 0, page, 1)
    plan.image(t.Hq, t.Hkv, dev())
    which = dict(repetition=True, presence=True, frequency=counts)
    got = s.call(plan, row_of, pool, **which)
    close(got, *s.want(**which))
    plan._logits_workspace = lambda *args: (0, 0)
    assert torch.equal(s.call(plan, row_of, pool, **which), got)


@pytest.mark.gpu
def test_one_token_more_often_than_sixteen_bits_hold():
    t = wl.config2_fewshot(prefix=70000, branches=3, gen=5)
    s = Inputs(t, 2000, 1, True, prompts=False)
    s.tokens[:69000] = 1999
    s.frequency[:] = [0.5, -0.001, 2.0 ** -12]
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    which = dict(frequency=True, repetition=True)
    close(s.call(plan, row_of, pool, **which), *s.want(**which))


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [False, True])
def test_extreme_logits_and_tables(wide):
    t = wl.random_tree(5, n_nodes=6, max_len=60, nq=7)
    s = Inputs(t, 600, 2, wide)
    for i, v in enumerate([math.inf, -math.inf, math.nan, 0.0, -0.0, 3e38, -3e38, 1e-40]):
        s.x[:, 37 * i:37 * i + 20] = v
    s.bias[0, ::7] = -math.inf
    s.bias[1, ::5] = np.finfo(np.float32).min
    s.bias[2, ::3] = math.nan
    s.bias_row[:4], s.mask_row[:4] = [0, 1, 2, -1], [3, 4, 0, -1]
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    for which in (dict(repetition=True), dict(bias=True, bias_row=True), dict(mask=True, mask_row=True), ALL):
        want, mag = s.want(**which)
        # what leaves fp32 (and bf16, by rounding) on the way is an infinity
        most = float(torch.finfo(s.x.dtype).max) * (1 + (2.0 ** -25 if wide else 2.0 ** -9))
        want = np.where(np.abs(want) >= most, np.copysign(np.inf, want), want)
        got = s.call(plan, row_of, pool, **which)
        near = np.isinf(want) & (mag < 1.01 * most) & (mag > 0.99 * most)
        keep = torch.from_numpy(~near)
        assert keep.float().mean() > 0.8
        close(got.cpu()[keep], want[~near], mag[~near])
    assert torch.isinf(got[0]).all() and (got[0] < 0).all()  # a mask that leaves nothing


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [False, True])
def test_the_repetition_penalty_is_a_quotient(wide):
    # two roundings of fp32, the reciprocal's and the product's, also where the reciprocal would leave fp32 or its normal numbers
    r = np.array([1.1, 1.3, 3.0, 0.7, 3e38, 1e-39, 2e-45, 2.0 ** 127, 1e-30], np.float32)
    t = wl.random_tree(6, n_nodes=9, max_len=200, nq=len(r))
    s = Inputs(t, 700, 8, wide)
    s.x[:, ::3] *= 2.0 ** -80
    s.x[:, 1::3] *= 2.0 ** 110
    s.x[:, 1::17] = 2.0 ** -126
    s.repetition = r
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    got = s.call(plan, row_of, pool, out_dtype=torch.float32, repetition=True).cpu().numpy()
    x = s.x.float().numpy()
    some = 0
    for j in range(t.nq):
        on = s.tokens[model.path(t, j)].astype(np.int64)
        on = np.bincount(on[(on >= 0) & (on % PROMPT < 700)] % PROMPT, minlength=700) > 0
        y = x[j].astype(np.float64)
        want = np.where(on, np.where(y > 0, y / float(r[j]), y * float(r[j])), y)
        # half a step each, 2^-24, and their product; below fp32's normal numbers half of their step, 2^-150
        out = np.abs(want) >= 2.0 ** 128 * (1 - 2.0 ** -24)
        assert (got[j][out] == np.copysign(np.inf, want[out])).all()
        off = np.abs(got[j][~out] - want[~out]) - (2.0 ** -23 * (1 + 2.0 ** -20) * np.abs(want[~out]) + 2.0 ** -150)
        assert (off <= 0).all(), (j, off.max())
        some += (on & (x[j] > 0)).sum()
    assert some > 500


@pytest.mark.gpu
def test_in_place_and_rows_apart():
    t = wl.random_tree(8, n_nodes=9, max_len=50, nq=6)
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    for wide in (True, False):
        s = Inputs(t, 1501, 3, wide)
        want = s.call(plan, row_of, pool, **ALL)
        args = {k: gpu(getattr(s, k)) for k in ALL}
        tokens = gpu(s.tokens)
        base = torch.full((6, 1700), 9.0, dtype=s.x.dtype, device=dev())
        x = base[:, 100:1601]
        x.copy_(s.x)
        assert torch.equal(binding.deft_adjust_logits(plan, x, tokens, **args), want)
        out = torch.full((6, 1503), 7.0, dtype=s.x.dtype, device=dev())
        assert torch.equal(binding.deft_adjust_logits(plan, x, tokens, out=out[:, 1:1502], **args), want)
        assert (out[:, 0] == 7).all() and (out[:, 1502] == 7).all() and torch.equal(x, s.x.to(dev()))
        assert binding.deft_adjust_logits(plan, x, tokens, out=x, **args) is x
        assert torch.equal(x, want) and (base[:, :100] == 9).all() and (base[:, 1601:] == 9).all()
        # one row of logits for every query, tables of one row
        one = s.x[:1].to(dev())
        same = {k: args[k] for k in ("repetition", "frequency", "presence")}
        a = binding.deft_adjust_logits(plan, one.expand(6, 1501), tokens, bias=args["bias"][1], mask=args["mask"][1], **same)
        b = binding.deft_adjust_logits(plan, one.repeat(6, 1), tokens, bias=args["bias"][1:2], mask=args["mask"][:, :][1:2], **same)
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_rows_behind_four_billion_elements():
    t = wl.random_tree(9, n_nodes=4, max_len=30, nq=5)
    s = Inputs(t, 1200, 4, False)
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    base = torch.empty((5, 1_100_000_000), dtype=torch.bfloat16, device=dev())
    x = base[:, -1200:]
    x.copy_(s.x)
    want = s.call(plan, row_of, pool, **ALL)
    assert torch.equal(s.call(plan, row_of, pool, x=x, **ALL), want)
    args = {k: gpu(getattr(s, k)) for k in ALL}
    binding.deft_adjust_logits(plan, s.x.to(dev()), gpu(s.tokens), out=base[:, 5:1205], **args)
    assert torch.equal(base[:, 5:1205], want)
    del base, x
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_gpu_refusals():
    t = wl.random_tree(8, n_nodes=9, max_len=50, nq=6)
    plan = plan_of(t)[0]
    s = Inputs(t, 100, 3, True)
    x, tokens = s.x.to(dev()), gpu(s.tokens)
    f = gpu(s.frequency)
    adjust = binding.deft_adjust_logits
    with pytest.raises(binding.DeftError) as e:
        adjust(plan, x, tokens, frequency=f)  # no image: it is not made here, that would choose how the attention is cut
    assert e.value.status == ENOTREADY
    plan.image(t.Hq, t.Hkv, dev())
    bias, mask, row = gpu(s.bias), gpu(s.mask), gpu(s.bias_row)
    bad = [
        lambda: adjust(plan, x.half()), lambda: adjust(plan, x[0]), lambda: adjust(plan, x.cpu()), lambda: adjust(plan, x[:5]), lambda: adjust(plan, x[:, :0]),
        lambda: adjust(plan, x[:, ::2]), lambda: adjust(plan, x, frequency=f), lambda: adjust(plan, x, tokens.long(), frequency=f), lambda: adjust(plan, x, tokens.cpu(), frequency=f),
        lambda: adjust(plan, x, tokens[:5], frequency=f), lambda: adjust(plan, x, tokens, frequency=f[:5]), lambda: adjust(plan, x, tokens, frequency=f.double()),
        lambda: adjust(plan, x, tokens, presence=f.cpu()), lambda: adjust(plan, x, tokens, repetition=f[None]), lambda: adjust(plan, x, bias=bias[:, :99]),
        lambda: adjust(plan, x, bias=bias.double()), lambda: adjust(plan, x, bias=bias[:0]), lambda: adjust(plan, x, bias_row=row), lambda: adjust(plan, x, mask_row=row),
        lambda: adjust(plan, x, bias=bias, bias_row=row.long()), lambda: adjust(plan, x, mask=mask, mask_row=row[:3]), lambda: adjust(plan, x, mask=mask[:, :3]),
        lambda: adjust(plan, x, mask=mask.long()), lambda: adjust(plan, x, mask=mask.bool()), lambda: adjust(plan, x, out=x[:, :50]), lambda: adjust(plan, x, out=x.to(torch.bfloat16)),
        lambda: adjust(plan, x, out_dtype=torch.bfloat16), lambda: adjust(plan, x, out=x.t().contiguous().t()), lambda: adjust(plan, x[:1].expand(6, 100), out=x),
        lambda: adjust(plan, x.view(-1)[:594].view(6, 99), out=x.view(-1)[1:595].view(6, 99)), lambda: adjust(plan, x, bias=bias[:1].expand(3, 100)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.DeftError):
            call()
            pytest.fail(f"call {i}")
    empty = binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, [], t.ntok)
    assert adjust(empty, x[:0], tokens, frequency=f[:0]).shape == (0, 100)


@pytest.mark.gpu
def test_tables_of_no_and_of_three_dimensions_are_refused():
    t = wl.random_tree(8, n_nodes=9, max_len=50, nq=6)
    plan, x = plan_of(t)[0], torch.zeros((6, 1), device=dev())
    for shape in ((), (1, 1, 1)):
        for bad in (dict(bias=torch.zeros(shape, device=dev())), dict(mask=torch.zeros(shape, dtype=torch.int32, device=dev()))):
            with pytest.raises(binding.DeftError, match="must be a"):
                binding.deft_adjust_logits(plan, x, **bad)


@pytest.mark.gpu
def test_images_are_those_of_the_attention():
    t = wl.random_tree(8, n_nodes=9, max_len=50, nq=6, Hq=8, Hkv=2)
    s = Inputs(t, 300, 3, True)
    plan, row_of, pool = plan_of(t)
    Q, K, V = (x.to(dev()) for x in wl.make_qkv(t))
    binding.deft_tree_attn_decode(plan, Q, K, V)
    images = dict(plan._images.of)
    got = s.call(plan, row_of, pool, **ALL)
    assert plan._images.of.keys() == images.keys()
    close(got, *s.want(**ALL))


@pytest.mark.gpu
def test_captured_and_replayed():
    t = wl.random_tree(18, n_nodes=20, max_len=50, nq=30)
    s = Inputs(t, 3001, 3, True)
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    x, tokens, args = s.x.to(dev()), gpu(s.tokens), {k: gpu(getattr(s, k)) for k in ALL}
    binding.deft_adjust_logits(plan, x, tokens, **args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.deft_adjust_logits(plan, x, tokens, **args)
        rest = binding.deft_adjust_logits(plan, x, tokens, repetition=args["repetition"])
    for i in range(4):
        n = Inputs(t, 3001, 20 + i, True)
        x.copy_(n.x)
        tokens.copy_(gpu(n.tokens))
        for k in ALL:
            args[k].copy_(gpu(getattr(n, k)))
        graph.replay()
        a, b = got.clone(), rest.clone()
        assert torch.equal(a.nan_to_num(), binding.deft_adjust_logits(plan, x, tokens, **args).nan_to_num())
        assert torch.equal(b, binding.deft_adjust_logits(plan, x, tokens, repetition=args["repetition"]))
        close(a, *n.want(**ALL))
        torch.cuda.synchronize()
    # a plan whose image is first sent inside a graph
    plan, _, _ = plan_of(t)
    Q, K, V = (z.to(dev()) for z in wl.make_qkv(t))
    binding.deft_tree_attn_decode(plan_of(t)[0], Q, K, V)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.deft_tree_attn_decode(plan, Q, K, V)
        got = binding.deft_adjust_logits(plan, x, tokens, **args)
    for _ in range(2):
        graph.replay()
        close(got, *n.want(**ALL))
        close(binding.deft_adjust_logits(plan, x, tokens, **args), *n.want(**ALL))


@pytest.mark.gpu
def test_two_streams_at_once():
    t = wl.config5_longcontext(root=3000, branches=16, lo=10, hi=300)
    s = Inputs(t, 20000, 3, True)
    plan, row_of, pool = plan_of(t)
    plan.image(t.Hq, t.Hkv, dev())
    x, tokens, args = s.x.to(dev()), gpu(s.tokens), {k: gpu(getattr(s, k)) for k in ALL}
    want = binding.deft_adjust_logits(plan, x, tokens, **args)
    other = binding.deft_adjust_logits(plan, x, tokens, presence=args["presence"])
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for side in sides:
            side.wait_stream(torch.cuda.current_stream())
            got.append(binding.deft_adjust_logits(plan, x, tokens, stream=side, **args))
            got.append(binding.deft_adjust_logits(plan, x, tokens, presence=args["presence"], stream=side.cuda_stream))
        for side in sides:
            torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(got, [want, other] * 2))


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [False, True])
def test_sorted_tokens_captured_and_replayed(counts):
    # two launches and a workspace of the graph's own, taken while it is captured; tokens, logits and tables change between replays,
    # and eager calls with other tokens, in workspaces of theirs, stand in between
    t, vocab = wl.config5_longcontext(root=3000, branches=16, lo=10, hi=300), 20000
    which = {k: v for k, v in ALL.items() if counts or k != "frequency"}
    s = Inputs(t, vocab, 3, True)
    plan, row_of, pool = plan_of(t)
    assert binding.load_library().deft_logits_workspace_bytes(plan.handle, vocab) > 0
    plan.image(t.Hq, t.Hkv, dev())
    x, tokens, args = s.x.to(dev()), gpu(s.tokens), {k: gpu(getattr(s, k)) for k in which}
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            results.append((binding.deft_adjust_logits(plan, x, tokens, **args), binding.deft_adjust_logits(plan, x, tokens, presence=args["presence"])))
    spaces = [w[0] for k, w in plan._workspaces.items() if k[0] == "logits"]
    assert len(spaces) == len(set(spaces)) == 2
    other_tokens = gpu(Inputs(t, vocab, 99, True).tokens)
    side = torch.cuda.Stream()
    for i in range(4):
        n = Inputs(t, vocab, 20 + i, True)
        x.copy_(n.x)
        tokens.copy_(gpu(n.tokens))
        for k in which:
            args[k].copy_(gpu(getattr(n, k)))
        torch.cuda.synchronize()
        for graph, (a, b) in zip(graphs, results):
            graph.replay()
            # at the same time, on another stream
            with torch.cuda.stream(side):
                between = binding.deft_adjust_logits(plan, x, other_tokens, presence=args["presence"])
            eager = binding.deft_adjust_logits(plan, x, tokens, **args)
            assert torch.equal(a.nan_to_num(), eager.nan_to_num())
            assert torch.equal(b, binding.deft_adjust_logits(plan, x, tokens, presence=args["presence"]))
            side.synchronize()
            assert torch.equal(between, binding.deft_adjust_logits(plan, x, other_tokens, presence=args["presence"]))
        if i in (0, 3):
            close(results[0][0], *n.want(**which))
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_two_host_threads():
    # each on a stream of its own, with the same plan and lists: logits of both forms, and heads
    import threading
    from concurrent.futures import ThreadPoolExecutor

    big, small = wl.config5_longcontext(root=3000, branches=16, lo=10, hi=300), wl.random_tree(18, n_nodes=20, max_len=50, nq=30)
    room = binding.load_library().deft_logits_workspace_bytes
    work = []
    for t, vocab in ((big, 20000), (small, 3001)):
        s = Inputs(t, vocab, 3, True)
        plan = plan_of(t)[0]
        assert (room(plan.handle, vocab) > 0) == (t is big)
        plan.image(t.Hq, t.Hkv, dev())
        work.append((plan, s.x.to(dev()), gpu(s.tokens), {k: gpu(getattr(s, k)) for k in ALL}))
    want = [binding.deft_adjust_logits(p, x, tokens, **a) for p, x, tokens, a in work]
    n, Hq, Hkv, d = 500, 8, 2, 128
    heads = torch.randn((n, Hq + 2 * Hkv, d), device=dev()).to(torch.bfloat16)
    rope, p = binding.deft_rope(d), torch.arange(n, dtype=torch.int32, device=dev())
    rows = binding.deft_kv_rows(np.random.default_rng(1).permutation(n), n, 1)

    def store(pools):
        return binding.deft_qkv_store(rows, heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], pools, p, rope)

    def pools():
        return [torch.zeros((n, Hkv, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]

    kept = pools()
    q = store(kept)
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def one():
        with torch.cuda.stream(torch.cuda.Stream()):
            mine = pools()
            start.wait(30)
            for _ in range(30):
                got = [binding.deft_adjust_logits(p, x, tokens, **a) for p, x, tokens, a in work]
                mine_q = store(mine)
            torch.cuda.current_stream().synchronize()
            return all(torch.equal(a.nan_to_num(), b.nan_to_num()) for a, b in zip(got, want)) and torch.equal(mine_q, q) and all(torch.equal(a, b) for a, b in zip(mine, kept))

    with ThreadPoolExecutor(2) as pool:
        done = [pool.submit(one) for _ in range(2)]
        assert [f.result(60) for f in done] == [True, True]

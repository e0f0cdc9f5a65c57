"""Calls on another stream than torch's current one: what they allocate, and what two streams or two graphs may do at once."""

import numpy as np
import pytest
import torch

from paper_2404_00242_amd import binding, workloads as wl

pytestmark = pytest.mark.gpu


def dev():
    return torch.device("cuda:0")


def star(prefix, branches, length, Hq, Hkv, d):
    return wl._finish("star", [prefix] + [length] * branches, [-1] + [0] * branches, list(range(1, branches + 1)), Hq, Hkv, d, 5)


def some_milliseconds():
    """Work for the current stream, about 20 ms of it."""
    x = torch.ones((8192, 8192), dtype=torch.bfloat16, device=dev())
    for _ in range(20):
        torch.mm(x, x)


class Calls:
    """Attention over both caches and rows read back, on one tree: what they give as a dict of tensors."""

    def __init__(self, chunk=128, nq=9):
        self.t = t = star(700, nq, 40, 8, 2, 128)
        self.q, self.k, self.v = (x.to(dev()) for x in wl.make_qkv(t))
        self.cache = binding.alloc_kv_cache_q8(t.ntok, 2, 128, 16, dev())
        self.rows = binding.deft_kv_rows(np.arange(t.ntok), t.ntok, 16)
        binding.deft_kv_store_q8(self.rows, self.k, self.v, self.cache)
        self.plan = self.new_plan(chunk)

    def new_plan(self, chunk=128):
        t = self.t
        return binding.deft_plan(t.node_tok_begin, t.node_tok_len, t.node_parent, t.query_node, t.ntok, chunk)

    def call(self, name, stream=None):
        if name == "bf16":
            return [binding.deft_tree_attn_decode(self.plan, self.q, self.k, self.v, stream=stream)]
        if name == "q8":
            return [binding.deft_tree_attn_decode_q8(self.plan, self.q, self.cache, stream=stream)]
        if name == "q8_f32":
            return [binding.deft_tree_attn_decode_q8(self.plan, self.q, self.cache, out_dtype=torch.float32, stream=stream)]
        return list(binding.deft_kv_load_q8(self.rows, self.cache, stream=stream))


NAMES = ["bf16", "q8", "q8_f32", "load"]


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_a_result_takes_no_memory_that_the_current_stream_still_reads(name, as_handle):
    c = Calls()
    want = c.call(name)
    other = torch.cuda.Stream()
    c.call(name, other)  # images, workspaces
    torch.cuda.synchronize()
    for _ in range(3):
        held = [torch.full_like(x, 3.0) for x in want]
        read = [torch.zeros_like(x) for x in want]
        torch.cuda.synchronize()
        some_milliseconds()
        for x, y in zip(held, read):
            y.copy_(x)
        x = None
        del held  # the allocator has these blocks back, the copies have not run
        got = c.call(name, other.cuda_stream if as_handle else other)
        torch.cuda.synchronize()
        assert all(bool((y == 3).all()) for y in read)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_a_result_that_is_dropped_early_is_not_the_current_streams_to_reuse(name):
    c = Calls()
    want = c.call(name)
    other = torch.cuda.Stream()
    c.call(name, other)
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(other):
            some_milliseconds()
        c.call(name, other)  # dropped before it was written
        new = [torch.full_like(x, 5.0) for x in want]
        torch.cuda.synchronize()
        assert all(bool((x == 5).all()) for x in new)


@pytest.mark.parametrize("name", NAMES)
def test_a_result_is_kept_while_the_current_stream_reads_it(name):
    c = Calls()
    want = c.call(name)
    other = torch.cuda.Stream()
    c.call(name, other)
    torch.cuda.synchronize()
    for _ in range(3):
        got = c.call(name, other)
        torch.cuda.current_stream().wait_stream(other)
        some_milliseconds()
        read = [x.clone() for x in got]
        x = None
        del got
        with torch.cuda.stream(other):  # what it would give these blocks to
            new = [torch.full_like(x, 7.0) for x in want]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(read, want))
        assert all(bool((x == 7).all()) for x in new)


@pytest.mark.parametrize("name", ["bf16", "q8"])
def test_an_output_that_is_given_stays_the_callers(name):
    c = Calls()
    want = c.call(name)[0]
    out, other = torch.zeros_like(want), torch.cuda.Stream()
    torch.cuda.synchronize()
    if name == "bf16":
        got = binding.deft_tree_attn_decode(c.plan, c.q, c.k, c.v, out=out, stream=other)
    else:
        got = binding.deft_tree_attn_decode_q8(c.plan, c.q, c.cache, out=out, stream=other)
    torch.cuda.synchronize()
    assert got is out and torch.equal(out, want)


# ---- workspaces ----

@pytest.mark.parametrize("name", ["bf16", "q8_f32"])
def test_calls_of_several_streams_at_once_have_a_workspace_each(name):
    c = Calls(chunk=32)
    want = c.call(name)[0]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = [c.call(name, st)[0] for _ in range(20) for st in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)
    spaces = [c.plan.workspace(8, 2, 128, dev(), st) for st in streams] + [c.plan.workspace(8, 2, 128, dev())]
    assert len({x.data_ptr() for x in spaces}) == 4 and spaces[3] is c.plan.workspace(8, 2, 128, dev())


@pytest.mark.parametrize("name", ["bf16", "q8"])
def test_two_graphs_of_one_stream_and_eager_calls_at_once(name):
    c = Calls(chunk=32)
    side, others = torch.cuda.Stream(), [torch.cuda.Stream(), torch.cuda.Stream()]
    with torch.cuda.stream(side):
        c.call(name)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append([c.call(name)[0] for _ in range(12)])
    for step in range(3):
        c.q.normal_()
        want = c.call(name)[0]
        torch.cuda.synchronize()
        for g, st in zip(graphs, others):
            with torch.cuda.stream(st):
                g.replay()
        with torch.cuda.stream(side):
            eager = [c.call(name)[0] for _ in range(12)]
        torch.cuda.synchronize()
        for o in (*outs, eager):
            # a captured call takes two launches and an eager one may take one, which sums in another order: a bf16 result may be the
            # next number, 2^-7 of it; near zero 2 n 2^-24 of the largest |V|, 5, with n < 50 partial results
            for x in o:
                assert bool(((x.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2.0 ** -14).all())
        assert all(torch.equal(x, outs[0][0]) for o in outs for x in o)


# ---- images ----

@pytest.mark.parametrize("name", NAMES)
def test_an_image_that_a_graph_uploads_is_not_used_before_its_replay(name):
    # first use under capture; then eager calls on the very stream, before any replay; then replays of what two captures made
    c = Calls()
    want = c.call(name)
    side = torch.cuda.Stream()
    c.plan, c.rows = c.new_plan(), binding.deft_kv_rows(np.arange(c.t.ntok), c.t.ntok, 16)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            outs.append([c.call(name) for _ in range(3)])
    with torch.cuda.stream(side):
        eager = c.call(name)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, want))
    for _ in range(4):
        for o in outs:
            for x in o:
                for y in x:
                    y.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        with torch.cuda.stream(side):
            eager = c.call(name)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want))
        for o in outs:
            for x in o:
                for a, b in zip(x, want):  # (two launches and one: as above)
                    assert bool(((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 2.0 ** -14).all())


def test_a_capture_on_two_streams_uploads_its_image_once():
    c = Calls()
    want = c.call("q8_f32")[0]
    side, fork = torch.cuda.Stream(), torch.cuda.Stream()
    c.plan = c.new_plan()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        a = c.call("q8_f32")[0]
        fork.wait_stream(side)
        with torch.cuda.stream(fork):
            b = c.call("q8_f32")[0]
        side.wait_stream(fork)
    assert len(c.plan._images.of) == 1 and len(c.plan._workspaces) == 2
    for _ in range(4):
        a.zero_()
        b.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        # sums of at most 50 fp32 terms in another order where the eager call took one launch
        assert float((a - want).abs().max()) <= 2 * 50 * 2.0 ** -24 * 8 and torch.equal(a, b)


@pytest.mark.parametrize("name", NAMES)
def test_a_plan_or_list_that_is_dropped_leaves_its_memory_to_streams_that_still_use_it(name):
    c = Calls()
    want = c.call(name)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        c.plan, c.rows = c.new_plan(), binding.deft_kv_rows(np.arange(c.t.ntok), c.t.ntok, 16)
        c.call(name)  # uploads on the current stream
        torch.cuda.synchronize()
        sizes = [x.tensor.numel() for y in (c.plan, c.rows) for x in y._images.of.values()]
        with torch.cuda.stream(other):
            some_milliseconds()
        got = c.call(name, other)
        c.plan = c.rows = None
        new = [torch.full((n,), 255, dtype=torch.uint8, device=dev()) for n in sizes for _ in range(4)]  # all bits, on the current stream
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(bool((x == 255).all()) for x in new)


@pytest.mark.parametrize("name", NAMES)
def test_a_captured_call_on_a_stream_that_is_named(name):
    c = Calls()
    want = c.call(name)
    side, fork = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        fork.wait_stream(side)
        got = [c.call(name, fork) for _ in range(3)]
        c.call(name, fork)  # dropped
        after = c.call(name, fork)
        side.wait_stream(fork)
        copies = [[x.clone() for x in y] for y in (*got, after)]
    for _ in range(4):
        for y in copies:
            for x in y:
                x.zero_()
        some_milliseconds()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for y in copies:
            for a, b in zip(y, want):  # (two launches and one: as above)
                assert bool(((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 2.0 ** -14).all())


def test_a_call_leaves_the_current_stream_as_it_was():
    c = Calls()
    other, side = torch.cuda.Stream(), torch.cuda.Stream()
    for here in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(here):
            for name in NAMES:
                c.call(name, other)
                assert torch.cuda.current_stream() == here and torch.cuda.current_device() == 0
    torch.cuda.synchronize()


def test_every_capture_has_a_number_of_its_own():
    c, lib = Calls(), binding.load_library()
    side, fork = torch.cuda.Stream(), torch.cuda.Stream()
    seen = []
    for _ in range(3):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            seen.append(lib.deft_capture_id(side.cuda_stream))
            assert lib.deft_capture_id(fork.cuda_stream) == 0
            fork.wait_stream(side)
            with torch.cuda.stream(fork):
                c.call("q8")
            assert lib.deft_capture_id(fork.cuda_stream) == seen[-1]
            side.wait_stream(fork)
        assert lib.deft_capture_id(side.cuda_stream) == 0
    assert len(set(seen)) == 3 and 0 not in seen
    assert {k[-1] for k in c.plan._workspaces} == set(seen) and len(c.plan._workspaces) == 3

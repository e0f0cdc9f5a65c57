"""The calls on an 8-bit KV cache whose speed is watched, each beside its plain form in elementary torch operations.

The cache holds K and V in e4m3 with one power of two as the scale of each (block of rows, KV head).  "attention" is
tree-attention decode over it, "store" quantises new K/V rows into it (a prompt, or a token for every leaf of a tree) and
reads the whole pool back, "load" reads rows back as bf16, "copy" copies pages inside the pools of several layers (forks of
branches, compaction).  `own` chooses between the plain forms and the framework's entry points.
"""

import math

import numpy as np
import torch

own = False

E_MIN, E_MAX = 10, 246  # scale bytes (2^(byte - 127)) whose products with e4m3 values are normal bf16 numbers


# ---- cases ----

def _attention(name, tree, a, b, lo, hi, Hq, Hkv, d, block, page=0):
    """tree: shape with its sizes a (prefix or root tokens), b (width or depth), lo..hi (branch lengths); page: rows of a
    page, handed out in random order (0: contiguous cache); block: rows that share a scale."""
    c = dict(kind="attention", tree=tree, a=a, b=b, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, block=block, page=page)
    return dict(c, name=name) if name else c


def _store(name, n, append, Hkv, d, block, page):
    """append: n leaves get one token each behind what their page holds; otherwise a prompt of n tokens goes into pages in
    random order.  K and V are slices of a fused projection's output."""
    c = dict(kind="store", n=n, append=append, Hkv=Hkv, d=d, block=block, page=page)
    return dict(c, name=name) if name else c


def _load(name, n, Hkv, d, block, page):
    c = dict(kind="load", n=n, Hkv=Hkv, d=d, block=block, page=page)
    return dict(c, name=name) if name else c


def _copy(name, pages, moves, layers, Hkv, d, page, block, compact):
    """compact: `moves` pages change places among themselves; otherwise each goes to a free page.  block: 0 for bf16 pools,
    else 8-bit ones, whose values are read back."""
    c = dict(kind="copy", pages=pages, moves=moves, layers=layers, Hkv=Hkv, d=d, page=page, block=block, compact=compact)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the benchmark's smallest tree: launch latency and the host path
        _attention("attention_tiny", "fewshot", 256, 4, 32, 32, 4, 4, 64, 32),
        # one sequence, one query: where every tree begins; a scale for each token
        _attention("attention_single", "single", 8191, 1, 0, 0, 32, 8, 128, 1),
        # few-shot prompting with multi-head attention, the benchmark's second workload: reading the cache is all there is
        _attention("attention_fewshot_mha", "fewshot", 4000, 20, 256, 256, 32, 32, 128, 32),
        # multi-step reasoning, 256 leaves, over 64-row pages: the benchmark's fourth workload as a server stores it
        _attention("attention_reasoning_paged", "reasoning", 1000, 4, 128, 512, 32, 8, 128, 32, page=64),
        # a very long shared prefix with ragged branches: the benchmark's fifth workload and the largest call
        _attention("attention_longcontext", "longcontext", 32768, 64, 64, 2048, 32, 8, 128, 64),
        # a decode iteration's new tokens, one for each of 64 leaves, into partly filled 16-row pages
        _store("store_append", 64, True, 8, 128, 16, 16),
        # a long prompt, multi-head
        _store("store_prompt", 8192, False, 32, 128, 32, 64),
        # odd sizes: token-level pool, head count that divides nothing, short heads
        _store("store_tokens", 1237, False, 5, 64, 1, 1),
        # a branch of 500 tokens read back for another kernel
        _load("load_branch", 500, 8, 128, 32, 64),
        # a speculative prefix read back for a second model's prefill
        _load("load_prefix", 12345, 8, 128, 16, 16),
        # beams of a tree fork: 40 last pages are copied in every one of 32 layers
        _copy("copy_fork", 600, 40, 32, 8, 128, 16, 0, False),
        # a pool whose pages lie in any order is put in order, 8-bit, in 8 layers
        _copy("copy_compact", 160, 150, 8, 8, 128, 64, 32, True),
    ]


def draw(rng):
    """A case of the same ranges in another combination and size."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["kind"], {"bytes": 0.0, "flops": 0.0})
        most[c["kind"]] = {k: max(m[k], w[k]) for k in m}
    while True:
        kind = rng.choice(["attention", "attention", "attention", "attention", "store", "store", "load", "copy"])
        block = rng.choice([1, 2, 4, 8, 16, 16, 32, 32, 32, 64])
        Hq, Hkv = rng.choice([(32, 32), (32, 8), (32, 8), (64, 8), (28, 4), (16, 16), (12, 2), (8, 8), (5, 5), (4, 4), (6, 1)])
        d = rng.choice([128, 128, 128, 64])
        page = block * rng.choice([1, 2, 4])
        if kind == "attention":
            tree = rng.choice(["fewshot", "speculative", "reasoning", "longcontext", "single", "forest"])
            a, b, lo = log(100, 8000), log(2, 50), log(1, 256)
            if tree == "reasoning":
                a, b, lo = log(100, 2000), rng.randint(2, 4), log(16, 128)
            elif tree == "longcontext":
                a, b, lo = log(8192, 32768), log(4, 64), log(16, 64)
            elif tree == "single":
                a, b = log(384, 32768), 1
            elif tree == "forest":
                b, lo = log(2, 32), log(64, 512)
            hi = rng.randint(lo, 4 * lo + 16)
            if tree in ("speculative", "single"):
                lo = hi = int(tree == "speculative")
            c = _attention(None, tree, a, b, lo, hi, Hq, Hkv, d, block, rng.choice([0, page]))
        elif kind == "store":
            append = rng.random() < 0.5
            c = _store(None, log(1, 300) if append else log(1, 8192), append, Hkv, d, block, page)
        elif kind == "load":
            c = _load(None, log(1, 16384), Hkv, d, block, page)
        else:
            pages = log(8, 1000)
            moves = rng.randint(1, pages // 2)
            c = _copy(None, pages, moves, log(1, 32), Hkv, d, page, rng.choice([0, block]), rng.random() < 0.5)
            if c["block"] and c["layers"] > 16:
                continue
        w = work(c)
        if all(w[k] <= most[kind][k] for k in w):
            return c


# ---- trees and storage: what the serving program's tables say ----

def _tree(case):
    """(node lengths, parents, query nodes); ragged lengths depend on the case's sizes alone."""
    tree, a, b, lo, hi = (case[k] for k in ("tree", "a", "b", "lo", "hi"))
    rng = np.random.default_rng([a, b, lo, hi])
    if tree == "single":
        return [a], [-1], [0]
    if tree == "forest":
        return [int(x) for x in rng.integers(lo, hi + 1, b)], [-1] * b, list(range(b))
    parents, level = [-1], [0]
    if tree == "reasoning":  # four children to a node, b levels, queries at the leaves
        for _ in range(b):
            first = len(parents)
            parents += [u for u in level for _ in range(4)]
            level = list(range(first, len(parents)))
        queries = level
    elif tree == "speculative":  # b one-token nodes below the prefix, up to ten to a node, each with a query
        parents += [max(0, (i - 1) // 10) for i in range(1, b + 1)]
        queries = list(range(1, b + 1))
    else:  # branches under a prompt; a long context's first few have branches of their own
        parents += [0] * b
        if tree == "longcontext":
            parents += [1 + i // 8 for i in range(8 * min(8, b // 8))]
        inner = set(parents)
        queries = [u for u in range(1, len(parents)) if u not in inner]
    lens = [a] + [int(x) for x in rng.integers(lo, hi + 1, len(parents) - 1)]
    if tree == "longcontext":
        lens[1 + b:] = [128] * (len(lens) - 1 - b)
    return lens, parents, queries


def _paths(parents, queries):
    up = [[int(u)] for u in queries]
    for p in up:
        while parents[p[-1]] >= 0:
            p.append(parents[p[-1]])
    return up


def _pages(case, lens):
    """(node_page_ptr, page_ids, pool pages): pages in random order, three to spare."""
    need = [-(-n // case["page"]) for n in lens]
    ptr = np.concatenate([[0], np.cumsum(need)])
    room = int(ptr[-1]) + 3
    return ptr, np.random.default_rng([len(lens), room, case["page"]]).permutation(room)[: int(ptr[-1])], room


def _layout(case, lens):
    """Storage tables of the nodes, rows of the pool, and the pool row of every token, node by node."""
    if not case["page"]:
        begins = np.concatenate([[0], np.cumsum(lens)[:-1]])
        return (begins,), int(sum(lens)), np.arange(sum(lens))
    ptr, ids, room = _pages(case, lens)
    t = np.concatenate([np.arange(n) for n in lens])
    u = np.repeat(np.arange(len(lens)), lens)
    return (ptr, ids, room), room * case["page"], ids[ptr[u] + t // case["page"]] * case["page"] + t % case["page"]


def _row_tables(case):
    """Of a store or load: pool rows, rows in use before the call (per page), and the rows that the call names."""
    P = case["page"]
    if case["kind"] == "store" and case["append"]:
        room = case["n"] + 3
        rng = np.random.default_rng([case["n"], P, case["block"]])
        fill = rng.integers(0, P, case["n"])  # tokens that a leaf's page holds
        return room * P, rng.permutation(room)[: case["n"]] * P + fill
    _, rows, at = _layout(case, [case["n"]])
    return rows, at


# ---- the cache's plain form ----

def _scale_byte(amax):
    """Of the smallest power of two that brings the largest magnitude to e4m3's largest value, 448, or below."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.875, x - 9, x - 8) + 127
    return torch.where(amax > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _power(byte):
    return torch.ldexp(torch.ones((), device=byte.device, dtype=torch.float32), byte.to(torch.int32) - 127)


def _to_e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _quantise(x, bytes_, rows, block, low):
    """The rows x [n, Hkv, d] into pool x8 with scales s [blocks, Hkv] (pair `bytes_`).  low: [blocks] lowest position in its
    block that is written, `block` where none is.  A block's rows in front of that are kept, and take part in its scale."""
    x8, s = bytes_
    x = x.float()
    blk = rows // block
    old = s.view(torch.uint8).to(torch.int32)
    new = torch.zeros_like(old).index_reduce_(0, blk, _scale_byte(x.abs().amax(-1)), "amax")
    hit = (low < block)[:, None]
    new = torch.where(hit, torch.where((low > 0)[:, None], torch.maximum(old, new), new), old)
    touched = low.repeat_interleave(block)[: x8.shape[0]] < block
    pos = torch.arange(x8.shape[0], device=x8.device)
    keep = (touched & (pos % block < low[pos // block])).nonzero()[:, 0]
    k8 = x8[keep].float() * _power(old - new + 127)[keep // block][..., None]
    x8[keep] = _to_e4m3(k8)
    x8[rows] = _to_e4m3(x * _power(254 - new)[blk][..., None])
    s.view(torch.uint8).copy_(new.to(torch.uint8))


def _values(x8, s, rows, block):
    return x8[rows].float() * _power(s.view(torch.uint8))[rows // block][..., None]


def _lowest(rows, block, blocks):
    return torch.full((blocks,), block, device=rows.device).index_reduce_(0, rows // block, rows % block, "amin")


def _empty(rows, Hkv, d, block, g):
    """A pool as an allocator leaves it: bytes of earlier contents (numbers, no NaN), scales of earlier blocks."""
    dev = g.device
    x8 = torch.randint(0, 0x7f, (rows, Hkv, d), generator=g, device=dev, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.randint(118, 126, (-(-rows // block), Hkv), generator=g, device=dev, dtype=torch.uint8)
    return x8, s.view(torch.float8_e8m0fnu)


def _kv(n, Hkv, d, g):
    """K and V of n tokens as slices of a fused projection's output.  Keys have loud and quiet channels, tokens differ in
    magnitude, as those of trained models do."""
    x = torch.randn((n, 3, Hkv, d), generator=g, device=g.device)
    x[:, 1] *= torch.exp(0.4 * torch.randn((Hkv, d), generator=g, device=g.device))
    x[:, 2] *= torch.exp(0.4 * torch.randn((n, Hkv, 1), generator=g, device=g.device))
    x = x.to(torch.bfloat16)
    return x[:, 1], x[:, 2]


# ---- state ----

def _cache(s):
    from paper_2404_00242_amd import binding

    return binding.CacheQ8(s["k8"], s["v8"], s["ks"], s["vs"], s["case"]["block"])


def _plan(case, where, rows):
    """The attention call's plan and its device image, made once for all layers and kept."""
    from paper_2404_00242_amd import binding

    lens, parents, queries = _tree(case)
    flags = binding.DEFT_SPLIT_BALANCED | binding.rows_per_query(case["Hq"] // case["Hkv"])
    chunk = binding.deft_suggest_chunk_size(lens, parents, queries, case["Hq"], case["Hkv"], flags)
    if case["page"]:
        plan = binding.deft_plan_paged(where[0], where[1], case["page"], where[2], lens, parents, queries, chunk, flags)
    else:
        plan = binding.deft_plan(where[0], lens, parents, queries, rows, chunk, flags)
    plan.image(case["Hq"], case["Hkv"], torch.device("cuda", torch.cuda.current_device()))
    return plan


def _row_list(rows, pool_rows, block):
    from paper_2404_00242_amd import binding

    rows = binding.deft_kv_rows(rows, pool_rows, block)
    rows.image(torch.device("cuda", torch.cuda.current_device()))
    return rows


def _page_list(src, dst, pages):
    from paper_2404_00242_amd import binding

    copies = binding.deft_kv_copies(src, dst, pages)
    copies.image(torch.device("cuda", torch.cuda.current_device()))
    return copies


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev).manual_seed(int(seed))
    kind, Hkv, d, block = case["kind"], case["Hkv"], case["d"], case["block"]
    s = {"case": case}
    if kind == "attention":
        lens, parents, queries = _tree(case)
        where, pool, at = _layout(case, lens)
        node = torch.from_numpy(np.repeat(np.arange(len(lens)), lens)).to(dev)
        on_path = torch.zeros((len(queries), len(lens)), dtype=torch.bool)
        for j, path in enumerate(_paths(parents, queries)):
            on_path[j, path] = True
        s["sees"] = on_path.to(dev)[:, node].contiguous()  # [queries, tokens]
        s["rows"] = torch.from_numpy(at).to(dev)
        s["q"] = torch.randn((len(queries), case["Hq"], d), generator=g, device=dev).to(torch.bfloat16)
        if own:
            s["plan"] = _plan(case, where, pool)
    elif kind in ("store", "load"):
        pool, at = _row_tables(case)
        s["rows"] = torch.from_numpy(at).to(dev)
        s["all"] = s["rows"] if kind == "load" else torch.arange(pool, device=dev)
        if own:
            s["named"] = _row_list(at, pool, block)
            s["named_all"] = s["named"] if kind == "load" else _row_list(np.arange(pool), pool, block)
        if kind == "store":
            s["k"], s["v"] = _kv(case["n"], Hkv, d, g)
    else:
        rng = np.random.default_rng([case["pages"], case["moves"], case["layers"], int(seed)])
        order = rng.permutation(case["pages"])
        n = case["moves"]
        src = order[:n]
        dst = rng.permutation(src) if case["compact"] else order[case["pages"] - n:]
        s["src"], s["dst"] = torch.from_numpy(src).to(dev), torch.from_numpy(dst).to(dev)
        pool = case["pages"] * case["page"]
        if own:
            s["copies"] = _page_list(src, dst, case["pages"])
        if not block:
            s["pools"] = [torch.randn((pool, Hkv, d), generator=g, device=dev).to(torch.bfloat16) for _ in range(2 * case["layers"])]
            return s
        s["pools"] = [x for _ in range(2 * case["layers"]) for x in _empty(pool, Hkv, d, block, g)]
        s["all"] = torch.arange(pool, device=dev)
        if own:
            s["named_all"] = _row_list(np.arange(pool), pool, block)
        return s
    s["k8"], s["ks"] = _empty(pool, Hkv, d, block, g)
    s["v8"], s["vs"] = _empty(pool, Hkv, d, block, g)
    if kind != "store" or case["append"]:  # every row of the pool holds a token of some sequence
        every = torch.arange(pool, device=dev)
        low = torch.zeros((s["ks"].shape[0],), device=dev, dtype=torch.int64)
        k, v = _kv(pool, Hkv, d, g)
        _quantise(k, (s["k8"], s["ks"]), every, block, low)
        _quantise(v, (s["v8"], s["vs"]), every, block, low)
    return s


# ---- the operators ----

def _plain_attention(s):
    case = s["case"]
    q, block, Hkv, d = s["q"], case["block"], case["Hkv"], case["d"]
    nq, G = q.shape[0], case["Hq"] // case["Hkv"]
    k = _values(s["k8"], s["ks"], s["rows"], block).permute(1, 2, 0).contiguous()  # [Hkv, d, tokens]
    v = _values(s["v8"], s["vs"], s["rows"], block).transpose(0, 1).contiguous()
    q = q.float().view(nq, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, nq * G, d)
    x = torch.matmul(q, k) * (1.0 / math.sqrt(d))
    x = x.view(Hkv, nq, G, -1).masked_fill_(~s["sees"][None, :, None, :], -math.inf).view(Hkv, nq * G, -1)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    o = torch.matmul(x, v) / x.sum(-1, keepdim=True)
    return o.view(Hkv, nq, G, d).permute(1, 0, 2, 3).reshape(nq, case["Hq"], d).to(torch.bfloat16)


def _plain_store(s):
    case = s["case"]
    low = _lowest(s["rows"], case["block"], s["ks"].shape[0])
    _quantise(s["k"], (s["k8"], s["ks"]), s["rows"], case["block"], low)
    _quantise(s["v"], (s["v8"], s["vs"]), s["rows"], case["block"], low)


def _plain_load(s):
    block = s["case"]["block"]
    return [_values(x8, sc, s["all"], block).to(torch.bfloat16) for x8, sc in ((s["k8"], s["ks"]), (s["v8"], s["vs"]))]


def _plain_copy(s):
    pages = s["case"]["pages"]
    paged = [x.view(torch.uint8).view(pages, -1) for x in s["pools"]]
    for x in paged:
        x[s["dst"]] = x[s["src"]]


def _by_layer(s):
    """(k8, ks, v8, vs) of every layer of an 8-bit copy case."""
    return [s["pools"][i:i + 4] for i in range(0, len(s["pools"]), 4)]


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _run_own(s, kind)
    if kind == "attention":
        return _plain_attention(s)
    if kind == "load":
        return _plain_load(s)
    if kind == "store":
        _plain_store(s)
        return _plain_load(s)
    _plain_copy(s)
    if not s["case"]["block"]:
        return s["pools"]
    return [_plain_load(dict(s, k8=k8, ks=ks, v8=v8, vs=vs)) for k8, ks, v8, vs in _by_layer(s)]


def _run_own(s, kind):
    from paper_2404_00242_amd import binding

    if kind == "attention":
        return binding.deft_tree_attn_decode_q8(s["plan"], s["q"], _cache(s))
    if kind == "copy":
        binding.deft_kv_copy_pages(s["copies"], s["pools"])
        if not s["case"]["block"]:
            return s["pools"]
        return [binding.deft_kv_load_q8(s["named_all"], _cache(dict(s, k8=k8, ks=ks, v8=v8, vs=vs))) for k8, ks, v8, vs in _by_layer(s)]
    if kind == "store":
        binding.deft_kv_store_q8(s["named"], s["k"], s["v"], _cache(s))
    return binding.deft_kv_load_q8(s["named_all"], _cache(s))


def work(case):
    """Every byte that has to be read or written once, and the products of the attention."""
    kind, Hkv, d, block = case["kind"], case["Hkv"], case["d"], case["block"]
    if kind == "attention":
        lens, parents, queries = _tree(case)
        paths = _paths(parents, queries)
        tokens = sum(lens[u] for u in {u for p in paths for u in p})
        path_tokens = sum(lens[u] for p in paths for u in p)
        rows = len(queries) * case["Hq"]
        return {"bytes": float(2 * tokens * Hkv * d + 2 * -(-tokens // block) * Hkv + rows * d * 4),
                "flops": float(4 * path_tokens * case["Hq"] * d)}
    if kind == "copy":
        page = case["page"] * Hkv * d * (1 if block else 2) + (case["page"] // block * Hkv if block else 0)
        back = 3 * case["pages"] * case["page"] * Hkv * d if block else 0
        return {"bytes": float(2 * case["layers"] * (2 * case["moves"] * page + back)), "flops": 0.0}
    pool, at = _row_tables(case)
    back = len(at) if kind == "load" else pool
    wrote = len(at) if kind == "store" else 0
    return {"bytes": float(2 * Hkv * d * (3 * wrote + 3 * back) + 2 * Hkv * -(-(wrote + back) // block)), "flops": 0.0}


# ---- from the definitions, in 64 bits ----

def _exact_rows(x, x8, s, rows, block):
    """Values of the whole pool after the rows x were stored, block by block on the host."""
    x8, byte = x8.cpu().double().numpy(), s.view(torch.uint8).cpu().numpy().astype(np.int64)
    x, rows = x.cpu().double().numpy(), rows.cpu().numpy()
    out = x8 * np.exp2(byte - 127.0)[np.arange(len(x8)) // block][..., None]
    order = np.argsort(rows, kind="stable")
    cut = np.flatnonzero(np.diff(rows[order] // block)) + 1
    for part in np.split(order, cut):
        b, pos = rows[part[0]] // block, rows[part] % block
        kept = slice(b * block, b * block + pos.min())
        top = np.abs(x[part]).max(axis=(0, 2))
        e = np.full(top.shape, E_MIN)
        e[top > 0] = np.clip(np.ceil(np.log2(top[top > 0] / 448.0)) + 127, E_MIN, E_MAX)  # (far from a rounding: top has 8 bits)
        if pos.min() > 0:
            e = np.maximum(e, byte[b])
        behind = slice(kept.stop, (b + 1) * block)  # bytes stay, also of rows that hold nothing, and take the new scale
        out[behind] = x8[behind] * np.exp2(e - 127.0)[None, :, None]
        if pos.min() > 0:
            out[kept] = _round_e4m3(out[kept] / np.exp2(e - 127.0)[None, :, None]) * np.exp2(e - 127.0)[None, :, None]
        out[rows[part]] = _round_e4m3(x[part] / np.exp2(e - 127.0)[None, :, None]) * np.exp2(e - 127.0)[None, :, None]
    return torch.from_numpy(out)


def _round_e4m3(x):
    """To three bits behind the leading one, or to multiples of 2^-9 below 2^-6; ties to even, 448 at most."""
    with np.errstate(divide="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(x))), -6) - 3)
    return np.clip(np.rint(x / step) * step, -448, 448)


def exact(case, seed):
    if case["kind"] == "copy":
        return None  # nothing is computed
    if case["kind"] == "store" and case["n"] * case["Hkv"] * case["d"] > 40_000_000:
        return None  # over 20 seconds
    s = prepare(case, seed)
    pairs = [(s["k8"], s["ks"]), (s["v8"], s["vs"])]
    block = case["block"]
    if case["kind"] == "store":
        return [_exact_rows(x, x8, sc, s["rows"], block) for x, (x8, sc) in zip((s["k"], s["v"]), pairs)]
    whole = [x8.double() * torch.exp2(sc.view(torch.uint8).double() - 127).repeat_interleave(block, 0)[: x8.shape[0], :, None]
             for x8, sc in pairs]
    if case["kind"] == "load":
        return [x[s["rows"]] for x in whole]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    lens, parents, queries = _tree(case)
    first = np.concatenate([[0], np.cumsum(lens)])
    out = torch.zeros((len(queries), Hq, d), dtype=torch.float64, device=s["q"].device)
    for j, path in enumerate(_paths(parents, queries)):
        at = torch.cat([s["rows"][first[u]:first[u + 1]] for u in path])
        k, v = (x[at].transpose(0, 1).contiguous() for x in whole)
        p = torch.softmax(torch.matmul(s["q"][j].double().view(Hkv, Hq // Hkv, d), k.transpose(1, 2).contiguous()) / math.sqrt(d), -1)
        out[j] = torch.matmul(p, v).reshape(Hq, d)
    return out

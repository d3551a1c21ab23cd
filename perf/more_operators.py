"""The operators of a paged cache held in 4 bits, and of per-head norms before the
rotation, and what they are measured on: `run` in its plain form (elementary
torch operations, in 32 bits unless said otherwise) or, where `own` is true,
through the library's entry points.

A case's "kind" names the operator:

  norm     paged_kv_store_norm: queries and keys normed for each head, turned,
           keys and values written into 16-bit pages
  append   paged_kv_store_q4: the same into 4-bit pages, and the written rows
           read back as the cache now holds them (paged_kv_load_q4)
  load     paged_kv_load_q4: rows of several layers out of 4-bit pages
  attend   paged_tree_attention_q4 of one layer over 4-bit pages
  accept   paged_accept_q4: greedy acceptance of a batch, the accepted rows moved
           in the pages of every layer, the lengths advanced; then those rows
           read back

4 bits: 32 consecutive elements of a head share a scale, an unsigned 8-bit float
(5 exponent bits, 3 mantissa bits: an fp16 number's bits 7 to 14), and code c of
4 bits stands for (c - 8) * scale.  A page of one head holds its slots' codes
(element e in byte e / 2, the even one below), then its slots' scales.

A case fixes every size ("shape_seed" draws the ragged ones); the seed draws the
values.
"""
from __future__ import annotations

import itertools
import math
import random

import numpy as np
import torch

own = False

NODES = 64          # nodes of the largest tree
TREE_SIZES = (1, 2, 4, 8, 16, 26, 40, 64)
BRANCHING = (4, 3, 2, 2, 2)
GROUP = 32          # elements of a scale
MAX_SCALE = 9216.0  # 7 times it is an fp16 number
THETA = 10000.0
EPS = 1e-6
NEG = float("-inf")


# ---------------------------------------------------------------- the cases


def listed():
    gqa = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    mha = {"q_heads": 32, "kv_heads": 32, "head_dim": 128}
    plain = {"cap": 0.0, "window": 0, "sink": 0, "bias": False, "begin": False}
    return [
        # the new rows of a ragged batch of eight trees in one layer, a model that norms its heads
        {"name": "norm_step", "kind": "norm", "dtype": "bf16", "batch": 8, "rows_min": 4, "rows_max": 64, "page": 16,
         "layout": "heads", "axes": 1, "norm": True, "shape_seed": 5, **gqa},
        # a prompt of text and images (time, height, width), odd length
        {"name": "norm_prompt", "kind": "norm", "dtype": "f16", "batch": 1, "rows_min": 8191, "rows_max": 8191,
         "page": 64, "layout": "slots", "axes": 3, "norm": True, "shape_seed": 7, **mha},
        # the new rows of a ragged batch of eight trees in one layer, into 4 bits
        {"name": "append_step", "kind": "append", "dtype": "bf16", "batch": 8, "rows_min": 4, "rows_max": 64,
         "page": 16, "axes": 1, "norm": False, "shape_seed": 5, **gqa},
        # a prompt of odd length into 4 bits, normed heads
        {"name": "append_prompt", "kind": "append", "dtype": "bf16", "batch": 1, "rows_min": 8191, "rows_max": 8191,
         "page": 64, "axes": 1, "norm": True, "shape_seed": 7, **mha},
        # one layer of a short prefix, before the rest of its prompt attends to it
        {"name": "load_small", "kind": "load", "dtype": "f16", "batch": 1, "rows_min": 200, "rows_max": 200,
         "layers": 1, "page": 16, "shape_seed": 3, "q_heads": 4, "kv_heads": 4, "head_dim": 64},
        # all layers of four requests that leave the server
        {"name": "load_layers", "kind": "load", "dtype": "bf16", "batch": 4, "rows_min": 1000, "rows_max": 3000,
         "layers": 32, "page": 16, "shape_seed": 8, **gqa},
        # the smallest: one small head group, a 7-node tree, a distance bias
        {"name": "attend_tiny", "kind": "attend", "dtype": "f16", "batch": 1, "q_heads": 4, "kv_heads": 4,
         "head_dim": 64, "prefix_min": 128, "prefix_max": 128, "nodes_min": 7, "nodes_max": 7, "page": 16,
         "shape_seed": 1, **plain, "bias": True},
        # a ragged batch of trees with grouped queries, capped scores, and a window that the longest pass
        {"name": "attend_trees", "kind": "attend", "dtype": "bf16", "batch": 8, **gqa, "prefix_min": 512,
         "prefix_max": 8192, "nodes_min": 4, "nodes_max": 64, "page": 64, "shape_seed": 5, **plain, "cap": 50.0,
         "window": 4096},
        # plain decoding: one token for each of 64 requests
        {"name": "attend_decode", "kind": "attend", "dtype": "bf16", "batch": 64, **gqa, "prefix_min": 512,
         "prefix_max": 16384, "nodes_min": 1, "nodes_max": 1, "page": 16, "shape_seed": 8, **plain},
        # one layer of a long context, a chain of drafts, a document that begins inside the cache
        {"name": "attend_long", "kind": "attend", "dtype": "bf16", "batch": 1, **gqa, "prefix_min": 131000,
         "prefix_max": 131000, "nodes_min": 4, "nodes_max": 4, "page": 128, "shape_seed": 9, **plain, "begin": True},
        # one request of a two-layer draft model
        {"name": "accept_small", "kind": "accept", "dtype": "f16", "batch": 1, "layers": 2, "kv_heads": 4,
         "head_dim": 64, "prefix_min": 128, "prefix_max": 128, "nodes_min": 26, "nodes_max": 26, "page": 16,
         "shape_seed": 3},
        # 64 requests, all layers of a grouped-query model
        {"name": "accept_serving", "kind": "accept", "dtype": "bf16", "batch": 64, "layers": 32, "kv_heads": 8,
         "head_dim": 128, "prefix_min": 32, "prefix_max": 512, "nodes_min": 4, "nodes_max": 64, "page": 16,
         "shape_seed": 4},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_span(rng, lo, hi):
    a = _log_int(rng, lo, hi)
    return a, _log_int(rng, a, hi)


def _draw_heads(rng):
    while True:
        kv, group = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([1, 1, 2, 3, 4, 7, 8])
        if kv * group <= 64:
            return {"q_heads": kv * group, "kv_heads": kv, "head_dim": rng.choice([64, 128, 128])}


def draw(rng):
    """One more case of the ranges above: batches of 1 to 64, prefixes of 1 to
    32768, trees of 1 to 64 nodes, pages of 8 to 256 slots, groups of 1 to 8."""
    limits = {}
    for c in listed():
        w = work(c)
        limits.setdefault(c["kind"], []).append((w["bytes"], w["flops"]))
    while True:
        kind = rng.choice(["norm", "append", "append", "load", "attend", "attend", "attend", "attend", "accept"])
        c = {"kind": kind, "dtype": rng.choice(["bf16", "f16"]), "batch": _log_int(rng, 1, 64),
             "page": rng.choice([8, 16, 16, 32, 64, 128, 256]), **_draw_heads(rng), "shape_seed": rng.randint(0, 10**6)}
        if kind in ("norm", "append", "load"):
            c["rows_min"], c["rows_max"] = _draw_span(rng, 1, 8192)
        else:
            c["nodes_min"], c["nodes_max"] = _draw_span(rng, 1, 64)
        if kind in ("norm", "append"):
            c.update(axes=rng.choice([1, 2, 3]), norm=kind == "norm" or rng.random() < 0.5)
        if kind == "norm":
            c["layout"] = rng.choice(["heads", "slots"])
        if kind in ("load", "accept"):
            c["layers"] = _log_int(rng, 1, 32)
        if kind == "attend":
            c["prefix_min"], c["prefix_max"] = _draw_span(rng, 1, 32768)
            window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
            c.update(cap=rng.choice([0.0, 0.0, 30.0, 50.0]), window=window,
                     sink=rng.choice([0, 4, 130]) if window else 0, bias=rng.random() < 0.25, begin=rng.random() < 0.25)
        if kind == "accept":
            c["prefix_min"], c["prefix_max"] = _draw_span(rng, 1, 512)
        if _plain_cost(c) <= max(_plain_cost(x) for x in listed() if x["kind"] == kind):
            w = work(c)
            if any(w["bytes"] <= b and w["flops"] <= f for b, f in limits[kind]):
                return c


def _plain_cost(case):
    """Elements that a pass in the plain form goes through, a padded batch where it pads one."""
    kind, B = case["kind"], case["batch"]
    if kind in ("norm", "append"):
        return B * case["rows_max"] * (case["q_heads"] + 2 * case["kv_heads"]) * case["head_dim"]
    if kind == "load":
        return B * case["rows_max"] * case["layers"] * case["kv_heads"] * case["head_dim"]
    if kind == "attend":
        S = case["prefix_max"] + case["nodes_max"]
        return B * S * (case["kv_heads"] * case["head_dim"] + case["q_heads"] * case["nodes_max"])
    return B * (case["prefix_max"] + NODES) * case["layers"] * case["kv_heads"] * case["head_dim"]


# ---------------------------------------------------------------- shapes: part of a case, the same for every seed


def _rank_product_tree(n):
    """The first n nodes of the rank-product tree, in breadth-first order."""
    t = [()]
    for depth in range(1, len(BRANCHING) + 1):
        t.extend(itertools.product(*[range(b) for b in BRANCHING[:depth]]))
    kept = sorted(sorted(t, key=lambda x: (sum(x), len(x), x))[:n], key=lambda x: (len(x), x))
    index = {x: i for i, x in enumerate(kept)}
    return [index[x[:-1]] if x else -1 for x in kept]


def _shape(case):
    """The ragged sizes of a case: rows or prefix lengths, the trees and which
    request has which, and what else its kind needs."""
    r = random.Random(case["shape_seed"])
    B = case["batch"]
    s = {}
    if "nodes_min" in case:
        lo, hi = case["nodes_min"], case["nodes_max"]
        sizes = [n for n in TREE_SIZES if lo <= n <= hi] or [lo]
        trees = [_rank_product_tree(n) for n in sizes]
        n = r.randint(lo, hi)
        trees.append([-1] + sorted(r.randrange(i) for i in range(1, n)) if n > 1 else [-1])  # parents in order: breadth-first
        n = r.randint(lo, hi)
        trees.append(list(range(-1, min(n, 12) - 1)) if lo <= min(n, 12) else trees[0])  # a chain
        s["trees"] = [_canonical(t) for t in trees]
        s["tree"] = [r.randrange(len(trees)) for _ in range(B)]
        s["n"] = [len(s["trees"][t]) for t in s["tree"]]
        s["L"] = [r.randint(case["prefix_min"], case["prefix_max"]) for _ in range(B)]
    else:
        s["n"] = [r.randint(case["rows_min"], case["rows_max"]) for _ in range(B)]
    if case["kind"] == "attend":
        s["begin"] = [r.randint(0, L) // 2 if case["begin"] else 0 for L in s["L"]]
    if case["kind"] == "accept":
        s["last"] = [r.randrange(n) for n in s["n"]]  # the deepest accepted node
    return s


def _canonical(parent):
    """The tree renumbered breadth-first, children in increasing order."""
    kids = {i: [c for c, p in enumerate(parent) if p == i] for i in range(len(parent))}
    order = [0]
    for u in order:
        order.extend(kids[u])
    new = {u: i for i, u in enumerate(order)}
    return [-1 if u == 0 else new[parent[u]] for u in order]


def _depths(parent):
    d = [0] * len(parent)
    for i in range(1, len(parent)):
        d[i] = d[parent[i]] + 1
    return d


def _path(parent, u):
    p = []
    while u >= 0:
        p.append(u)
        u = parent[u]
    return p[::-1]


def _seen_keys(case, s):
    """Keys that some row of each request may see."""
    total = []
    for L, n, b0 in zip(s["L"], s["n"], s["begin"]):
        lo = max(b0, L - case["window"] + 1) if case["window"] else b0
        total.append(L + n - lo + max(0, min(b0 + case["sink"], lo) - b0))
    return total


def _row_bytes(d):
    """A head's row in 4 bits: codes and scales."""
    return d // 2 + d // GROUP


def work(case):
    s, kind, d = _shape(case), case["kind"], case["head_dim"]
    R, H = sum(s["n"]), case["kv_heads"]
    if kind in ("norm", "append"):
        Hq = case["q_heads"]
        ins = R * (2.0 * (Hq + 2 * H) * d + 8 + 4 * case["axes"])
        flops = R * d * (Hq + H) * (3.0 + (4.0 if case["norm"] else 0.0))
        if kind == "norm":
            return {"bytes": ins + 2.0 * R * (Hq + 2 * H) * d, "flops": flops}
        # the rows are written, read again and returned in 16 bits
        return {"bytes": ins + 2.0 * R * Hq * d + R * 2 * H * (2.0 * _row_bytes(d) + 2.0 * d) + 8.0 * R,
                "flops": flops + 4.0 * R * 2 * H * d}
    if kind == "load":
        return {"bytes": 8.0 * R + R * case["layers"] * 2 * H * (_row_bytes(d) + 2.0 * d),
                "flops": 2.0 * R * case["layers"] * 2 * H * d}
    if kind == "attend":
        keys = _seen_keys(case, s)
        return {"bytes": sum(2.0 * k * H * _row_bytes(d) for k in keys) + 4.0 * R * case["q_heads"] * d,
                "flops": sum(4.0 * k * n for k, n in zip(keys, s["n"])) * case["q_heads"] * d}
    paths = [_path(s["trees"][t], u) for t, u in zip(s["tree"], s["last"])]
    moved = sum(i != p for path in paths for i, p in enumerate(path))
    kept = sum(len(path) for path in paths)
    heads = case["layers"] * H * 2.0
    return {"bytes": heads * (2 * moved * _row_bytes(d) + kept * (_row_bytes(d) + 2 * d)) + 8.0 * R + 400.0 * case["batch"],
            "flops": 2.0 * heads * kept * d}


# ---------------------------------------------------------------- inputs

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & (2**62 - 1))
    return g


def _normal(shape, g, dtype, std=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    out.normal_(0.0, std, generator=g)
    return out


def _ints(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def _starts(n):
    return [0, *itertools.accumulate(n)]


def _pool_q4(case, n_pages, g, layers=1):
    """K and V pages [layers][pages][kv heads][bytes of a page's head], full of rows as a
    cache holds them: codes as normal values give them, scales of about 0.2 to 0.4."""
    H, P, d = case["kv_heads"], case["page"], case["head_dim"]
    pools = []
    for _ in range(2):
        pool = torch.empty((layers, n_pages, H, P * _row_bytes(d)), dtype=torch.uint8, device="cuda")
        codes, scales = _parts(pool, P, d)
        for layer in range(layers):
            for at in range(0, n_pages, 4096):  # in pieces: the values take 16 bits each on the way
                x = _normal((min(4096, n_pages - at), H, P, d), g, torch.float16, 2.5)
                c = (x.round_().clamp_(-7, 7) + 8).to(torch.uint8)
                codes[layer, at:at + 4096] = c[..., 0::2] | (c[..., 1::2] << 4)
            scales[layer] = torch.randint(0x64, 0x6D, scales[layer].shape, generator=g, device="cuda", dtype=torch.uint8)
        pools.append(pool)
    return pools


def _parts(pool, P, d):
    """The codes [...][P][d / 2] and the scales [...][P][d / 32] of a pool, as views."""
    cut = P * d // 2
    return pool[..., :cut].unflatten(-1, (P, d // 2)), pool[..., cut:].unflatten(-1, (P, d // GROUP))


def _pool_16(case, n_pages, g):
    H, P, d, dt = case["kv_heads"], case["page"], case["head_dim"], DTYPES[case["dtype"]]
    if case["layout"] == "heads":
        return [_normal((1, n_pages, H, P, d), g, dt) for _ in range(2)]
    return [_normal((1, n_pages, P, H, d), g, dt).transpose(2, 3) for _ in range(2)]


def _tables(case, spans, r):
    """A block table with scattered pages for each request's span of slots; how many pages the pool has."""
    P = case["page"]
    counts = [-(-x // P) for x in spans]
    n_pages = sum(counts) + 3
    ids = list(range(n_pages))
    r.shuffle(ids)
    width = max(max(counts), 1) + 1
    table = torch.full((case["batch"], width), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = torch.tensor(ids[at:at + c], dtype=torch.int32)
        at += c
    return table.cuda(), n_pages


def _tree_tables(trees):
    """[trees][64] parents and depths and [trees][64][64] ancestor-or-self flags."""
    par = torch.full((len(trees), NODES), -1, dtype=torch.int64)
    dep = torch.zeros((len(trees), NODES), dtype=torch.int64)
    anc = torch.zeros((len(trees), NODES, NODES), dtype=torch.bool)
    for t, p in enumerate(trees):
        par[t, :len(p)] = torch.tensor(p)
        dep[t, :len(p)] = torch.tensor(_depths(p))
        for i in range(len(p)):
            anc[t, i, _path(p, i)] = True
    return {"par": par.cuda(), "dep": dep.cuda(), "anc": anc.cuda()}


def _rows_of(n):
    """Request and place within it of every row."""
    owner = [b for b, k in enumerate(n) for _ in range(k)]
    place = [i for k in n for i in range(k)]
    return _ints(owner, torch.int64), _ints(place, torch.int64)


def prepare(case, seed):
    kind, s = case["kind"], _shape(case)
    g, r = _generator(seed, 1), random.Random(seed * 7919 + 17)
    st = {"case": case, "n": s["n"], "R": sum(s["n"])}
    if "trees" in s:
        st["tree"] = _ints(s["tree"])
        st["tables"] = _tree_tables(s["trees"])
        st["L"] = _ints(s["L"])
    st["row_start"] = _ints(_starts(s["n"]))
    {"norm": _prepare_rows, "append": _prepare_rows, "load": _prepare_load, "attend": _prepare_attend,
     "accept": _prepare_accept}[kind](case, s, st, g, r)
    if own:
        import paper_2606_27550_gb300 as tv

        st["tv"] = tv
        if kind == "norm":
            st["pages"] = tv.Pages(st["k_pages"], st["v_pages"])
        else:
            st["pages"] = tv.PagesQ4(st["k_pages"], st["v_pages"], case["page"], case["head_dim"], DTYPES[case["dtype"]])
        if "trees" in s:
            st["bank"] = tv.Bank(len(s["trees"]), torch.cuda.current_device())
            for t in s["trees"]:
                st["bank"].add(t)
            st["req"] = tv.Requests(lens=st["L"], table=st["table"], page_size=case["page"],
                                    row_start=st["row_start"], tree=st["tree"], key_begin=st.get("begin"))
        if kind == "attend":
            # as for the first layer of a step: the same plan serves every layer
            st["plan"] = tv.make_paged_plan(case["batch"])
            slots = torch.zeros(st["R"], dtype=torch.int64, device="cuda")
            positions = torch.zeros(st["R"], dtype=torch.int32, device="cuda")
            status = torch.zeros(case["batch"], dtype=torch.int32, device="cuda")
            tv.paged_plan(st["bank"], st["req"], slots, positions, status, st["plan"], n_q_heads=case["q_heads"],
                          n_kv_heads=case["kv_heads"], window=case["window"], sink=case["sink"])
            st["ws"] = tv.make_workspace(tv.tb_workspace_size(1, 1, case["kv_heads"], case["q_heads"],
                                                              case["head_dim"], 1, torch.cuda.current_device()))
    return st


def _prepare_rows(case, s, st, g, r):
    R, d, P, H, Hq = st["R"], case["head_dim"], case["page"], case["kv_heads"], case["q_heads"]
    dt = DTYPES[case["dtype"]]
    table, n_pages = _tables(case, s["n"], r)
    owner, place = _rows_of(s["n"])
    page = table.long()[owner, place // P]
    st["slots"] = page * P + place % P
    st["k_pages"], st["v_pages"] = (_pool_16 if case["kind"] == "norm" else _pool_q4)(case, n_pages, g)
    # the projection's output, as a model has it: q, k and v side by side, some channels larger than others
    qkv = _normal((R, Hq + 2 * H, d), g, dt)
    qkv *= torch.exp(_normal((Hq + 2 * H, d), g, torch.float32, 0.5)).to(dt)
    st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    st["q_out"] = torch.empty((R, Hq, d), dtype=dt, device="cuda")
    if case["norm"]:
        for name in ("q_norm", "k_norm"):
            st[name] = (1.0 + _normal((d,), g, torch.float32, 0.2)).to(dt)
    axes = [torch.randint(0, m, (R,), generator=g, device="cuda", dtype=torch.int32) for m in (100000, 256, 256)]
    st["positions"] = torch.stack(axes[:case["axes"]]).contiguous()
    half = d // 2
    st["sections"] = {1: (half,), 2: (half // 2, half - half // 2),
                      3: (half // 4, half * 3 // 8, half - half // 4 - half * 3 // 8)}[case["axes"]]
    # cos and sin are computed from the frequencies in the call: positions are new in every step
    st["freq"] = torch.from_numpy(THETA ** (-2.0 * np.arange(half) / d)).cuda()
    st["axis"] = _ints([a for a, n in enumerate(st["sections"]) for _ in range(n)], torch.int64)
    if case["kind"] == "append":
        st["k_rows"], st["v_rows"] = (torch.empty((R, H, d), dtype=dt, device="cuda") for _ in range(2))


def _prepare_load(case, s, st, g, r):
    R, d, P, H = st["R"], case["head_dim"], case["page"], case["kv_heads"]
    table, n_pages = _tables(case, s["n"], r)
    owner, place = _rows_of(s["n"])
    st["slots"] = table.long()[owner, place // P] * P + place % P
    st["k_pages"], st["v_pages"] = _pool_q4(case, n_pages, g, case["layers"])
    st["k_rows"], st["v_rows"] = (torch.empty((case["layers"], R, H, d), dtype=DTYPES[case["dtype"]], device="cuda")
                                  for _ in range(2))


def _prepare_attend(case, s, st, g, r):
    d, dt = case["head_dim"], DTYPES[case["dtype"]]
    st["table"], n_pages = _tables(case, [L + n for L, n in zip(s["L"], s["n"])], r)
    st["k_pages"], st["v_pages"] = _pool_q4(case, n_pages, g)
    st["q"] = _normal((st["R"], case["q_heads"], d), g, dt, 2.0)
    st["out"] = torch.empty((st["R"], case["q_heads"], d), dtype=dt, device="cuda")
    st["lse"] = torch.empty((st["R"], case["q_heads"]), dtype=torch.float32, device="cuda")
    if case["bias"]:
        st["slopes"] = 2.0 ** (-8.0 * torch.arange(1, case["q_heads"] + 1, device="cuda") / case["q_heads"])
    if case["begin"]:
        st["begin"] = _ints(s["begin"])
    st["owner"], st["place"] = _rows_of(s["n"])
    st["keys"] = max(L + n for L, n in zip(s["L"], s["n"]))
    st["width"] = max(s["n"])


def _prepare_accept(case, s, st, g, r):
    B, P = case["batch"], case["page"]
    st["table"], n_pages = _tables(case, [L + n for L, n in zip(s["L"], s["n"])], r)
    st["k_pages"], st["v_pages"] = _pool_q4(case, n_pages, g, case["layers"])
    vocab = st["vocab"] = 32000
    draft, argmax, kept = [], [], []
    table = st["table"].tolist()
    for b in range(B):
        tree = s["trees"][s["tree"][b]]
        path = _path(tree, s["last"][b])
        tokens = r.sample(range(vocab - 1), len(tree))
        then = {u: tokens[v] for u, v in zip(path, path[1:])}
        draft += tokens
        argmax += [then.get(u, vocab - 1) for u in range(len(tree))]
        kept += [table[b][x // P] * P + x % P for x in range(s["L"][b], s["L"][b] + len(path))]
    st["draft"], st["argmax"] = _ints(draft), _ints(argmax)
    st["results"] = torch.zeros((B, 4 + NODES), dtype=torch.int32, device="cuda")
    st["lens_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    st["depth"] = max(max(_depths(t)) for t in s["trees"]) + 1
    st["slots"] = _ints(kept, torch.int64)
    st["k_rows"], st["v_rows"] = (torch.empty((case["layers"], len(kept), case["kv_heads"], case["head_dim"]),
                                              dtype=DTYPES[case["dtype"]], device="cuda") for _ in range(2))


# ---------------------------------------------------------------- one pass


def run(st):
    return {"norm": _norm, "append": _append, "load": _load, "attend": _attend, "accept": _accept}[st["case"]["kind"]](st)


def _head_norm(x, weight):
    """x / sqrt(mean(x^2) + eps) * weight.  The root in 64 bits: what follows rounds to 4 bits,
    and a value next to a border between two of them must not depend on the order of a sum."""
    r = torch.rsqrt(x.double().square().mean(-1, keepdim=True) + EPS).float()
    return x * r * weight.float()


def _turn(x, cos, sin):
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _turned_rows(st):
    """Queries and keys, normed where the case has norms, turned, in 32 bits."""
    # angles past a few turns lose their fraction in 32 bits: this product is taken in 64
    angle = st["positions"].T[:, st["axis"]].double() * st["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q, k = st["q"].float(), st["k"].float()
    if st["case"]["norm"]:
        q, k = _head_norm(q, st["q_norm"]), _head_norm(k, st["k_norm"])
    return _turn(q, cos, sin), _turn(k, cos, sin)


def _rules(st):
    """The arguments of both stores."""
    more = {"q_norm": st["q_norm"], "k_norm": st["k_norm"], "eps": EPS} if st["case"]["norm"] else {}
    return dict(q=st["q"], q_out=st["q_out"], positions=st["positions"], sections=st["sections"], rope_theta=THETA, **more)


def _norm(st):
    out = {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if own:
        st["tv"].paged_kv_store_norm(st["pages"], st["slots"], st["k"], st["v"], **_rules(st))
        return out
    P = st["case"]["page"]
    q, k = _turned_rows(st)
    st["q_out"].copy_(q)
    page, at = st["slots"] // P, st["slots"] % P
    st["k_pages"][0].transpose(1, 2)[page, at] = k.to(st["k_pages"].dtype)
    st["v_pages"][0].transpose(1, 2)[page, at] = st["v"]
    return out


def _quantize(x):
    """Codes [..., d / 2] (two to a byte) and scales [..., d / 32] of rows in 32 bits."""
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    t = top / torch.full_like(top, 7.0)                            # (by a plain number it would be a product with 1/7)
    low = torch.frexp(t).exponent.clamp(min=-13) - 4
    step = ((low + 127) << 23).view(torch.float32)                 # 2^low: the last of 4 significant bits
    scale = (torch.ceil(t / step) * step).clamp(max=MAX_SCALE)
    code = torch.where(scale[..., None] > 0, torch.round(g / scale[..., None]), 0.0).clamp(-7, 7)
    code = (code + 8).to(torch.uint8).flatten(-2)
    bits = (scale.half().view(torch.int16) >> 7).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), bits


def _values(codes, scales):
    """Rows [..., d] in 32 bits of codes and scales."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    s = (scales.to(torch.int16) << 7).view(torch.float16).float()
    return ((c.float() - 8).unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def _append(st):
    case = st["case"]
    out = {"q": st["q_out"], "k": st["k_rows"], "v": st["v_rows"]}
    if own:
        st["tv"].paged_kv_store_q4(st["pages"], st["slots"], st["k"], st["v"], **_rules(st))
        st["tv"].paged_kv_load_q4(st["pages"], st["slots"], st["k_rows"], st["v_rows"])
        return out
    P, d = case["page"], case["head_dim"]
    q, k = _turned_rows(st)
    st["q_out"].copy_(q)
    page, at = st["slots"] // P, st["slots"] % P
    for pool, x, rows in ((st["k_pages"], k, st["k_rows"]), (st["v_pages"], st["v"].float(), st["v_rows"])):
        codes, scales = (p[0].transpose(1, 2) for p in _parts(pool, P, d))
        codes[page, at], scales[page, at] = _quantize(x)
        rows.copy_(_values(codes[page, at], scales[page, at]))
    return out


def _read(st):
    P, d = st["case"]["page"], st["case"]["head_dim"]
    page, at = st["slots"] // P, st["slots"] % P
    for pool, rows in ((st["k_pages"], st["k_rows"]), (st["v_pages"], st["v_rows"])):
        codes, scales = (p.transpose(2, 3) for p in _parts(pool, P, d))   # [layers, pages, slots, heads, bytes]
        rows.copy_(_values(codes[:, page, at], scales[:, page, at]))


def _load(st):
    if own:
        st["tv"].paged_kv_load_q4(st["pages"], st["slots"], st["k_rows"], st["v_rows"])
    else:
        _read(st)
    return {"k": st["k_rows"], "v": st["v_rows"]}


def _attend(st):
    case = st["case"]
    if own:
        st["tv"].paged_tree_attention_q4(st["bank"], st["req"], st["pages"], st["plan"], st["q"], st["out"], st["ws"],
                                         softcap=case["cap"], slopes=st.get("slopes"), lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    P, B, S, N = case["page"], case["batch"], st["keys"], st["width"]
    H, Hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    G, L = Hq // H, st["L"].long()
    slot = torch.arange(S, device="cuda")
    page = st["table"].long()[:, slot // P].clamp(min=0)
    k, v = (_values(*(p[0].transpose(1, 2)[page, slot % P] for p in _parts(pool, P, d)))  # [B, S, H, d]
            for pool in (st["k_pages"], st["v_pages"]))
    q = torch.zeros((B, N, Hq, d), dtype=torch.float32, device="cuda")
    q[st["owner"], st["place"]] = st["q"].float()
    q = q.view(B, N, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, d)
    z = (q @ k.permute(0, 2, 3, 1)) / math.sqrt(d)
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    z = z.view(B, H, G, N, S)
    t = st["tree"].long()
    node = (slot - L[:, None])                                     # [B, S]: tree index of a slot
    inside = (node >= 0) & (node < NODES)
    node_c = node.clamp(0, NODES - 1)
    anc, dep = st["tables"]["anc"][t], st["tables"]["dep"][t]      # [B, 64, 64], [B, 64]
    pos_k = torch.where(node < 0, slot, L[:, None] + torch.gather(dep, 1, node_c))
    dist = (L[:, None] + dep[:, :N])[:, :, None] - pos_k[:, None]  # [B, N, S]
    see = torch.gather(anc[:, :N], 2, node_c[:, None].expand(B, N, S)) & inside[:, None]
    see |= (node < 0)[:, None]
    first = st["begin"].long()[:, None] if "begin" in st else torch.zeros_like(L)[:, None]
    if case["window"]:
        see &= (dist < case["window"]) | (slot < first + case["sink"])[:, None]
    see &= (slot >= first)[:, None]
    if case["bias"]:
        z = z - st["slopes"].view(1, H, G, 1, 1) * dist[:, None, None]
    z = z.masked_fill(~see[:, None, None], NEG)
    m = z.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(z - m)
    l = p.sum(-1, keepdim=True)
    o = (p / l.clamp(min=1e-38)).reshape(B, H, G * N, S) @ v.permute(0, 2, 1, 3)
    o = o.view(B, H, G, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, Hq, d)
    lse = (m + torch.log(l)).view(B, H, G, N).permute(0, 3, 1, 2).reshape(B, N, Hq)
    st["out"].copy_(o[st["owner"], st["place"]])
    st["lse"].copy_(lse[st["owner"], st["place"]])
    return {"out": st["out"], "lse": st["lse"]}


def _accept(st):
    case = st["case"]
    out = {"results": st["results"], "lens": st["lens_out"], "k": st["k_rows"], "v": st["v_rows"]}
    if own:
        tv = st["tv"]
        tv.paged_accept_q4(st["bank"], st["req"], st["pages"], st["results"], draft=st["draft"], argmax=st["argmax"],
                           vocab=st["vocab"], lens_out=st["lens_out"])
        tv.paged_kv_load_q4(st["pages"], st["slots"], st["k_rows"], st["v_rows"])
        return out
    P, B, R, D = case["page"], case["batch"], st["R"], st["depth"]
    t, L = st["tree"].long(), st["L"].long()
    par, dep, anc = (st["tables"][k][t] for k in ("par", "dep", "anc"))
    node = torch.arange(NODES, device="cuda")
    first = st["row_start"].long()[:-1, None]
    row = (first + node).clamp(max=R - 1)
    real = anc.any(2)
    agree = st["draft"][row] == torch.gather(st["argmax"][row], 1, par.clamp(min=0))
    agree = (agree | (node == 0)) & real
    good = real & ~(anc & ~agree[:, None]).any(2)                 # every node of the root path agrees
    last = torch.where(good, dep * NODES + (NODES - 1 - node), -1).argmax(1)
    length = torch.gather(dep, 1, last[:, None])[:, 0] + 1
    on = anc[torch.arange(B, device="cuda"), last]                # nodes of the path, in order of depth
    path = torch.zeros((B, NODES), dtype=torch.int64, device="cuda")
    path.scatter_add_(1, dep, torch.where(on, node, 0))
    res = st["results"]
    res[:, 0], res[:, 2], res[:, 3] = length, L + length, 0
    res[:, 1] = st["argmax"][(first[:, 0] + last)]
    step = node < length[:, None]
    res[:, 4:] = torch.where(step, path, 0)
    st["lens_out"].copy_(L + length)
    to = (L[:, None] + node)[:, :D]
    to = torch.where(step[:, :D], to, L[:, None])
    src = torch.where(step[:, :D], L[:, None] + path[:, :D], L[:, None])
    table = st["table"].long()
    to_page, src_page = torch.gather(table, 1, to // P), torch.gather(table, 1, src // P)
    for pool in (st["k_pages"], st["v_pages"]):
        for part in _parts(pool, P, case["head_dim"]):
            flat = part.transpose(2, 3)                           # [layers, pages, slots, heads, bytes]
            flat[:, to_page, to % P] = flat[:, src_page, src % P]
    _read(st)
    return out


# ---------------------------------------------------------------- the same from the definitions, in 64 bits


def exact(case, seed):
    st = _plain_state(case, seed)
    return {"norm": _exact_rows, "append": _exact_rows, "load": _exact_load, "attend": _exact_attend,
            "accept": _exact_accept}[case["kind"]](case, _shape(case), st)


def _plain_state(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


# what a scale's byte stands for: (8 + m) 2^(e - 18), without the 8 and one step up where e is 0
_SCALES = np.array([(8 * (b >> 3 > 0) + (b & 7)) * 2.0 ** (max(b >> 3, 1) - 18) for b in range(256)])


def _exact_rows(case, s, st):
    d, P = case["head_dim"], case["page"]
    half = d // 2
    pos = st["positions"].double()
    turned = {}
    for name in ("q", "k"):
        x = st[name].double()
        if case["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS) * st[name + "_norm"].double()
        y = torch.empty_like(x)
        i = 0
        for axis, n in enumerate(st["sections"]):
            for _ in range(n):
                a = pos[axis] * THETA ** (-2.0 * i / d)
                c, n_ = torch.cos(a)[:, None], torch.sin(a)[:, None]
                y[:, :, i] = x[:, :, i] * c - x[:, :, i + half] * n_
                y[:, :, i + half] = x[:, :, i] * n_ + x[:, :, i + half] * c
                i += 1
        turned[name] = y
    v = st["v"].double()
    if case["kind"] == "norm":
        kp, vp = st["k_pages"].double(), st["v_pages"].double()
        page, at = st["slots"] // P, st["slots"] % P
        kp[0][page, :, at] = turned["k"]
        vp[0][page, :, at] = v
        return {"q": turned["q"], "k_pages": kp, "v_pages": vp}
    # the scale: the smallest of the table (up to its limit) that 7 codes reach the largest element with
    steps = torch.from_numpy(_SCALES[:int(np.argmax(_SCALES == MAX_SCALE)) + 1]).cuda()
    rows = {}
    for name, x in (("k", turned["k"]), ("v", v)):
        g = x.reshape(-1, GROUP)
        scale = steps[torch.searchsorted(7 * steps, g.abs().max(1).values).clamp(max=len(steps) - 1)][:, None]
        rows[name] = (torch.clamp(torch.round(g / scale.clamp(min=1e-30)), -7, 7) * scale).reshape(x.shape)
    return {"q": turned["q"], **rows}


def _exact_pool(case, pool):
    """The values [layers][pages][slots][heads][d] of a pool, in 64 bits."""
    P, d = case["page"], case["head_dim"]
    layers, pages, H, _ = pool.shape
    codes = pool[..., :P * d // 2].reshape(layers, pages, H, P, d // 2).int()
    scale = torch.from_numpy(_SCALES).cuda()[pool[..., P * d // 2:].reshape(layers, pages, H, P, d // GROUP).long()]
    x = torch.empty((layers, pages, H, P, d), dtype=torch.float64, device="cuda")
    x[..., 0::2] = (codes % 16 - 8) * scale.repeat_interleave(GROUP // 2, -1)
    x[..., 1::2] = (codes // 16 - 8) * scale.repeat_interleave(GROUP // 2, -1)
    return x.transpose(2, 3)


def _exact_load(case, s, st):
    out = {}
    for name in ("k", "v"):
        rows = []
        for layer in range(case["layers"]):
            x = _exact_pool(case, st[name + "_pages"][layer:layer + 1])[0].flatten(0, 1)
            rows.append(x[st["slots"]])
        out[name] = torch.stack(rows)
    return out


def _exact_attend(case, s, st):
    if _plain_cost(case) > 4e9:
        return None
    P, H, Hq, d = case["page"], case["kv_heads"], case["q_heads"], case["head_dim"]
    outs, lses = [], []
    at = 0
    table = st["table"].long()
    for b, (L, n) in enumerate(zip(s["L"], s["n"])):
        tree = s["trees"][s["tree"][b]]
        dep = _depths(tree)
        ids = table[b, :-(-(L + n) // P)]
        k, v = (_exact_pool(case, st[x][:, ids])[0].flatten(0, 1)[:L + n] for x in ("k_pages", "v_pages"))
        pos = list(range(L)) + [L + x for x in dep]
        q = st["q"][at:at + n].double()
        see = np.zeros((n, L + n), dtype=bool)
        dist = np.zeros((n, L + n))
        for i in range(n):
            see[i, :L] = True
            see[i, [L + a for a in _path(tree, i)]] = True
            dist[i] = L + dep[i] - np.asarray(pos)
            if case["window"]:
                near = dist[i] < case["window"]
                near[s["begin"][b]:s["begin"][b] + case["sink"]] = True
                see[i] &= near
            see[i, :s["begin"][b]] = False
        see, dist = torch.from_numpy(see).cuda(), torch.from_numpy(dist).cuda()
        o = torch.zeros((n, Hq, d), dtype=torch.float64, device="cuda")
        lse = torch.full((n, Hq), NEG, dtype=torch.float64, device="cuda")
        for h in range(Hq):
            g = h // (Hq // H)
            z = q[:, h] @ k[:, g].T / math.sqrt(d)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["bias"]:
                z = z - st["slopes"][h].double() * dist
            z = z.masked_fill(~see, NEG)
            lse[:, h] = torch.logsumexp(z, 1)
            o[:, h] = torch.softmax(z, 1) @ v[:, g]
        outs.append(o)
        lses.append(lse)
        at += n
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_accept(case, s, st):
    P, table = case["page"], st["table"].tolist()
    out = {"results": None, "lens": None}
    for name in ("k", "v"):
        rows = []
        for layer in range(case["layers"]):
            x = _exact_pool(case, st[name + "_pages"][layer:layer + 1])[0]
            for b in range(case["batch"]):
                L = s["L"][b]
                for u in _path(s["trees"][s["tree"][b]], s["last"][b]):
                    rows.append(x[table[b][(L + u) // P], (L + u) % P])
        kept = len(rows) // case["layers"]
        out[name] = torch.stack(rows).reshape(case["layers"], kept, case["kv_heads"], case["head_dim"])
    return out

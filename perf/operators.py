"""The operators of a serving step over a paged cache, and what they are
measured on: `run` in its plain form (elementary torch operations in 32 bits)
or, where `own` is true, through the library's entry points.

A case's "kind" names the operator:

  plan     paged_plan: block tables, slot maps, row offsets and positions of a
           batch from its lengths, with the pages that change hands
  store    paged_kv_store: queries and keys rotated at one to three position
           axes, keys and values written into their pages
  attend   paged_tree_attention of one layer over the pages
  logits   logits_process: penalties for repeated tokens, biases, grammar
           masks, and the statistics that the acceptance rules read
  accept   paged_accept: greedy acceptance of a batch, the accepted rows moved
           in the pages of every layer, the lengths advanced

A case fixes every size ("shape_seed" draws the ragged ones: prefix lengths,
trees, accepted paths); the seed draws the values.
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
TEMPERATURE = 0.7
THETA = 10000.0
NEG = float("-inf")


# ---------------------------------------------------------------- the cases


def listed():
    gqa = {"q_heads": 32, "kv_heads": 8, "head_dim": 128}
    mha = {"q_heads": 32, "kv_heads": 32, "head_dim": 128}
    return [
        # a ragged batch of eight between two steps: latency
        {"name": "plan_small", "kind": "plan", "batch": 8, "page": 16, "prefix_min": 512, "prefix_max": 8192,
         "nodes_min": 4, "nodes_max": 64, "prompts": False, "shape_seed": 5, **gqa},
        # a full server: growing, waiting and finished requests, a small page
        {"name": "plan_serving", "kind": "plan", "batch": 1024, "page": 16, "prefix_min": 1, "prefix_max": 8192,
         "nodes_min": 1, "nodes_max": 64, "prompts": False, "shape_seed": 6, **gqa},
        # the new rows of a ragged batch of eight trees in one layer
        {"name": "store_step", "kind": "store", "dtype": "bf16", "batch": 8, "rows_min": 4, "rows_max": 64, "page": 16,
         "layout": "heads", "axes": 1, "shape_seed": 5, **gqa},
        # a prompt of text and images (time, height, width), odd length
        {"name": "store_prompt", "kind": "store", "dtype": "f16", "batch": 1, "rows_min": 8191, "rows_max": 8191,
         "page": 64, "layout": "slots", "axes": 3, "shape_seed": 7, **mha},
        # the smallest: one small head group, a 7-node tree, a distance bias
        {"name": "attend_tiny", "kind": "attend", "dtype": "f16", "batch": 1, "q_heads": 4, "kv_heads": 4,
         "head_dim": 64, "prefix_min": 128, "prefix_max": 128, "nodes_min": 7, "nodes_max": 7, "page": 16,
         "layout": "heads", "cap": 0.0, "window": 0, "sink": 0, "bias": True, "begin": False, "shape_seed": 1},
        # a ragged batch of trees with grouped queries, capped scores, and a window that the longest pass
        {"name": "attend_trees", "kind": "attend", "dtype": "bf16", "batch": 8, **gqa, "prefix_min": 512,
         "prefix_max": 8192, "nodes_min": 4, "nodes_max": 64, "page": 64, "layout": "slots", "cap": 50.0,
         "window": 4096, "sink": 0, "bias": False, "begin": False, "shape_seed": 5},
        # plain decoding: one token for each of 64 requests
        {"name": "attend_decode", "kind": "attend", "dtype": "bf16", "batch": 64, **gqa, "prefix_min": 512,
         "prefix_max": 8192, "nodes_min": 1, "nodes_max": 1, "page": 16, "layout": "heads", "cap": 0.0, "window": 0,
         "sink": 0, "bias": False, "begin": False, "shape_seed": 8},
        # one layer of the long-context step, a document that begins inside the cache
        {"name": "attend_long", "kind": "attend", "dtype": "bf16", "batch": 1, **mha, "prefix_min": 16384,
         "prefix_max": 16384, "nodes_min": 64, "nodes_max": 64, "page": 128, "layout": "heads", "cap": 0.0,
         "window": 0, "sink": 0, "bias": False, "begin": True, "shape_seed": 9},
        # one 26-node tree over a small vocabulary
        {"name": "logits_tree", "kind": "logits", "dtype": "f32", "batch": 1, "nodes_min": 26, "nodes_max": 26,
         "vocab": 32000, "history_min": 1024, "history_max": 1024, "biases": 16, "mask": True, "shape_seed": 2},
        # a ragged batch of eight trees over a large vocabulary, long conversations
        {"name": "logits_serving", "kind": "logits", "dtype": "f32", "batch": 8, "nodes_min": 26, "nodes_max": 64,
         "vocab": 128256, "history_min": 512, "history_max": 8192, "biases": 300, "mask": True, "shape_seed": 5},
        # one request of a two-layer draft model
        {"name": "accept_small", "kind": "accept", "dtype": "f16", "batch": 1, "layers": 2, "kv_heads": 4,
         "head_dim": 64, "prefix_min": 128, "prefix_max": 128, "nodes_min": 26, "nodes_max": 26, "page": 16,
         "layout": "heads", "shape_seed": 3},
        # 64 requests, all layers of a grouped-query model
        {"name": "accept_serving", "kind": "accept", "dtype": "bf16", "batch": 64, "layers": 32, "kv_heads": 8,
         "head_dim": 128, "prefix_min": 32, "prefix_max": 512, "nodes_min": 4, "nodes_max": 64, "page": 16,
         "layout": "heads", "shape_seed": 4},
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
    """One more case of the ranges above: batches of 1 to 1024, prefixes of 1 to
    16384, trees of 1 to 64 nodes, pages of 8 to 256 slots, groups of 1 to 8,
    vocabularies of 1000 to 152064."""
    limits = {}
    for c in listed():
        w = work(c)
        limits.setdefault(c["kind"], []).append((w["bytes"], w["flops"]))
    while True:
        kind = rng.choice(["plan", "store", "attend", "attend", "attend", "attend", "logits", "logits", "accept"])
        c = {"kind": kind, "shape_seed": rng.randint(0, 10**6)}
        c["nodes_min"], c["nodes_max"] = _draw_span(rng, 1, 64)
        page = rng.choice([8, 16, 16, 32, 64, 128, 256])
        layout = rng.choice(["heads", "slots"])
        if kind == "plan":
            lo, hi = _draw_span(rng, 1, 8192)
            c.update(_draw_heads(rng), batch=_log_int(rng, 1, 1024), page=page, prefix_min=lo, prefix_max=hi,
                     prompts=rng.random() < 0.3)
            if c["prompts"]:
                c.update(nodes_min=1, nodes_max=_log_int(rng, 1, 4096))
        elif kind == "store":
            del c["nodes_min"], c["nodes_max"]
            lo, hi = _draw_span(rng, 1, 8192)
            c.update(_draw_heads(rng), batch=_log_int(rng, 1, 64), rows_min=lo, rows_max=hi, page=page, layout=layout,
                     axes=rng.choice([1, 2, 3]), dtype=rng.choice(["bf16", "f16"]))
        elif kind == "attend":
            lo, hi = _draw_span(rng, 1, 16384)
            window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
            c.update(_draw_heads(rng), batch=_log_int(rng, 1, 64), prefix_min=lo, prefix_max=hi, page=page,
                     layout=layout, dtype=rng.choice(["bf16", "f16"]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                     window=window, sink=rng.choice([0, 4, 130]) if window else 0, bias=rng.random() < 0.25,
                     begin=rng.random() < 0.25)
        elif kind == "logits":
            lo, hi = _draw_span(rng, 1, 8192)
            c.update(batch=_log_int(rng, 1, 256), vocab=_log_int(rng, 1000, 152064), history_min=lo, history_max=hi,
                     biases=rng.choice([0, 1, 16, 300]), mask=rng.random() < 0.7, dtype=rng.choice(["f32", "f32", "bf16"]))
        else:
            lo, hi = _draw_span(rng, 1, 512)
            c.update(batch=_log_int(rng, 1, 64), layers=_log_int(rng, 1, 32), kv_heads=rng.choice([1, 4, 8, 32]),
                     head_dim=rng.choice([64, 128]), prefix_min=lo, prefix_max=hi, page=page, layout=layout,
                     dtype=rng.choice(["bf16", "f16"]))
        if _plain_cost(c) <= max(_plain_cost(x) for x in listed() if x["kind"] == kind):
            w = work(c)
            if any(w["bytes"] <= b and w["flops"] <= f for b, f in limits[kind]):
                return c


def _plain_cost(case):
    """Elements that a pass in the plain form goes through, a padded batch where it pads one."""
    kind, B = case["kind"], case["batch"]
    if kind == "plan":
        return B * case["nodes_max"] + B * case["prefix_max"] / case["page"]
    if kind == "store":
        return B * case["rows_max"] * (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
    if kind == "attend":
        S = case["prefix_max"] + case["nodes_max"]
        return B * S * (case["kv_heads"] * case["head_dim"] + case["q_heads"] * case["nodes_max"])
    if kind == "logits":
        return B * case["nodes_max"] * case["vocab"]
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
    """The ragged sizes of a case: prefix lengths, the trees and which request has
    which, and what else its kind needs."""
    r = random.Random(case["shape_seed"])
    B = case["batch"]
    s = {}
    if "nodes_min" in case and not case.get("prompts"):
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
    elif case.get("prompts"):
        s["n"] = [_log_int(r, case["nodes_min"], case["nodes_max"]) if r.random() < 0.9 else 0 for _ in range(B)]
    if "rows_min" in case:
        s["n"] = [r.randint(case["rows_min"], case["rows_max"]) for _ in range(B)]
    if "prefix_min" in case:
        s["L"] = [r.randint(case["prefix_min"], case["prefix_max"]) for _ in range(B)]
    if case["kind"] == "plan":
        s["held"] = []
        for b in range(B):
            u, P = r.random(), case["page"]
            s["held"].append(-(-s["L"][b] // P) + r.randint(0, -(-64 // P)))  # what the last step held
            if B > 1 and u < 0.1:  # finished: its pages go back
                s["L"][b] = s["n"][b] = 0
            elif B > 1 and u < 0.2:  # waiting
                s["n"][b] = 0
            if s["n"][b] == 0 and "tree" in s:
                s["tree"][b] = -1
    if case["kind"] == "attend":
        s["begin"] = [r.randint(0, L) // 2 if case["begin"] else 0 for L in s["L"]]
    if case["kind"] == "logits":
        s["history"] = [r.randint(case["history_min"], case["history_max"]) for _ in range(B)]
        s["prompt"] = [r.randint(0, h) for h in s["history"]]
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


def _tile_keys(case, s):
    """Keys that some row of each request may see."""
    total = []
    for L, n, b0 in zip(s["L"], s["n"], s["begin"]):
        lo = max(b0, L - case["window"] + 1) if case["window"] else b0
        total.append(L + n - lo + max(0, min(b0 + case["sink"], lo) - b0))
    return total


def work(case):
    s, kind = _shape(case), case["kind"]
    R = sum(s["n"])
    if kind == "plan":
        P = case["page"]
        pages = sum(abs(-(-(L + n) // P) - h) for L, n, h in zip(s["L"], s["n"], s["held"]))
        used = sum((L + n - 1) // P - L // P + 1 for L, n in zip(s["L"], s["n"]) if n)
        return {"bytes": 20.0 * case["batch"] + 8.0 * pages + 4.0 * used + 12.0 * R, "flops": 0.0}
    if kind == "store":
        d = case["head_dim"]
        heads = case["q_heads"] + 2 * case["kv_heads"]
        return {"bytes": R * (4.0 * heads * d + 8 + 4 * case["axes"]), "flops": 3.0 * R * d * (heads - case["kv_heads"])}
    if kind == "attend":
        keys, d = _tile_keys(case, s), case["head_dim"]
        return {"bytes": sum(4.0 * k * case["kv_heads"] * d for k in keys) + 4.0 * R * case["q_heads"] * d,
                "flops": sum(4.0 * k * n for k, n in zip(keys, s["n"])) * case["q_heads"] * d}
    if kind == "logits":
        size = 4 if case["dtype"] == "f32" else 2
        V = case["vocab"]
        return {"bytes": R * V * (size + 4 + (0.125 if case["mask"] else 0)) + 4.0 * sum(s["history"]) + 24.0 * R,
                "flops": 8.0 * R * V}
    moved = sum(sum(i != p for i, p in enumerate(_path(s["trees"][t], u))) for t, u in zip(s["tree"], s["last"]))
    row = case["layers"] * case["kv_heads"] * case["head_dim"] * 4.0
    return {"bytes": 2 * row * moved + 8.0 * R + 400.0 * case["batch"], "flops": 0.0}


# ---------------------------------------------------------------- inputs

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


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


def _pool(case, n_pages, g, layers=1):
    """K and V pages [layers][pages][kv heads][slots][d], stored with heads or slots outermost in a page."""
    H, P, d, dt = case["kv_heads"], case["page"], case["head_dim"], DTYPES[case["dtype"]]
    if case["layout"] == "heads":
        return [_normal((layers, n_pages, H, P, d), g, dt) for _ in range(2)]
    return [_normal((layers, n_pages, P, H, d), g, dt).transpose(2, 3) for _ in range(2)]


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
    if "L" in s:
        st["L"] = _ints(s["L"])
    st["row_start"] = _ints(_starts(s["n"]))
    {"plan": _prepare_plan, "store": _prepare_store, "attend": _prepare_attend, "logits": _prepare_logits,
     "accept": _prepare_accept}[kind](case, s, st, g, r)
    if own:
        import paper_2606_27550_gb300 as tv

        st["tv"] = tv
        if "trees" in s:
            st["bank"] = tv.Bank(len(s["trees"]), torch.cuda.current_device())
            for t in s["trees"]:
                st["bank"].add(t)
        if "table" in st:
            st["req"] = tv.Requests(lens=st["L"], table=st["table"], page_size=case["page"],
                                    row_start=st["row_start"], tree=st.get("tree"), n_new=st.get("n_new"),
                                    key_begin=st.get("begin"))
        if kind == "plan":
            st["plan"] = tv.make_paged_plan(case["batch"])
            st["pool"] = tv.PagePool(ring=st["ring"], state=st["ring_state"], held=st["held"],
                                     state_out=st["state_out"], held_out=st["held_out"])
        if kind == "attend":
            # as for the first layer of a step: the same plan serves every layer
            st["plan"] = tv.make_paged_plan(case["batch"])
            tv.paged_plan(st["bank"], st["req"], st["slots"], st["positions"], st["status"], st["plan"],
                          n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"], window=case["window"],
                          sink=case["sink"])
            st["ws"] = tv.make_workspace(tv.tb_workspace_size(1, 1, case["kv_heads"], case["q_heads"],
                                                              case["head_dim"], 1, torch.cuda.current_device()))
        if kind == "logits":
            st["req"] = tv.Requests(row_start=st["row_start"], tree=st["tree"])
            st["ws"] = tv.make_workspace(tv.tb_logits_workspace_size(case["batch"], st["R"], case["vocab"]))
    return st


def _row_arrays(st, rows):
    st["slots"] = torch.zeros(rows, dtype=torch.int64, device="cuda")
    st["positions"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    st["status"] = torch.zeros(st["case"]["batch"], dtype=torch.int32, device="cuda")


def _prepare_plan(case, s, st, g, r):
    P, B = case["page"], case["batch"]
    need = [-(-(L + n) // P) for L, n in zip(s["L"], s["n"])]
    free = sum(max(0, a - h) for a, h in zip(need, s["held"])) + 7
    width = max(max(need), max(s["held"])) + 1
    n_pages = sum(s["held"]) + free
    ids = list(range(n_pages))
    r.shuffle(ids)
    table = np.full((B, width), -1, dtype=np.int32)
    at = 0
    for b, h in enumerate(s["held"]):
        table[b, :h] = ids[at:at + h]
        at += h
    head = r.randrange(n_pages)
    ring = np.full(n_pages, -1, dtype=np.int32)
    ring[(head + np.arange(free)) % n_pages] = ids[at:]
    st.update(table=torch.from_numpy(table).cuda(), ring=torch.from_numpy(ring).cuda(), held=_ints(s["held"]),
              ring_state=_ints([head, free]), held_out=_ints([0] * B), state_out=_ints([0, 0]),
              rows=st["R"] + 5)
    if "tree" not in st:
        st["n_new"] = _ints(s["n"])
    st["row_start"] = torch.zeros_like(st["row_start"])  # the call's to write
    _row_arrays(st, st["rows"])


def _prepare_store(case, s, st, g, r):
    R, d, P, H, Hq = st["R"], case["head_dim"], case["page"], case["kv_heads"], case["q_heads"]
    table, n_pages = _tables(case, s["n"], r)
    owner, place = _rows_of(s["n"])
    page = table.long()[owner, place // P]
    st["slots"] = page * P + place % P
    st["k_pages"], st["v_pages"] = _pool(case, n_pages, g)
    # the projection's output, as a model has it: q, k and v side by side
    qkv = _normal((R, Hq + 2 * H, d), g, DTYPES[case["dtype"]])
    st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    st["q_out"] = torch.empty((R, Hq, d), dtype=qkv.dtype, device="cuda")
    axes = [torch.randint(0, m, (R,), generator=g, device="cuda", dtype=torch.int32) for m in (100000, 256, 256)]
    st["positions"] = torch.stack(axes[:case["axes"]]).contiguous()
    half = d // 2
    st["sections"] = {1: (half,), 2: (half // 2, half - half // 2),
                      3: (half // 4, half * 3 // 8, half - half // 4 - half * 3 // 8)}[case["axes"]]
    # cos and sin are computed from the frequencies in the call: positions are new in every step
    inv = THETA ** (-2.0 * np.arange(half) / d)
    st["freq"] = torch.from_numpy(inv).cuda()
    st["axis"] = _ints([a for a, n in enumerate(st["sections"]) for _ in range(n)], torch.int64)


def _prepare_attend(case, s, st, g, r):
    d, dt = case["head_dim"], DTYPES[case["dtype"]]
    st["table"], n_pages = _tables(case, [L + n for L, n in zip(s["L"], s["n"])], r)
    st["k_pages"], st["v_pages"] = _pool(case, n_pages, g)
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
    _row_arrays(st, st["R"])


def _prepare_logits(case, s, st, g, r):
    B, V, R = case["batch"], case["vocab"], st["R"]
    z = _normal((R, V), g, torch.float32, 2.5)
    likely = torch.randint(0, V, (R,), generator=g, device="cuda")
    z[torch.arange(R, device="cuda"), likely] += 12.0 * torch.rand(R, generator=g, device="cuda")
    st["logits"] = z.to(DTYPES[case["dtype"]])
    st["out"] = torch.empty((R, V), dtype=torch.float32, device="cuda")
    # words of a text: a few of them often
    width = max(s["history"])
    st["history"] = (V * torch.rand((B, width), generator=g, device="cuda") ** 4).int().clamp_(max=V - 1)
    st["history_len"], st["prompt_len"] = _ints(s["history"]), _ints(s["prompt"])
    st["draft"] = (V * torch.rand(R, generator=g, device="cuda") ** 4).int().clamp_(max=V - 1)
    u = torch.rand((3, B), generator=g, device="cuda")
    st["repetition"], st["presence"], st["frequency"] = 1.0 + 0.5 * u[0], 0.8 * u[1], 0.4 * u[2]
    n = case["biases"]
    st["bias_start"] = _ints([b * n for b in range(B + 1)])
    st["bias_token"] = torch.rand((B, V), generator=g, device="cuda").argsort(1)[:, :n].int().reshape(-1).contiguous()
    st["bias_value"] = 4.0 * torch.randn(B * n, generator=g, device="cuda")
    if case["mask"]:
        words = -(-V // 32)
        bits = torch.randint(-2**31, 2**31, (R, words), generator=g, device="cuda", dtype=torch.int64)
        bits |= torch.randint(-2**31, 2**31, (R, words), generator=g, device="cuda", dtype=torch.int64)
        st["mask"] = bits.int()
    st["temperature"] = TEMPERATURE
    st["owner"], st["place"] = _rows_of(s["n"])
    st["argmax"] = torch.empty(R, dtype=torch.int32, device="cuda")
    for name in ("top1", "entropy", "logz_t", "entropy_t", "draft_logit"):
        st[name] = torch.zeros(R, dtype=torch.float32, device="cuda")


def _prepare_accept(case, s, st, g, r):
    B = case["batch"]
    st["table"], n_pages = _tables(case, [L + n for L, n in zip(s["L"], s["n"])], r)
    st["k_pages"], st["v_pages"] = _pool(case, n_pages, g, case["layers"])
    vocab = st["vocab"] = 32000
    draft, argmax = [], []
    for b in range(B):
        tree = s["trees"][s["tree"][b]]
        path = _path(tree, s["last"][b])
        tokens = r.sample(range(vocab - 1), len(tree))
        then = {u: tokens[v] for u, v in zip(path, path[1:])}
        draft += tokens
        argmax += [then.get(u, vocab - 1) for u in range(len(tree))]
    st["draft"], st["argmax"] = _ints(draft), _ints(argmax)
    st["results"] = torch.zeros((B, 4 + NODES), dtype=torch.int32, device="cuda")
    st["lens_out"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    st["depth"] = max(max(_depths(t)) for t in s["trees"]) + 1


# ---------------------------------------------------------------- one pass


def run(st):
    return {"plan": _plan, "store": _store, "attend": _attend, "logits": _logits, "accept": _accept}[st["case"]["kind"]](st)


def _plan(st):
    case = st["case"]
    out = {k: st[k] for k in ("row_start", "slots", "positions", "status", "held_out", "state_out", "ring", "table")}
    if own:
        st["tv"].paged_plan(st.get("bank"), st["req"], st["slots"], st["positions"], st["status"], st["plan"],
                            pool=st["pool"], n_q_heads=case["q_heads"] if "tree" in st else 0,
                            n_kv_heads=case["kv_heads"])
        return out
    P, L, held, table, ring = case["page"], st["L"].long(), st["held"].long(), st["table"], st["ring"]
    n_pages = ring.numel()
    if "tree" in st:
        sizes = (st["tables"]["anc"].any(2)).sum(1)
        n = torch.where(st["tree"] >= 0, sizes[st["tree"].long().clamp(min=0)], 0)
    else:
        n = st["n_new"].long()
    need = (L + n + P - 1) // P
    take, give = (need - held).clamp(min=0), (held - need).clamp(min=0)
    take_at, give_at = take.cumsum(0) - take, give.cumsum(0) - give
    head, count = st["ring_state"].long()
    column = torch.arange(table.shape[1], device=table.device)
    taken = (column >= held[:, None]) & (column < need[:, None])
    given = (column >= need[:, None]) & (column < held[:, None])
    fresh = ring[(head + take_at[:, None] + column - held[:, None]) % n_pages].long()
    table.copy_(torch.where(taken, fresh, table))  # entries past what a request holds keep what they had
    to = (head + count + give_at[:, None] + column - need[:, None]) % n_pages
    at = torch.where(given, to, n_pages).reshape(-1)
    ring.copy_(torch.cat([ring, ring[:1]]).scatter(0, at, torch.where(given, table, 0).reshape(-1))[:n_pages])
    st["held_out"].copy_(need)
    st["state_out"].copy_(torch.stack([(head + take.sum()) % n_pages, count - take.sum() + give.sum()]))
    st["row_start"][1:] = n.cumsum(0)
    row = torch.arange(st["rows"], device=table.device)
    b = torch.searchsorted(st["row_start"][1:].long(), row, right=True).clamp(max=case["batch"] - 1)
    i = row - st["row_start"].long()[b]
    real = row < st["row_start"][-1]
    slot = L[b] + i
    page = table.long()[b, (slot // P).clamp(max=table.shape[1] - 1)]
    st["slots"].copy_(torch.where(real, page * P + slot % P, -1))
    step = st["tables"]["dep"][st["tree"].long()[b].clamp(min=0), i.clamp(0, NODES - 1)] if "tree" in st else i
    st["positions"].copy_(torch.where(real, L[b] + step, 0))
    st["status"].zero_()
    return out


def _turn(x, cos, sin):
    x = x.float()
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _store(st):
    case = st["case"]
    out = {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if own:
        tv = st["tv"]
        tv.paged_kv_store(tv.Pages(st["k_pages"], st["v_pages"]), st["slots"], st["k"], st["v"], q=st["q"],
                          q_out=st["q_out"], positions=st["positions"], sections=st["sections"], rope_theta=THETA)
        return out
    P = case["page"]
    # angles past a few turns lose their fraction in 32 bits: this product is taken in 64
    angle = st["positions"].T[:, st["axis"]].double() * st["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    st["q_out"].copy_(_turn(st["q"], cos, sin))
    page, at = st["slots"] // P, st["slots"] % P
    st["k_pages"][0].transpose(1, 2)[page, at] = _turn(st["k"], cos, sin).to(st["k_pages"].dtype)
    st["v_pages"][0].transpose(1, 2)[page, at] = st["v"]
    return out


def _attend(st):
    case = st["case"]
    if own:
        tv = st["tv"]
        tv.paged_tree_attention(st["bank"], st["req"], tv.Pages(st["k_pages"], st["v_pages"]), st["plan"], st["q"],
                                st["out"], st["ws"], softcap=case["cap"], slopes=st.get("slopes"), lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    P, B, S, N = case["page"], case["batch"], st["keys"], st["width"]
    H, Hq, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    G, L = Hq // H, st["L"].long()
    slot = torch.arange(S, device="cuda")
    page = st["table"].long()[:, slot // P].clamp(min=0)
    k = st["k_pages"][0].transpose(1, 2)[page, slot % P].float()  # [B, S, H, d]
    v = st["v_pages"][0].transpose(1, 2)[page, slot % P].float()
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


LOGIT_OUTPUTS = ("argmax", "top1", "entropy", "logz_t", "entropy_t", "draft_logit")


def _logits(st):
    case = st["case"]
    if own:
        st["tv"].logits_process(st["bank"], st["req"], st["logits"], st["out"], st["ws"], draft=st["draft"],
                                history=st["history"], history_len=st["history_len"], prompt_len=st["prompt_len"],
                                repetition=st["repetition"], presence=st["presence"], frequency=st["frequency"],
                                bias_start=st["bias_start"], bias_token=st["bias_token"], bias_value=st["bias_value"],
                                mask=st.get("mask"), temperature=st["temperature"],
                                **{k: st[k] for k in LOGIT_OUTPUTS})
        return {"out": st["out"], **{k: st[k] for k in LOGIT_OUTPUTS}}
    B, V, R = case["batch"], case["vocab"], st["R"]
    owner, place = st["owner"], st["place"]
    at = torch.arange(st["history"].shape[1], device="cuda")
    h = st["history"].long()
    live = (at < st["history_len"][:, None])
    said = live & (at >= st["prompt_len"][:, None])
    zeros = torch.zeros((B, V), dtype=torch.int32, device="cuda")
    seen = zeros.scatter_add(1, h, live.int())
    made = zeros.scatter_add(1, h, said.int())
    t = st["tree"].long()[owner]
    anc = st["tables"]["anc"][t, place].clone()                  # [R, 64]
    anc[:, 0] = False                                            # the root is in the history
    first = st["row_start"].long()[owner]
    node = torch.arange(NODES, device="cuda")
    token = st["draft"].long()[(first[:, None] + node).clamp(max=R - 1)]
    path = torch.zeros((R, V), dtype=torch.int32, device="cuda").scatter_add(1, token, anc.int())
    count = made[owner] + path
    z = st["logits"].float()
    rep = st["repetition"][owner][:, None]
    z = torch.where(seen[owner] + path > 0, torch.where(z > 0, z / rep, z * rep), z)
    z = z - st["frequency"][owner][:, None] * count
    z = z - st["presence"][owner][:, None] * (count > 0)
    n = case["biases"]
    bias = torch.zeros((B, V), dtype=torch.float32, device="cuda")
    bias.scatter_(1, st["bias_token"].long().view(B, n), st["bias_value"].view(B, n))
    z = z + bias[owner]
    if "mask" in st:
        bit = torch.arange(V, device="cuda")
        z = torch.where((st["mask"][:, bit // 32] >> (bit % 32)) & 1 > 0, z, NEG)
    st["out"].copy_(z)
    m, a = z.max(1)
    st["argmax"].copy_(torch.where(m == NEG, -1, (z == m[:, None]).int().argmax(1)))
    st["top1"].copy_(_softmax_stats(z, m, 1.0)[2])
    st["entropy"].copy_(_softmax_stats(z, m, 1.0)[1])
    logz, ent, _ = _softmax_stats(z, m, st["temperature"])
    st["logz_t"].copy_(logz)
    st["entropy_t"].copy_(ent)
    parent = st["tables"]["par"][t, place]
    st["draft_logit"].copy_(torch.where(parent >= 0, z[first + parent.clamp(min=0), st["draft"].long()], 0.0))
    return {"out": st["out"], **{k: st[k] for k in LOGIT_OUTPUTS}}


def _softmax_stats(z, m, T):
    """ln sum e^(z/T), the entropy and the largest probability of softmax(z / T)."""
    x = (z - m[:, None]) / T
    e = torch.exp(x)
    s = e.sum(1)
    ent = torch.log(s) - torch.where(e > 0, e * x, 0.0).sum(1) / s
    return m / T + torch.log(s), ent, 1.0 / s


def _accept(st):
    case = st["case"]
    out = {"results": st["results"], "lens": st["lens_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    if own:
        tv = st["tv"]
        tv.paged_accept(st["bank"], st["req"], tv.Pages(st["k_pages"], st["v_pages"]), st["results"],
                        draft=st["draft"], argmax=st["argmax"], vocab=st["vocab"], lens_out=st["lens_out"])
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
        flat = pool.transpose(2, 3)                               # [layers, pages, slots, heads, d]
        flat[:, to_page, to % P] = flat[:, src_page, src % P]
    return out


# ---------------------------------------------------------------- the same from the definitions, in 64 bits


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None  # whole numbers
    plain = _plain_state(case, seed)
    return {"store": _exact_store, "attend": _exact_attend, "logits": _exact_logits, "accept": _exact_accept}[kind](
        case, _shape(case), plain)


def _plain_state(case, seed):
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def _exact_store(case, s, st):
    d, P = case["head_dim"], case["page"]
    half = d // 2
    pos = st["positions"].double()
    q, k = st["q"].double(), st["k"].double()
    out_q, out_k = torch.empty_like(q), torch.empty_like(k)
    i = 0
    for axis, n in enumerate(st["sections"]):
        for _ in range(n):
            a = pos[axis] * THETA ** (-2.0 * i / d)
            c, n_ = torch.cos(a)[:, None], torch.sin(a)[:, None]
            for x, y in ((q, out_q), (k, out_k)):
                y[:, :, i] = x[:, :, i] * c - x[:, :, i + half] * n_
                y[:, :, i + half] = x[:, :, i] * n_ + x[:, :, i + half] * c
            i += 1
    kp, vp = st["k_pages"].double(), st["v_pages"].double()
    page, at = st["slots"] // P, st["slots"] % P
    kp[0][page, :, at] = out_k
    vp[0][page, :, at] = st["v"].double()
    return {"q": out_q, "k_pages": kp, "v_pages": vp}


def _exact_attend(case, s, st):
    if _plain_cost(case) > 4e9:
        return None
    P, H, Hq, d = case["page"], case["kv_heads"], case["q_heads"], case["head_dim"]
    outs, lses = [], []
    at = 0
    table = st["table"].tolist()
    for b, (L, n) in enumerate(zip(s["L"], s["n"])):
        tree = s["trees"][s["tree"][b]]
        dep = _depths(tree)
        slots = range(L + n)
        pages = _ints([table[b][x // P] for x in slots], torch.int64)
        inner = _ints([x % P for x in slots], torch.int64)
        k = st["k_pages"][0][pages, :, inner].double()
        v = st["v_pages"][0][pages, :, inner].double()
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


def _exact_logits(case, s, st):
    V, at = case["vocab"], 0
    outs = []
    draft = st["draft"].tolist()
    history = st["history"].cpu().numpy()
    pen = {k: st[k].double().tolist() for k in ("repetition", "presence", "frequency")}
    stats = {k: [] for k in ("top1", "entropy", "logz_t", "entropy_t")}
    edges = []
    for b, n in enumerate(s["n"]):
        tree = s["trees"][s["tree"][b]]
        words = history[b, :s["history"][b]]
        all_n = np.bincount(words, minlength=V)
        out_n = np.bincount(words[s["prompt"][b]:], minlength=V)
        lo, hi = b * case["biases"], (b + 1) * case["biases"]
        bias = torch.zeros(V, dtype=torch.float64, device="cuda")
        bias[st["bias_token"][lo:hi].long()] = st["bias_value"][lo:hi].double()
        z = st["logits"][at:at + n].double()
        extra = np.zeros((n, V), dtype=np.int64)
        for i in range(n):
            for u in _path(tree, i)[1:]:
                extra[i, draft[at + u]] += 1
        any_n = torch.from_numpy(all_n + extra).cuda()
        count = torch.from_numpy(out_n + extra).cuda()
        f = torch.where(z > 0, torch.full_like(z, 1 / pen["repetition"][b]), torch.full_like(z, pen["repetition"][b]))
        z = torch.where(any_n > 0, z * f, z)
        z = z - pen["frequency"][b] * count - pen["presence"][b] * (count > 0) + bias
        if "mask" in st:
            w = st["mask"][at:at + n].cpu().numpy().view(np.uint32)
            ok = np.unpackbits(w.view(np.uint8), axis=1, bitorder="little")[:, :V]
            z = z.masked_fill(~torch.from_numpy(ok.astype(bool)).cuda(), NEG)
        for T, names in ((1.0, ("top1", "entropy")), (st["temperature"], ("logz_t", "entropy_t"))):
            lp = torch.log_softmax(z / T, 1)
            p = lp.exp()
            e = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
            stats[names[0]].append(p.amax(1) if T == 1.0 else torch.logsumexp(z / T, 1))
            stats[names[1]].append(e)
        edges += [0.0] + [float(z[tree[j], draft[at + j]]) for j in range(1, n)]
        outs.append(z)
        at += n
    return {"out": torch.cat(outs), "argmax": None, "draft_logit": torch.tensor(edges, dtype=torch.float64),
            **{k: torch.cat(v) for k, v in stats.items()}}


def _exact_accept(case, s, st):
    P, table = case["page"], st["table"].tolist()
    for pool in (st["k_pages"], st["v_pages"]):
        for b in range(case["batch"]):
            L = s["L"][b]
            path = _path(s["trees"][s["tree"][b]], s["last"][b])
            for j, u in enumerate(path):
                if j != u:
                    pool[:, table[b][(L + j) // P], :, (L + j) % P] = pool[:, table[b][(L + u) // P], :, (L + u) % P]
    return {"results": None, "lens": None, "k_pages": st["k_pages"], "v_pages": st["v_pages"]}

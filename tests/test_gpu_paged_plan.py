"""paged_plan against the sequential reference: block tables, slots, positions,
the ring of free pages, refusals per request, in place and not."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2606_27550_gb300 as tv
from paper_2606_27550_gb300 import synth

pytestmark = pytest.mark.gpu


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def scene(seed, B, page, prompts=False, n_free=None, lens_max=700):
    """A batch in mid-flight: requests that grow, wait, shrink or end."""
    g = synth.rng(seed)
    all_trees = ref.trees()
    lens = [int(g.integers(0, lens_max)) for _ in range(B)]
    tree = [int(g.integers(-1, len(all_trees))) for _ in range(B)]
    n = [int(g.integers(0, 300)) if prompts else 0 if t < 0 else len(all_trees[t]) for t in tree]
    held = []
    for b in range(B):
        held.append(max(0, -(-lens[b] // page) + int(g.integers(-2, 4))))
        if not prompts and tree[b] < 0 and g.random() < 0.5:
            lens[b] = 0
    need = [-(-(a + b) // page) for a, b in zip(lens, n)]
    free = sum(max(0, x - h) for x, h in zip(need, held)) + 3 if n_free is None else n_free
    n_pages = sum(held) + free
    ids = g.permutation(n_pages)
    width = max(max(need), max(held)) + 2
    table = np.full((B, width), -7, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    head = int(g.integers(0, n_pages))
    ring = np.full(n_pages, -9, np.int32)
    ring[(head + np.arange(free)) % n_pages] = ids[at:at + free]
    return dict(lens=lens, tree=tree, n=n, held=held, ring=ring, table=table, state=(head, free), page=page)


def run(s, max_rows, prompts=False, in_place=True, bank=None, key_begin=None, pool=True):
    B = len(s["lens"])
    req = tv.Requests(row_start=torch.empty(B + 1, dtype=torch.int32, device="cuda"), lens=dev(s["lens"]),
                      table=dev(s["table"]), page_size=s["page"], tree=None if prompts else dev(s["tree"]),
                      n_new=dev(s["n"]) if prompts else None, key_begin=key_begin)
    p = tv.PagePool(dev(s["ring"]), dev(s["state"]), dev(s["held"]))
    if not in_place:
        p.state_out = torch.empty(2, dtype=torch.int32, device="cuda")
        p.held_out = torch.empty(B, dtype=torch.int32, device="cuda")
    slots = torch.empty(max_rows, dtype=torch.int64, device="cuda")
    positions = torch.empty(max_rows, dtype=torch.int32, device="cuda")
    status = torch.empty(B, dtype=torch.int32, device="cuda")
    plan = tv.make_paged_plan(B)
    tv.paged_plan(bank, req, slots, positions, status, plan, pool=p if pool else None,
                  n_q_heads=0 if prompts else 8, n_kv_heads=4)
    return req, p, slots, positions, status, plan


def check(s, got, max_rows, prompts, in_place, bad=()):
    req, p, slots, positions, status, plan = got
    e_status, row_start, e_slots, at, held, state, ring, table = ref.plan(
        s["lens"], s["n"], s["held"], s["state"], s["ring"], s["table"], s["page"], max_rows, bad)
    assert status.tolist() == e_status
    assert req.row_start.tolist() == row_start.tolist()
    assert slots.tolist() == e_slots.tolist()
    rows = int(row_start[-1])
    depth = [synth.depth_of(t) for t in ref.trees()]
    e_pos = [s["lens"][b] + (i if prompts else int(depth[s["tree"][b]][i])) for b, i in at[:rows]]
    assert positions.tolist() == e_pos + [0] * (max_rows - rows)
    assert (p.held if in_place else p.held_out).tolist() == held
    assert (p.state if in_place else p.state_out).tolist() == list(state)
    assert np.array_equal(p.ring.cpu().numpy(), ring)
    assert np.array_equal(req.table.cpu().numpy(), table)
    if not in_place:
        assert p.held.tolist() == s["held"] and p.state.tolist() == list(s["state"])
    assert int(plan[:4].view(torch.int32)) == 0  # the ticket is left at zero


@pytest.fixture(scope="module")
def bank():
    b = tv.Bank(16, 0)
    for t in ref.trees():
        b.add(t)
    yield b
    b.close()


@pytest.mark.parametrize("seed,B,page,prompts,in_place", [
    (1, 1, 16, False, True), (2, 7, 8, False, True), (3, 64, 16, False, False), (4, 511, 32, False, True),
    (5, 513, 16, False, True), (6, 1300, 64, False, False), (7, 4096, 16, False, True), (8, 3, 1024, False, True),
    (9, 5, 16, True, True), (10, 100, 128, True, False)])
def test_plan(bank, seed, B, page, prompts, in_place):
    s = scene(seed, B, page, prompts)
    max_rows = sum(s["n"]) + 3
    check(s, run(s, max_rows, prompts, in_place, bank), max_rows, prompts, in_place)


def test_requests_that_do_not_fit_get_nothing(bank):
    """Rows past max_rows, an empty ring, unknown trees, too many pages: each is refused alone."""
    s = scene(21, 40, 16)
    s["tree"][3], s["tree"][11] = 99, -5
    s["lens"][17] = -1
    s["lens"][20] = s["table"].shape[1] * 16 + 1
    for b in (3, 11):
        s["n"][b] = 0
    for max_rows in (sum(s["n"]) + 1, sum(s["n"]) // 2, 1):
        for free in (s["state"][1], 5, 0):
            t = dict(s, state=(s["state"][0], free))
            check(t, run(t, max_rows, False, True, bank), max_rows, False, True, bad=(3, 11))


def test_steps_follow_one_another(bank):
    """Twelve steps with lengths that grow and requests that end and begin, on one plan, pool and table: pages stay
    distinct and none is lost."""
    g = synth.rng(33)
    B, page, n_pages = 24, 16, 600
    all_trees = ref.trees()
    pool = tv.make_page_pool(n_pages, B)
    req = tv.Requests(row_start=torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
                      lens=torch.zeros(B, dtype=torch.int32, device="cuda"), page_size=page,
                      table=torch.full((B, 64), -1, dtype=torch.int32, device="cuda"),
                      tree=torch.zeros(B, dtype=torch.int32, device="cuda"))
    slots = torch.empty(B * 64, dtype=torch.int64, device="cuda")
    positions = torch.empty(B * 64, dtype=torch.int32, device="cuda")
    status = torch.empty(B, dtype=torch.int32, device="cuda")
    plan = tv.make_paged_plan(B)
    lens = np.zeros(B, int)
    for step in range(12):
        tree = g.integers(-1, len(all_trees), B)
        ended = (g.random(B) < 0.1) & (step > 0)
        lens[ended], tree[ended] = 0, -1
        lens += np.where(ended, 0, g.integers(0, 40, B))
        req.lens.copy_(dev(lens))
        req.tree.copy_(dev(tree))
        tv.paged_plan(bank, req, slots, positions, status, plan, pool=pool, n_q_heads=8, n_kv_heads=2)
        assert (status == 0).all()
        held, table = pool.held.tolist(), req.table.cpu().numpy()
        mine = [table[b, :h] for b, h in enumerate(held)]
        head, free = pool.state.tolist()
        ring = pool.ring.cpu().numpy()
        everything = np.concatenate([*mine, ring[(head + np.arange(free)) % n_pages]])
        assert sorted(everything.tolist()) == list(range(n_pages))
        n = [0 if t < 0 else len(all_trees[t]) for t in tree]
        assert held == [-(-(a + b) // page) for a, b in zip(lens, n)]


def test_without_a_pool_the_table_is_the_callers(bank):
    s = scene(50, 9, 16)
    need = [-(-(a + b) // 16) for a, b in zip(s["lens"], s["n"])]
    for b, c in enumerate(need):
        s["table"][b, :c] = 1000 * b + np.arange(c)
    s["table"][4, 0] = -1  # a hole
    max_rows = sum(s["n"])
    req, p, slots, positions, status, plan = run(s, max_rows, False, True, bank, pool=False)
    s2 = dict(s, held=need)
    e = ref.plan(s2["lens"], s2["n"], need, s["state"], s["ring"], s["table"], 16, max_rows)
    assert slots.tolist() == e[2].tolist() and status.tolist() == [0] * 9
    assert np.array_equal(req.table.cpu().numpy(), s["table"]) and p.held.tolist() == s["held"]


def test_on_another_stream_and_in_a_graph(bank):
    s = scene(60, 30, 16)
    max_rows = sum(s["n"]) + 1
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = run(s, max_rows, False, False, bank)
    side.synchronize()
    check(s, got, max_rows, False, False)
    req, p, slots, positions, status, plan = got
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tv.paged_plan(bank, req, slots, positions, status, plan, pool=p, n_q_heads=8, n_kv_heads=4)
    slots.zero_()
    graph.replay()
    torch.cuda.synchronize()
    check(s, got, max_rows, False, False)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("free,rows_share", [(None, 1.0), (5, 1.0), (0, 1.0), (5, 0.5), (None, 0.3)])
def test_a_further_plan_of_a_step_serves_the_same_requests(bank, in_place, free, rows_share):
    """Two plans of one step, the ring or the rows running out in the first: the second refuses the same requests,
    takes and gives nothing, and lays the same rows out."""
    s = scene(70, 40, 16)
    s["tree"][3], s["n"][3], s["lens"][17] = 99, 0, -1
    if free is not None:
        s["state"] = (s["state"][0], free)
    max_rows = max(1, int(sum(s["n"]) * rows_share))
    got = run(s, max_rows, False, in_place, bank)
    check(s, got, max_rows, False, in_place, bad=(3,))
    req, p, slots, positions, status, plan = got
    first = [t.clone() for t in (req.row_start, slots, positions, status, req.table, p.ring)]
    held = (p.held if in_place else p.held_out).clone()
    # the reference, with what the requests hold by now and nothing in the ring
    want = ref.plan(s["lens"], s["n"], held.tolist(), (0, 0), p.ring.cpu().numpy(), req.table.cpu().numpy(), 16, max_rows,
                    (3,))
    for t in (req.row_start, slots, positions, status):
        t.fill_(-77)
    other = tv.make_paged_plan(len(s["lens"]))
    tv.paged_plan(bank, req, slots, positions, status, other, pool=p.held_only(), n_q_heads=8, n_kv_heads=4, window=50)
    assert status.tolist() == want[0] and req.row_start.tolist() == want[1].tolist()
    assert slots.tolist() == want[2].tolist()
    for t, was in zip((req.row_start, slots, positions, status, req.table, p.ring), first):
        assert torch.equal(t, was)
    assert torch.equal(p.held if in_place else p.held_out, held) and want[4] == held.tolist()
    if free == 0:
        assert tv.TB_ECAPACITY in status.tolist()

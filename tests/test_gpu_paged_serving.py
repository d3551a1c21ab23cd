"""The example's decode loop over a paged cache, step by step against the
contiguous calls of the library and the 64-bit references."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
import paged_reference as ref
import paper_2606_27550_gb300 as tv
from paper_2606_27550_gb300 import synth

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def cached(server, layer, b, n):
    """K and V of the first n slots of request b, [n][heads][d], as stored."""
    slot = torch.arange(n, device="cuda")
    page = server.req.table[b].long()[slot // server.req.page_size]
    at = slot % server.req.page_size
    return [p[layer].transpose(1, 2)[page, at] for p in (server.pages.k, server.pages.v)]


def test_decode_loop():
    import paged_serving as ex

    server = ex.Server(ex.Model())
    m = server.m
    server.admit({b: list(range(5 * b + 2, 5 * b + 2 + n)) for b, n in enumerate((5, 40, 17, 100))})
    assert server.req.lens.tolist() == [4, 39, 16, 99] and server.status.tolist() == [0] * 4
    accepted = 0
    for step in range(6):
        trees = [(b + step) % 3 for b in range(server.B)]
        if step >= 3:
            trees[2] = -1
        if step == 3:
            server.finish(2)
        draft = ex.drafts(server, trees)
        before, said = server.req.lens.tolist(), server.said.tolist()
        old = {b: [cached(server, layer, b, before[b]) for layer in range(m.layers)] for b in range(server.B)}
        # what the layers' attention was given and gave
        seen = []
        real = tv.paged_tree_attention

        def spy(bank, req, pages, plan, q, out, w, **kw):
            real(bank, req, pages, plan, q, out, w, **kw)
            seen.append((q.clone(), out.clone(), [cached(server, kw["layer"], b, before[b] + (len(server.parents[t]) if t >= 0 else 0))
                                                  for b, t in enumerate(trees)]))

        tv.paged_tree_attention = spy
        try:
            logits, argmax = server.step(torch.tensor(trees, dtype=torch.int32), draft)
        finally:
            tv.paged_tree_attention = real
        torch.cuda.synchronize()
        assert server.status.tolist() == [0] * 4 and tv.tb_workspace_status(server.ws) == 0
        start = server.req.row_start.tolist()
        d = draft.cpu().numpy()
        for b, t in enumerate(trees):
            if t < 0:
                assert start[b] == start[b + 1] and server.results[b, 0] == 0
                continue
            parent, lo = server.parents[t], start[b]
            n = len(parent)
            assert start[b + 1] - lo == n
            for layer, (q, out, kv) in enumerate(seen):
                k, v = kv[b]
                # the prefix as it was, and the formula in 64 bits on the cache as stored
                assert torch.equal(k[:before[b]], old[b][layer][0]) and torch.equal(v[:before[b]], old[b][layer][1])
                o, _, absv, big = ref.attend(q[lo:lo + n].double().cpu().numpy(), k.double().cpu().numpy(),
                                             v.double().cpu().numpy(), parent, before[b], m.d ** -0.5, server.softcap)
                bound = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -21 * big[..., None]) * absv + 1e-7
                assert (np.abs(out[lo:lo + n].double().cpu().numpy() - o) <= bound).all()
            a = argmax[lo:lo + n].cpu().numpy()
            assert np.array_equal(a, logits[lo:lo + n].argmax(1).cpu().numpy())
            k_len, path, bonus = oracle.accept(parent, d[lo:lo + n], a)
            accepted += k_len - 1
            got = server.results[b].tolist()
            assert got[:4] == [k_len, bonus, before[b] + k_len, 0] and got[4:4 + k_len] == list(path)
            assert server.history[b, said[b]:said[b] + k_len].tolist() == [int(d[lo + u]) for u in path[1:]] + [bonus]
            for layer, (q, out, kv) in enumerate(seen):
                after = cached(server, layer, b, before[b] + k_len)
                for x, y in zip(after, kv[b]):
                    assert torch.equal(x[:before[b]], y[:before[b]])
                    assert torch.equal(x[before[b]:], y[before[b]:][torch.tensor(path, device="cuda", dtype=torch.long)])
        assert server.req.lens.tolist() == server.results[:, 2].tolist()
    head, free = server.pool.state.tolist()
    held, table = server.pool.held.tolist(), server.req.table.cpu().numpy()
    ring = server.pool.ring.cpu().numpy()
    everything = np.concatenate([*[table[b, :h] for b, h in enumerate(held)], ring[(head + np.arange(free)) % len(ring)]])
    assert sorted(everything.tolist()) == list(range(len(ring)))
    assert held[2] == 0
    assert accepted > 0  # the guesses are good enough that paths longer than the root come up


@pytest.mark.parametrize("Hq,H,d,L,nodes", [(8, 8, 64, 500, 26), (8, 2, 128, 1300, 40)])
def test_paged_and_contiguous_attention_agree(Hq, H, d, L, nodes):
    """The same cache in pages and in one slab: both kernels within their common bound of each other."""
    torch.manual_seed(L)
    parent = synth.rank_product_tree((4, 3, 2, 2, 2), nodes)
    bank = tv.Bank(2, 0)
    bid, _ = bank.add(parent)
    N, P = len(parent), 16
    k, v = (torch.randn(1, H, L + N, d, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(N, Hq, d, device="cuda").bfloat16()
    want = torch.empty((1, N, Hq, d), dtype=torch.bfloat16, device="cuda")
    ws = tv.make_workspace(tv.tb_workspace_size(64, 1, H, Hq, d, 1, 0))
    tv.tree_attention(bank, bid, tv.KvCache(k, v, L), q[None].contiguous(), want, ws)
    n = -(-(L + N) // P)
    ids = torch.randperm(n + 3, device="cuda")[:n]
    pages = [torch.zeros(1, n + 3, H, P, d, device="cuda").bfloat16() for _ in range(2)]
    slot = torch.arange(L + N, device="cuda")
    for pool, x in zip(pages, (k, v)):
        pool[0].transpose(1, 2)[ids[slot // P], slot % P] = x[0].transpose(0, 1)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    req = tv.Requests(row_start=i32([0, 0]), tree=i32([bid]), lens=i32([L]), table=ids.int()[None].contiguous(), page_size=P)
    plan = tv.make_paged_plan(1)
    tv.paged_plan(bank, req, torch.empty(N, dtype=torch.int64, device="cuda"), i32([0] * N), i32([0]), plan, n_q_heads=Hq,
                  n_kv_heads=H)
    out = torch.empty_like(q)
    tv.paged_tree_attention(bank, req, tv.Pages(*pages), plan, q, out, ws)
    # each within 2^-8 |o| + (2^-8 + 2^-12) A of the exact output, A <= max |v|
    err = (out.float() - want[0].float()).abs()
    lim = 2 * (2.0 ** -8 * want[0].float().abs() + (2.0 ** -8 + 2.0 ** -12) * v.float().abs().max())
    assert bool((err <= lim * 1.01).all())
    # and the same workspace serves both again
    again = torch.empty_like(want)
    tv.tree_attention(bank, bid, tv.KvCache(k, v, L), q[None].contiguous(), again, ws)
    assert torch.equal(again, want)
    bank.close()


def test_sampled_and_typical_rules_take_processed_logits():
    """logits_process feeds the other acceptance rules: its statistics are theirs."""
    torch.manual_seed(5)
    parent = synth.rank_product_tree((3, 2, 1), 8)
    bank = tv.Bank(2, 0)
    bid, _ = bank.add(parent)
    N, V, L, T = len(parent), 700, 33, 0.7
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    req = tv.Requests(row_start=i32([0, N]), tree=i32([bid]))
    logits = 2 * torch.randn(N, V, device="cuda")
    draft = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
    logits[torch.tensor(parent[1:], device="cuda").long(), draft[1:].long()] += 6.0
    ws = tv.make_workspace(tv.tb_logits_workspace_size(1, N, V))
    st = {k: torch.zeros(N, device="cuda") for k in ("top1", "entropy", "logz_t", "entropy_t", "draft_logit")}
    argmax = torch.zeros(N, dtype=torch.int32, device="cuda")
    mask = torch.full((N, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    mask[:, 3] = 0  # tokens 96 .. 127 are not allowed
    out = torch.empty_like(logits)
    tv.logits_process(bank, req, logits, out, ws, draft=draft, mask=mask, temperature=T, argmax=argmax, **st)
    z = out.double().cpu().numpy()
    res = tv.make_result()
    tv.typical_accept(bank, bid, draft, argmax, st["logz_t"], st["entropy_t"], st["draft_logit"], V, L, res, T, 0.09, 0.3)
    k, path, bonus = oracle.typical_accept(parent, draft.cpu().numpy(), z, T, 0.09, 0.3)
    r = tv.parse_result(res)
    assert (r["accept_len"], r["path"], r["bonus_token"]) == (k, list(path), bonus)
    q = torch.softmax(torch.randn(N, V, device="cuda"), 1)
    u = torch.rand(2 * N, device="cuda")
    tv.spec_sample_accept(bank, bid, draft, out, st["logz_t"], q, u, L, T, torch.empty(V, device="cuda"), res)
    r = tv.parse_result(res)
    assert not 96 <= r["bonus_token"] < 128
    assert all(not 96 <= int(draft[j]) < 128 for j in r["path"][1:])
    bank.close()


def test_a_step_without_rows():
    """Requests that all wait or have ended: pages go back, nothing else moves, and no result says "accepted"."""
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    torch.manual_seed(8)
    B, H, Hq, d, P, V = 3, 2, 4, 64, 16, 100
    bank = tv.Bank(2, 0)
    bank.add(synth.chain(3))
    pool = tv.make_page_pool(9, B)
    pages = tv.Pages(torch.randn(2, 9, H, P, d, device="cuda").bfloat16(), torch.randn(2, 9, H, P, d, device="cuda").bfloat16())
    req = tv.Requests(row_start=i32([7] * (B + 1)), tree=i32([0, 0, 0]), lens=i32([20, 30, 5]), table=i32([[-1] * 4] * B),
                      page_size=P)
    status, plan = i32([9] * B), tv.make_paged_plan(B)

    def lay(rows):
        slots, pos = torch.empty(rows, dtype=torch.int64, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
        tv.paged_plan(bank, req, slots, pos, status, plan, pool=pool, n_q_heads=Hq, n_kv_heads=H)
        return slots, pos

    lay(9)
    assert status.tolist() == [0] * 3 and pool.held.tolist() == [2, 3, 1] and pool.state.tolist() == [6, 3]
    req.tree.fill_(-1)
    req.lens[2] = 0
    slots, pos = lay(0)
    assert status.tolist() == [0] * 3 and req.row_start.tolist() == [0] * 4
    assert pool.held.tolist() == [2, 2, 0] and pool.state.tolist() == [6, 5]
    before = [pages.k.clone(), pages.v.clone()]
    kv, q = (torch.empty(0, h, d, dtype=torch.bfloat16, device="cuda") for h in (H, Hq))
    ws = tv.make_workspace(tv.tb_workspace_size(0, 1, H, Hq, d, 0, 0))
    tv.paged_kv_store(pages, slots, kv, kv, layer=1, q=q, q_out=torch.empty_like(q), positions=pos, rope_theta=1e4)
    tv.paged_tree_attention(bank, req, pages, plan, q, torch.empty_like(q), ws, layer=1,
                            lse=torch.empty(0, Hq, device="cuda"))
    z = torch.empty(0, V, device="cuda")
    tv.logits_process(bank, req, z, z, tv.make_workspace(tv.tb_logits_workspace_size(B, 0, V)), draft=pos, argmax=pos)
    results = tv.make_results(B)
    results.fill_(4)
    tv.paged_accept(bank, req, pages, results, draft=pos, argmax=pos, vocab=V)
    torch.cuda.synchronize()
    assert results.tolist() == [[0, -1, L, 0] + [0] * 64 for L in (20, 30, 0)] and req.lens.tolist() == [20, 30, 0]
    assert torch.equal(pages.k, before[0]) and torch.equal(pages.v, before[1])
    assert tv.tb_workspace_status(ws) == tv.TB_OK
    # rows that no request may have, none given room for: refused one by one
    req.tree.fill_(0)
    lay(0)
    assert status.tolist() == [tv.TB_ECAPACITY] * 3 and req.row_start.tolist() == [0] * 4
    assert pool.held.tolist() == [2, 2, 0] and pool.state.tolist() == [6, 5]
    bank.close()


def test_the_example_when_the_pages_run_out():
    """A prompt and a tree that find no room: their requests wait, and the others go on as they would alone."""
    import paged_serving as ex

    model = ex.Model()
    prompts = {b: list(range(5 * b + 2, 5 * b + 2 + n)) for b, n in enumerate((5, 16, 6, 7))}
    small, large = ex.Server(model, n_pages=4), ex.Server(model)
    for server in (small, large):
        assert not server.admit(prompts)
    assert small.pool.state.tolist()[1] == 0
    # request 1 needs two more pages for its tree and there is none; in the other server it waits by itself
    small.step(torch.tensor([1, 2, 1, 0], dtype=torch.int32), ex.drafts(small, [1, 2, 1, 0]))
    large.step(torch.tensor([1, -1, 1, 0], dtype=torch.int32), ex.drafts(large, [1, -1, 1, 0]))
    assert small.status.tolist() == [0, tv.TB_ECAPACITY, 0, 0] and large.status.tolist() == [0] * 4
    assert tv.tb_workspace_status(small.ws) == 0
    for name in ("results", "said", "history"):
        assert torch.equal(getattr(small, name), getattr(large, name)), name
    assert torch.equal(small.req.lens, large.req.lens) and small.req.lens.tolist()[1] == 15
    for layer in range(model.layers):
        for b in (0, 2, 3):
            for x, y in zip(cached(small, layer, b, 8), cached(large, layer, b, 8)):
                assert torch.equal(x[:int(small.req.lens[b])], y[:int(small.req.lens[b])])
    # a prompt that finds no room, and with it the one behind it, which does the next time
    server = ex.Server(model, n_pages=3)
    assert server.admit({0: prompts[0]}) == []
    kept = [cached(server, layer, 0, 5) for layer in range(model.layers)]
    assert server.admit({1: list(range(40)), 2: [9, 3]}) == [1, 2]
    assert server.req.lens.tolist() == [4, 0, 0, 0] and server.pool.held.tolist() == [1, 0, 0, 0]
    assert server.admit({2: [9, 3]}) == []
    assert server.req.lens.tolist() == [4, 0, 1, 0] and server.pool.held.tolist() == [1, 0, 1, 0]
    assert server.said.tolist() == [5, 0, 2, 0]
    for layer in range(model.layers):
        for x, y in zip(cached(server, layer, 0, 5), kept[layer]):
            assert torch.equal(x, y)

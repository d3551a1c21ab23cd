"""The calls over a 4-bit cache together: the example's decode loop step by step
(store, attention, acceptance, and the rows read back), a step over 4 bits beside
one over 16 that hold the same numbers, one captured into a graph, calls from two
threads, and workspaces and streams of their own."""
import os
import sys
import threading

import numpy as np
import pytest
import torch

import oracle
import paged_reference as ref
import paper_2606_27550_gb300 as tv
import q4_reference as q4
from paper_2606_27550_gb300 import synth
from test_gpu_paged_attention import BF, HF, bank, i32  # noqa: F401
from test_gpu_paged_attention_q4 import Scene

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def cached(server, b, n):
    """K and V of the first n slots of request b in every layer, [layers][n][heads][d], as stored."""
    m, P = server.m, server.req.page_size
    slot = torch.arange(n, device="cuda")
    slots = server.req.table[b].long()[slot // P] * P + slot % P
    out = [torch.empty((m.layers, n, m.H, m.d), dtype=BF, device="cuda") for _ in range(2)]
    tv.paged_kv_load_q4(server.pages, slots, *out)
    return out


def test_decode_loop(monkeypatch):
    import paged_serving as ex

    server = ex.Server(ex.Model(), q4=True)
    m = server.m
    assert not server.admit({b: list(range(5 * b + 2, 5 * b + 2 + n)) for b, n in enumerate((5, 40, 17, 100))})
    accepted = 0
    for step in range(6):
        trees = [(b + step) % 3 for b in range(server.B)]
        if step >= 3:
            trees[2] = -1
        if step == 3:
            server.finish(2)
        draft = ex.drafts(server, trees)
        before = server.req.lens.tolist()
        old = [cached(server, b, before[b]) for b in range(server.B)]
        stored, seen = [], []
        real_store, real_attend = tv.paged_kv_store_q4, tv.paged_tree_attention_q4

        def store(pages, slots, k, v, **kw):
            stored.append((k.clone(), v.clone(), kw["q"].clone(), kw["positions"].clone()))
            real_store(pages, slots, k, v, **kw)

        def attend(bank, req, pages, plan, q, out, w, **kw):  # noqa: F811
            real_attend(bank, req, pages, plan, q, out, w, **kw)
            seen.append((q.clone(), out.clone()))

        monkeypatch.setattr(tv, "paged_kv_store_q4", store)
        monkeypatch.setattr(tv, "paged_tree_attention_q4", attend)
        real_accept = tv.paged_accept_q4
        whole = {}

        def accept(*a, **kw):  # the trees' rows before those that were not accepted are overwritten
            whole.update({b: cached(server, b, before[b] + len(server.parents[t])) for b, t in enumerate(trees) if t >= 0})
            real_accept(*a, **kw)

        monkeypatch.setattr(tv, "paged_accept_q4", accept)
        logits, argmax = server.step(torch.tensor(trees, dtype=torch.int32), draft)
        monkeypatch.undo()
        torch.cuda.synchronize()
        assert server.status.tolist() == [0] * 4 and tv.tb_workspace_status(server.ws) == 0
        start, d = server.req.row_start.tolist(), draft.cpu().numpy()
        for b, t in enumerate(trees):
            if t < 0:
                assert start[b] == start[b + 1] and server.results[b, 0] == 0
                continue
            parent, lo, hi = server.parents[t], start[b], start[b + 1]
            n, L = len(parent), before[b]
            assert hi - lo == n
            for layer in range(m.layers):
                k, v = (x[layer] for x in whole[b])
                # the prefix as it was; the new rows are the projection's, normed, turned, in 4 bits
                assert torch.equal(k[:L], old[b][0][layer]) and torch.equal(v[:L], old[b][1][layer])
                ki, vi, qi, pos = (x[lo:hi].float().cpu().numpy() for x in stored[layer])
                turned = [q4.turn(q4.head_norm(x, w[layer].float().cpu().numpy(), 1e-6), pos[None], (m.d // 2,), 10000.0)
                          for x, w in ((ki, m.k_norm), (qi, m.q_norm))]
                for got, x in ((k, turned[0]), (v, vi)):
                    assert np.array_equal(got[L:].double().cpu().numpy(), q4.values(*q4.quantize(x)))
                q, out = seen[layer]
                assert torch.equal(q[lo:hi].cpu(), torch.from_numpy(turned[1]).to(BF))
                # the formula in 64 bits on the cache as stored
                o, _, absv, big = ref.attend(q[lo:hi].double().cpu().numpy(), k.double().cpu().numpy(),
                                             v.double().cpu().numpy(), parent, L, m.d ** -0.5, server.softcap)
                bound = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -21 * big[..., None]) * absv + 1e-7
                assert (np.abs(out[lo:hi].double().cpu().numpy() - o) <= bound).all()
            k_len, path, bonus = oracle.accept(parent, d[lo:hi], argmax[lo:hi].cpu().numpy())
            accepted += k_len - 1
            got = server.results[b].tolist()
            assert got[:4] == [k_len, bonus, L + k_len, 0] and got[4:4 + k_len] == list(path)
            after = cached(server, b, L + k_len)
            keep = torch.tensor([*range(L), *(L + u for u in path)], device="cuda")
            assert all(torch.equal(x, y[:, keep]) for x, y in zip(after, whole[b]))
        assert server.req.lens.tolist() == server.results[:, 2].tolist()
    assert accepted > 0


@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
@pytest.mark.parametrize("tree", [(7, 5, 0, 2), (0, 0, 1, 0)])
def test_the_same_numbers_in_16_bits(bank, d, dtype, tree):  # noqa: F811
    """A cache of 16 bits that holds what the 4 bits stand for gives the same attention: each side is within the
    bound of the formula's value."""
    s = Scene(33, [500, 3000, 64, 129], list(tree), 8, 2, d, 16, dtype=dtype)
    out, _ = s.run(bank)
    _, n_pages, H, _ = s.pages.k.shape
    slots = torch.arange(n_pages * 16, device="cuda")
    rows = [torch.empty((n_pages * 16, H, d), dtype=dtype, device="cuda") for _ in range(2)]
    tv.paged_kv_load_q4(s.pages, slots, *rows)
    pages = tv.Pages(*(x.view(1, n_pages, 16, H, d).transpose(2, 3) for x in rows))
    out16 = torch.empty_like(s.out)
    tv.paged_tree_attention(bank, s.req, pages, s.plan, s.q, out16, s.ws)
    torch.cuda.synchronize()
    eps = 2.0 ** -8 if dtype == BF else 2.0 ** -11
    at = 0
    for b, n in enumerate(s.n):
        o, _, absv, big = ref.attend(s.q[at:at + n].double().cpu().numpy(), *s.dense[b], s.trees[s.tree[b]], s.lens[b],
                                     d ** -0.5)
        bound = eps * np.abs(o) + (eps + 2.0 ** -12 + 2.0 ** -21 * big[..., None]) * absv + 1e-7
        assert (np.abs(out[at:at + n] - out16[at:at + n].double().cpu().numpy()) <= 2 * bound).all()
        at += n


def test_a_captured_step_replayed_over_growing_lengths(bank):  # noqa: F811
    """Plan, store, attention and acceptance in one graph; each replay goes on from the lengths that the last one left,
    as the same calls do one by one on a second cache."""
    torch.manual_seed(12)
    B, Hq, H, d, P, V, R, n_pages = 3, 4, 2, 64, 8, 50, 3 * 26, 60
    qkv = torch.randn(R, Hq + 2 * H, d, device="cuda").bfloat16()
    w = torch.rand(d, device="cuda").bfloat16()
    draft = torch.randint(0, 3, (R,), device="cuda", dtype=torch.int32)
    argmax = torch.randint(0, 3, (R,), device="cuda", dtype=torch.int32)

    class Side:
        def __init__(self):
            self.pages = tv.make_pages_q4(1, n_pages, H, P, d, BF)
            self.pool = tv.make_page_pool(n_pages, B)
            self.req = tv.Requests(row_start=i32([0] * (B + 1)), tree=i32([5, 2, 0]), lens=i32([0, 5, 17]),
                                   table=i32([[0] * 20] * B), page_size=P)
            self.slots, self.pos = torch.zeros(R, dtype=torch.int64, device="cuda"), i32([0] * R)
            self.status, self.plan = i32([0] * B), tv.make_paged_plan(B)
            self.ws = tv.make_workspace(tv.tb_workspace_size(0, 1, H, Hq, d, 0, 0))
            self.q, self.out = (torch.zeros(R, Hq, d, dtype=BF, device="cuda") for _ in range(2))
            self.results = tv.make_results(B)

        def step(self):
            tv.paged_plan(bank, self.req, self.slots, self.pos, self.status, self.plan, pool=self.pool, n_q_heads=Hq,
                          n_kv_heads=H)
            tv.paged_kv_store_q4(self.pages, self.slots, qkv[:, Hq:Hq + H], qkv[:, Hq + H:], q=qkv[:, :Hq], q_out=self.q,
                                 q_norm=w, k_norm=w, positions=self.pos, rope_theta=1e4)
            tv.paged_tree_attention_q4(bank, self.req, self.pages, self.plan, self.q, self.out, self.ws)
            tv.paged_accept_q4(bank, self.req, self.pages, self.results, draft=draft, argmax=argmax, vocab=V)

    one, two = Side(), Side()
    one.step()
    two.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.step()
    for _ in range(5):
        one.step()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((one.out, two.out), (one.results, two.results), (one.req.lens, two.req.lens),
                     (one.pages.k, two.pages.k), (one.pages.v, two.pages.v), (one.pool.held, two.pool.held)):
            assert torch.equal(x, y)
        assert tv.tb_workspace_status(two.ws) == 0 and two.status.tolist() == [0] * B
    assert one.req.lens[0] > 5


def test_two_threads_on_two_streams(bank):  # noqa: F811
    """Two calls at once, each with its own workspace and stream: what each gives alone."""
    scenes = [Scene(50 + i, [4000 - 900 * i, 20, 300], [[7, 0, 2], [0, 1, 0]][i], 8, 2, 128, 16) for i in range(2)]
    for s in scenes:
        s.run(bank)
        s.want = [s.out.clone(), s.lse.clone()]
    torch.cuda.synchronize()
    failed = []

    def work(s):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    s.out.zero_(), s.lse.zero_()
                    s.call()
                    torch.cuda.current_stream().synchronize()
                    if not (torch.equal(s.out, s.want[0]) and torch.equal(s.lse, s.want[1])):
                        failed.append(s)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in scenes]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_a_step_without_rows(bank):  # noqa: F811
    """Requests that all wait: nothing is written, nothing moves."""
    B, H, Hq, d, P = 3, 2, 4, 64, 16
    pages = tv.make_pages_q4(2, 9, H, P, d, BF)
    pages.k.random_(0, 200), pages.v.random_(0, 200)
    before = [pages.k.clone(), pages.v.clone()]
    req = tv.Requests(row_start=i32([7] * (B + 1)), tree=i32([-1] * B), lens=i32([20, 30, 0]), table=i32([[0] * 4] * B),
                      page_size=P)
    status, plan = i32([9] * B), tv.make_paged_plan(B)
    none, pos = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    tv.paged_plan(bank, req, none, pos, status, plan, n_q_heads=Hq, n_kv_heads=H)
    kv, q = (torch.empty(0, h, d, dtype=BF, device="cuda") for h in (H, Hq))
    ws = tv.make_workspace(tv.tb_workspace_size(0, 1, H, Hq, d, 0, 0))
    tv.paged_kv_store_q4(pages, none, kv, kv, layer=1, q=q, q_out=torch.empty_like(q), positions=pos, rope_theta=1e4)
    tv.paged_tree_attention_q4(bank, req, pages, plan, q, torch.empty_like(q), ws, layer=1)
    tv.paged_kv_load_q4(pages, none, kv, torch.empty_like(kv))
    # rows there, but none of a request's
    q8, out = (torch.full((8, Hq, d), 3.0, dtype=BF, device="cuda") for _ in range(2))
    tv.paged_tree_attention_q4(bank, req, pages, plan, q8, out, ws, layer=1)
    results = tv.make_results(B)
    results.fill_(4)
    tv.paged_accept_q4(bank, req, pages, results, draft=pos, argmax=pos, vocab=9)
    torch.cuda.synchronize()
    assert results.tolist() == [[0, -1, L, 0] + [0] * 64 for L in (20, 30, 0)]
    assert torch.equal(pages.k, before[0]) and torch.equal(pages.v, before[1]) and bool((out == 3).all())
    assert tv.tb_workspace_status(ws) == tv.TB_OK


def test_the_widest_groups(bank):  # noqa: F811
    """64 query heads of one kv head: rows in blocks of 128, of which a tree's last may hold few."""
    Scene(60, [700, 130], [1, 3], 64, 1, 64, 16).check(bank)
    Scene(61, [3000], [2], 64, 1, 128, 64).check(bank, cap=20.0)
    # 33 heads: 4 nodes are 132 rows, a block of four behind one of 128; long enough for the way of few rows
    Scene(62, [40000], [2], 33, 1, 64, 128).check(bank)

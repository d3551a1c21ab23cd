"""paged_accept: acceptance against the oracle, moved rows and untouched ones
byte for byte, lengths in place."""
import numpy as np
import pytest
import torch

import oracle
import paged_reference as ref
import paper_2606_27550_gb300 as tv
from paper_2606_27550_gb300 import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bank():
    b = tv.Bank(16, 0)
    for t in ref.trees():
        b.add(t)
    yield b
    b.close()


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).cuda()


class Scene:
    def __init__(self, seed, lens, tree, layers, H, d, P, layout, vocab=50, match=0.7, refused=()):
        g = self.g = synth.rng(seed)
        torch.manual_seed(seed)
        self.trees, self.lens, self.tree, self.P, self.vocab = ref.trees(), lens, tree, P, vocab
        B = len(lens)
        self.n = [0 if t < 0 or b in refused else len(self.trees[t]) for b, t in enumerate(tree)]
        counts = [-(-(a + b) // P) for a, b in zip(lens, self.n)]
        n_pages = sum(counts) + 2
        ids = g.permutation(n_pages)
        self.table = np.full((B, max(counts) + 1), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        shape = (layers, n_pages, H, P, d) if layout == "heads" else (layers, n_pages, P, H, d)
        self.pools = []
        for _ in range(2):
            t = torch.randint(-30000, 30000, shape, dtype=torch.int16, device="cuda").view(torch.bfloat16)
            self.pools.append(t if layout == "heads" else t.transpose(2, 3))
        self.start = np.concatenate([[0], np.cumsum(self.n)])
        R = int(self.start[-1])
        self.argmax = g.integers(0, vocab, R).astype(np.int32)
        self.draft = g.integers(0, vocab, R).astype(np.int32)
        for b in range(B):
            p = self.trees[tree[b]] if self.n[b] else []
            for j in range(1, len(p)):
                if g.random() < match:
                    self.draft[self.start[b] + j] = self.argmax[self.start[b] + p[j]]
        self.req = tv.Requests(row_start=i32(self.start), lens=i32(np.array(lens)), table=i32(self.table), page_size=P,
                               tree=i32(np.array(tree)))
        self.results = tv.make_results(B)

    def expected(self, b):
        lo, hi = self.start[b], self.start[b + 1]
        return oracle.accept(self.trees[self.tree[b]], self.draft[lo:hi], self.argmax[lo:hi])

    def moved(self, paths):
        want = [p.clone() for p in self.pools]
        for b, path in paths.items():
            L, t = self.lens[b], self.table[b]
            for new, old in zip(want, self.pools):
                for j, u in enumerate(path):
                    new[:, t[(L + j) // self.P], :, (L + j) % self.P] = old[:, t[(L + u) // self.P], :, (L + u) % self.P]
        return want


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("seed,B,layers,H,d,P,layout,in_place", [
    (1, 1, 1, 1, 64, 8, "heads", True), (2, 9, 3, 4, 128, 16, "slots", True), (3, 40, 2, 8, 64, 32, "heads", False),
    (4, 5, 33, 3, 128, 16, "heads", True), (5, 300, 1, 2, 64, 128, "slots", True), (6, 4, 2, 40, 128, 1024, "slots", False)])
@pytest.mark.parametrize("match", [0.0, 0.7, 1.0])
def test_accept(bank, seed, B, layers, H, d, P, layout, in_place, match):
    g = synth.rng(seed + 500)
    lens = [int(g.integers(0, 200)) for _ in range(B)]
    tree = [int(g.integers(-1 if B > 1 else 0, 11)) for _ in range(B)]
    s = Scene(seed, lens, tree, layers, H, d, P, layout, match=match, refused=(2,))
    paths, results = {}, []
    for b in range(B):
        if s.n[b]:
            k, path, bonus = s.expected(b)
            paths[b] = path
            results.append([k, bonus, lens[b] + k, 0] + list(path) + [0] * (64 - k))
        else:
            results.append([0, -1, lens[b], 0] + [0] * 64)
    want = s.moved(paths)
    out = None if in_place else torch.zeros(B, dtype=torch.int32, device="cuda")
    tv.paged_accept(bank, s.req, tv.Pages(*s.pools), s.results, draft=i32(s.draft), argmax=i32(s.argmax),
                    vocab=s.vocab, lens_out=out)
    torch.cuda.synchronize()
    assert s.results.tolist() == results
    assert (s.req.lens if in_place else out).tolist() == [r[2] for r in results]
    if not in_place:
        assert s.req.lens.tolist() == lens
    assert same(s.pools[0], want[0]) and same(s.pools[1], want[1])


def test_results_of_another_rule(bank):
    """accept_len and path given: the rows move, the lengths advance, the results keep their words."""
    s = Scene(31, [100, 20, 0, 64], [5, 8, -1, 10], 2, 2, 64, 16, "heads")
    paths = {}
    res = np.zeros((4, 68), np.int32)
    for b in (0, 1, 3):
        parent, u = s.trees[s.tree[b]], len(s.trees[s.tree[b]]) - 1
        path = []
        while u >= 0:
            path.insert(0, int(u))
            u = parent[u]
        paths[b] = path
        res[b, 0], res[b, 1], res[b, 4:4 + len(path)] = len(path), 9, path
    want = s.moved(paths)
    s.results.copy_(i32(res))
    tv.paged_accept(bank, s.req, tv.Pages(*s.pools), s.results)
    torch.cuda.synchronize()
    new = [x + len(paths.get(b, ())) for b, x in enumerate(s.lens)]
    assert s.req.lens.tolist() == new
    got = s.results.cpu().numpy()
    assert got[:, 2].tolist() == new
    got[:, 2] = res[:, 2]
    assert np.array_equal(got, res)
    assert same(s.pools[0], want[0]) and same(s.pools[1], want[1])


def test_bad_tokens_and_no_pages(bank):
    s = Scene(41, [10, 30], [3, 3], 1, 1, 64, 16, "heads", match=1.0)
    s.draft[1] = s.vocab
    s.draft[8 + 2] = -4
    before = [p.clone() for p in s.pools]
    tv.paged_accept(bank, s.req, None, s.results, draft=i32(s.draft), argmax=i32(s.argmax), vocab=s.vocab)
    torch.cuda.synchronize()
    for b in range(2):
        k, path, bonus = s.expected(b)
        got = s.results[b].tolist()
        assert got[:4] == [k, bonus, s.lens[b] + k, tv.TB_EINVAL] and got[4:4 + k] == list(path)
    assert same(before[0], s.pools[0]) and same(before[1], s.pools[1])


@pytest.mark.parametrize("layers,H", [(4, 4), (12, 4), (12, 8), (20, 8)])
def test_requests_of_one_and_more_ctas(bank, layers, H):
    """From one CTA per request to a cluster of eight; lengths in place."""
    g = synth.rng(layers)
    B = 90
    lens, tree = [int(g.integers(0, 60)) for _ in range(B)], [int(g.integers(0, 11)) for _ in range(B)]
    s = Scene(layers + H, lens, tree, layers, H, 128, 16, "heads", match=0.9)
    paths = {b: s.expected(b)[1] for b in range(B)}
    want = s.moved(paths)
    tv.paged_accept(bank, s.req, tv.Pages(*s.pools), s.results, draft=i32(s.draft), argmax=i32(s.argmax), vocab=s.vocab)
    torch.cuda.synchronize()
    assert s.req.lens.tolist() == [L + len(paths[b]) for b, L in enumerate(lens)]
    assert same(s.pools[0], want[0]) and same(s.pools[1], want[1])


@pytest.mark.parametrize("layers,H", [(1, 1), (8, 8)])
def test_results_left_by_an_earlier_step(bank, layers, H):
    """Given results: a waiting and a refused request get accept_len 0 whatever their results held, and an accept_len
    above the tree's nodes or below 0 is clamped in the result as in the length."""
    s = Scene(51, [100, 20, 30, 64, 7], [3, -1, 5, 8, 2], layers, H, 64, 16, "heads", refused=(2,))
    res = np.zeros((5, 68), np.int32)
    res[:, 0], res[:, 1], res[:, 2], res[:, 3] = (99, 3, 4, 20, -6), 9, 1234, 0
    res[:, 4:] = 1
    n = [8, 0, 0, 20, 4]
    paths = {0: [0, 1, 2, 3, 4, 5, 6, 7], 3: list(range(20))}
    for b, path in paths.items():
        res[b, 4:4 + len(path)] = path
    res[3, 4:24] = range(20)
    s.results.copy_(i32(res))
    before = [p.clone() for p in s.pools]
    tv.paged_accept(bank, s.req, tv.Pages(*s.pools), s.results)
    torch.cuda.synchronize()
    want = res.copy()
    want[:, 0] = n[0], 0, 0, 20, 0
    want[:, 2] = 108, 20, 30, 84, 7
    for b in (1, 2):
        want[b, 1], want[b, 4:] = -1, 0
    assert s.results.tolist() == want.tolist()
    assert s.req.lens.tolist() == want[:, 2].tolist()
    assert same(before[0], s.pools[0]) and same(before[1], s.pools[1])  # every path is in place already


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("entry", [-1, 10 ** 6])
def test_rows_that_cannot_move_are_reported(bank, given, entry):
    """A hole in the table under the last accepted node: that row stays, the others move, the request says so."""
    s = Scene(61, [5, 40], [7, 7], 3, 2, 64, 8, "heads", match=1.0)
    paths = {b: list(s.expected(b)[1]) for b in range(2)}
    assert paths[0][-1] > 20
    hole = (5 + paths[0][-1]) // 8
    s.req.table[0, hole] = entry
    stays = [j for j, u in enumerate(paths[0]) if hole in ((5 + u) // 8, (5 + j) // 8)]
    assert len(paths[0]) - 1 in stays and len(stays) < len(paths[0])
    kept = {0: [j if j in stays else u for j, u in enumerate(paths[0])], 1: paths[1]}
    want = s.moved(kept)
    kw = dict(draft=i32(s.draft), argmax=i32(s.argmax), vocab=s.vocab)
    if given:
        kw = {}
        for b, path in paths.items():
            s.results[b, 0] = len(path)
            s.results[b, 4:4 + len(path)] = i32(np.array(path))
    tv.paged_accept(bank, s.req, tv.Pages(*s.pools), s.results, **kw)
    torch.cuda.synchronize()
    assert s.results[:, 3].tolist() == [tv.TB_EINVAL, 0]
    assert s.results[:, 0].tolist() == [len(paths[0]), len(paths[1])]
    assert s.req.lens.tolist() == [5 + len(paths[0]), 40 + len(paths[1])]
    assert same(s.pools[0], want[0]) and same(s.pools[1], want[1])

"""paged_tree_attention against 64 bits: page sizes and layouts, types, head
groups, windows, caps, biases, rows that see nothing, pages whose unseen slots
hold NaN, slots past 32-bit offsets, streams and graphs."""
import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2606_27550_gb300 as tv
from paper_2606_27550_gb300 import synth

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def bank():
    b = tv.Bank(16, 0)
    for t in ref.trees():
        b.add(t)
    yield b
    b.close()


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class Scene:
    """A batch with its pages; every slot that no row may see holds NaN."""

    def __init__(self, seed, lens, tree, Hq, H, d, P=16, layout="heads", dtype=BF, layers=1, layer=0, begin=None,
                 q_std=1.5, n_extra=0):
        torch.manual_seed(seed)
        self.g = synth.rng(seed)
        self.trees = ref.trees()
        self.lens, self.tree, self.P, self.H, self.Hq, self.d, self.dtype = lens, tree, P, H, Hq, d, dtype
        self.begin, self.layer = begin, layer
        self.n = [0 if t < 0 else len(self.trees[t]) for t in tree]
        counts = [-(-(a + b) // P) for a, b in zip(lens, self.n)]
        n_pages = sum(counts) + 2 + n_extra
        ids = n_extra + self.g.permutation(n_pages - n_extra)  # the pool's last pages
        table = np.full((len(lens), max(counts) + 1), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            table[b, :c] = ids[at:at + c]
            at += c
        shape = (layers, n_pages, H, P, d) if layout == "heads" else (layers, n_pages, P, H, d)
        pools = []
        self.dense = []
        for _ in range(2):
            t = torch.empty(shape, dtype=dtype, device="cuda")
            t[:, n_extra:] = float("nan")
            pools.append(t if layout == "heads" else t.transpose(2, 3))
        self.table = torch.from_numpy(table).cuda()
        for b, (L, n) in enumerate(zip(lens, self.n)):
            kv = [torch.randn(L + n, H, d, device="cuda").to(dtype) for _ in range(2)]
            self.dense.append([x.double().cpu().numpy() for x in kv])
            slot = torch.arange(L + n, device="cuda")
            if begin:  # before the document: NaN stays
                slot = slot[begin[b]:]
            for pool, x in zip(pools, kv):
                pool[layer].transpose(1, 2)[self.table[b].long()[slot // P], slot % P] = x[slot]
        self.pages = tv.Pages(*pools)
        self.R = sum(self.n)
        self.q = (q_std * torch.randn(self.R, Hq, d, device="cuda")).to(dtype)

    def run(self, bank, window=0, sink=0, cap=0.0, slopes=None, scale=None, stream=None, extra_rows=0):
        B = len(self.lens)
        self.req = tv.Requests(row_start=torch.empty(B + 1, dtype=torch.int32, device="cuda"), lens=i32(self.lens),
                               table=self.table, page_size=self.P, tree=i32(self.tree),
                               key_begin=i32(self.begin) if self.begin else None)
        slots = torch.empty(max(1, self.R), dtype=torch.int64, device="cuda")
        pos = torch.empty(max(1, self.R), dtype=torch.int32, device="cuda")
        status = torch.empty(B, dtype=torch.int32, device="cuda")
        self.plan = tv.make_paged_plan(B)
        tv.paged_plan(bank, self.req, slots, pos, status, self.plan, n_q_heads=self.Hq, n_kv_heads=self.H,
                      window=window, sink=sink)
        assert status.tolist() == [0] * B
        out = torch.full((self.R + extra_rows, self.Hq, self.d), 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full((self.R + extra_rows, self.Hq), 7.0, dtype=torch.float32, device="cuda")
        q = torch.cat([self.q, self.q[:1].expand(extra_rows, -1, -1)]) if extra_rows else self.q
        self.ws = tv.make_workspace(tv.tb_workspace_size(0, 1, self.H, self.Hq, self.d, 0, 0))
        self.call = lambda: tv.paged_tree_attention(bank, self.req, self.pages, self.plan, q, out, self.ws,
                                                    layer=self.layer, softcap=cap, slopes=slopes, lse=lse, scale=scale)
        self.call()
        torch.cuda.synchronize()
        assert tv.tb_workspace_status(self.ws) == 0
        if extra_rows:
            assert bool((out[self.R:] == 7).all()) and bool((lse[self.R:] == 7).all())
        self.out, self.lse = out, lse
        return out[:self.R].double().cpu().numpy(), lse[:self.R].double().cpu().numpy()

    def check(self, bank, window=0, sink=0, cap=0.0, slopes=None, scale=None, only=None, extra_rows=0):
        out, lse = self.run(bank, window, sink, cap, slopes, scale, extra_rows=extra_rows)
        q = self.q.double().cpu().numpy()
        at = 0
        # weights and outputs are each rounded once to the type; 2^-12 for the 32-bit steps, and a score
        # of size z carries a rounding of 2^-22 z into its weight
        eps = 2.0 ** -8 if self.dtype == BF else 2.0 ** -11
        s64 = None if slopes is None else slopes.double().cpu().numpy()
        for b, n in enumerate(self.n):
            if n and (only is None or b in only):
                k, v = self.dense[b]
                o, ls, absv, big = ref.attend(q[at:at + n], k, v, self.trees[self.tree[b]], self.lens[b],
                                              self.d ** -0.5 if scale is None else scale, cap, s64, window, sink,
                                              self.begin[b] if self.begin else 0)
                bound = eps * np.abs(o) + (eps + 2.0 ** -12 + 2.0 ** -21 * big[..., None]) * absv + 1e-7
                err = np.abs(out[at:at + n] - o)
                assert np.isfinite(out[at:at + n]).all(), f"request {b}"
                assert (err <= bound).all(), f"request {b}: {(err - bound).max()} over at |o| {np.abs(o).max()}"
                empty = np.isneginf(ls)
                assert (np.isneginf(lse[at:at + n]) == empty).all()
                tol = 1e-5 + 2.0 ** -21 * np.maximum(np.abs(ls), big)
                assert (np.abs(lse[at:at + n][~empty] - ls[~empty]) <= tol[~empty]).all()
                assert (out[at:at + n][empty] == 0).all()
            at += n


# trees by number: 0..7 the bank's (1, 2, 4, 8, 16, 26, 40, 64 nodes), 8 a chain of 20, 9 a star of 12, 10 random 37
@pytest.mark.parametrize("Hq,H,d,P,layout,dtype", [
    (4, 4, 64, 16, "heads", BF), (8, 2, 128, 16, "slots", BF), (12, 4, 64, 32, "slots", HF),
    (16, 1, 128, 64, "heads", HF), (7, 1, 128, 8, "heads", BF), (32, 8, 128, 128, "slots", BF),
    (5, 5, 64, 256, "heads", HF), (6, 3, 128, 1024, "slots", HF), (64, 2, 64, 16, "heads", BF)])
@pytest.mark.parametrize("mode", ["plain", "cap", "bias", "window", "all"])
def test_ragged_batches(bank, Hq, H, d, P, layout, dtype, mode):
    lens = [0, 1, 127, 128, 129, 300, 63, 511, 65, 1000, 17]
    tree = [0, 7, 5, 3, 10, 8, -1, 9, 6, 0, 4]
    s = Scene(Hq * 7 + P, lens, tree, Hq, H, d, P, layout, dtype)
    slopes = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if mode in ("bias", "all") else None
    kw = dict(cap=6.0 if mode in ("cap", "all") else 0.0, slopes=slopes, window=100 if mode in ("window", "all") else 0,
              sink=5 if mode == "all" else 0)
    s.check(bank, **kw)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (2, 130), (5, 0), (64, 4), (128, 128), (129, 300), (2000, 7),
                                         (400, 257)])
def test_windows(bank, window, sink):
    """Windows shorter than the tree, ends inside and at tiles, first tokens that meet the window."""
    s = Scene(window + sink, [700, 3, 128, 1500, 0, 255, 384], [8, 7, 10, 7, 8, 0, 2], 8, 4, 64, 16)
    s.check(bank, window=window, sink=sink)


@pytest.mark.parametrize("sink", [0, 20])
def test_documents_that_begin_late_and_rows_that_see_nothing(bank, sink):
    lens = [300, 40, 256, 500, 130, 0, 64]
    tree = [5, 8, 7, 10, 0, 4, 9]
    # inside the prefix, at its end, at a tile's edge, inside the tree, past everything
    begin = [77, 40, 128, 0, 131, 3, 200]
    s = Scene(90 + sink, lens, tree, 8, 2, 128, 16, begin=[min(b, x + len(ref.trees()[t])) for b, x, t in
                                                          zip(begin, lens, tree)])
    s.check(bank)
    s.begin = begin
    s.check(bank, window=60, sink=sink)


def test_one_token_for_many_requests(bank):
    """Plain decoding, batch larger than the SM count, empty slots between."""
    g = synth.rng(5)
    B = 200
    lens = [int(x) for x in g.integers(0, 400, B)]
    tree = [0 if g.random() < 0.8 else -1 for _ in range(B)]
    Scene(5, lens, tree, 8, 2, 64, 16).check(bank)


@pytest.mark.parametrize("L,Hq,H,tree", [(20000, 4, 2, 7), (9000, 2, 1, 0), (5000, 1, 1, 5)])
def test_few_long_units_are_split(bank, L, Hq, H, tree):
    Scene(L, [L], [tree], Hq, H, 128, 64).check(bank)
    Scene(L + 1, [L], [tree], Hq, H, 64, 16, dtype=HF).check(bank, cap=20.0, window=L // 2, sink=300)


def test_large_scores_and_weights(bank):
    """Scores of several hundred, increasing along the keys so that the running maximum keeps growing."""
    s = Scene(11, [900], [5], 4, 4, 64, 16, q_std=1.0)
    k = s.pages.k[0]
    d0 = torch.zeros(64, device="cuda")
    d0[0] = 1.0
    ramp = torch.arange(926, device="cuda") * 0.5
    slot = torch.arange(926, device="cuda")
    page = s.table[0].long()[slot // 16]
    kk = (torch.randn(926, 4, 64, device="cuda") * 0.1 + ramp[:, None, None] * d0).to(BF)
    k.transpose(1, 2)[page, slot % 16] = kk
    s.dense[0][0] = kk.double().cpu().numpy()
    s.q[..., 0] = 8.0
    s.check(bank)
    s.q[..., 0] = -8.0
    s.check(bank)


def test_layers_strides_and_side_by_side_pools(bank):
    """K and V in one tensor, layers between other data, the second of three layers."""
    torch.manual_seed(2)
    s = Scene(77, [200, 90], [5, 7], 8, 4, 64, 16, layers=3, layer=1)
    n = s.pages.k.shape[1]
    both = torch.full((3, n, 2, 4, 16, 72), float("nan"), dtype=BF, device="cuda")
    both[:, :, 0, :, :, :64] = s.pages.k
    both[:, :, 1, :, :, :64] = s.pages.v
    s.pages = tv.Pages(both[:, :, 0, :, :, :64], both[:, :, 1, :, :, :64])
    s.check(bank)


def test_rows_past_the_batch_and_scale(bank):
    Scene(15, [100, 0, 30], [2, -1, 3], 4, 2, 128, 16).check(bank, scale=0.3, extra_rows=9)


def test_offsets_past_32_bits(bank):
    """Pages behind more than 2^32 bytes and 2^31 elements of the pool."""
    n = (1 << 31) // (2 * 128 * 128) + 40
    s = Scene(19, [300, 700], [5, 0], 4, 2, 128, 128, n_extra=n)
    assert s.pages.k.stride(1) * n > 2**31
    s.check(bank)


def test_streams_graphs_and_repeats(bank):
    s = Scene(23, [600, 4000, 20], [7, 5, 0], 8, 2, 128, 32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.check(bank, cap=30.0)
    side.synchronize()
    first = [s.out.clone(), s.lse.clone()]
    for _ in range(3):
        s.out.zero_()
        s.call()
        torch.cuda.synchronize()
        assert torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    s.out.zero_()
    s.lse.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])


def test_a_plan_of_other_heads_is_refused_on_the_device(bank):
    s = Scene(29, [50], [2], 4, 2, 64, 16)
    s.run(bank)
    out = torch.full((s.R, 8, 64), 3.0, dtype=BF, device="cuda")
    q = torch.zeros_like(out)
    tv.paged_tree_attention(bank, s.req, s.pages, s.plan, q, out, s.ws)
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_EINVAL and bool((out == 3).all())


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(bank, seed):
    g = synth.rng(1000 + seed)
    B = int(g.integers(1, 12))
    H, group = int(g.choice([1, 2, 3, 4, 8])), int(g.choice([1, 1, 2, 3, 4, 8]))
    d, P = int(g.choice([64, 128])), int(g.choice([8, 16, 32, 64, 128, 512]))
    lens = [int(g.integers(0, int(g.choice([4, 200, 3000])))) for _ in range(B)]
    tree = [int(g.integers(-1, 11)) for _ in range(B)]
    if all(t < 0 for t in tree):
        tree[0] = 3
    begin = [int(g.integers(0, L + 1)) for L in lens] if g.random() < 0.3 else None
    s = Scene(seed, lens, tree, H * group, H, d, P, str(g.choice(["heads", "slots"])), BF if g.random() < 0.5 else HF,
              begin=begin)
    window = int(g.choice([0, 0, int(g.integers(1, 600))]))
    slopes = torch.rand(H * group, device="cuda") if g.random() < 0.3 else None
    s.check(bank, window=window, sink=int(g.integers(0, 200)) if window else 0,
            cap=float(g.choice([0.0, 0.0, 5.0, 50.0])), slopes=slopes)


@pytest.mark.parametrize("cap", [0.01, 0.5, 50.0, 1024.0])
@pytest.mark.parametrize("biased", [False, True])
def test_caps_from_saturated_to_hardly_bent(bank, cap, biased):
    """Scores far past the cap in both directions, and caps far past the scores; hidden slots hold NaN."""
    s = Scene(int(cap) + 3, [130, 5, 0, 260], [7, 5, 8, 0], 6, 3, 64, 16, q_std=20.0 if cap < 100 else 2.0)
    slopes = torch.full((6,), 0.05, device="cuda") if biased else None
    out, lse = s.run(bank, cap=cap, slopes=slopes)
    q, at = s.q.double().cpu().numpy(), 0
    s64 = None if slopes is None else slopes.double().cpu().numpy()
    for b, n in enumerate(s.n):
        k, v = s.dense[b]
        o, ls, absv, big = ref.attend(q[at:at + n], k, v, s.trees[s.tree[b]], s.lens[b], s.d ** -0.5, cap, s64)
        # as for the others, and the documented cap 2^-20 of every score (once in the weight, once in the sum)
        z = 2.0 ** -21 * big + 2.0 ** -20 * cap
        bound = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -12 + 2 * z[..., None]) * absv + 1e-7
        assert (np.abs(out[at:at + n] - o) <= bound).all()
        assert (np.abs(lse[at:at + n] - ls) <= 1e-5 + 2.0 ** -21 * np.abs(ls) + z).all()
        at += n


def test_a_query_that_is_not_a_number_shows(bank):
    """With a cap, NaN in one row's query makes that row NaN and leaves the others as they were."""
    s = Scene(4, [70], [5], 2, 2, 64, 16)
    want, _ = s.run(bank, cap=30.0)
    s.q[3, 1, 5] = float("nan")
    got, _ = s.run(bank, cap=30.0)
    assert np.isnan(got[3, 1]).all()
    got[3, 1] = want[3, 1]
    assert np.array_equal(got, want)


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("L", [70, 9000])
def test_a_score_that_is_not_finite_shows_in_the_log_sum_exp(bank, form, dtype, L):
    """NaN in a query, NaN in one visible key, a score of +inf: output and log-sum-exp of those rows are NaN, in units
    of one CTA and of several, and all others are as they were."""
    s = Scene(L, [L], [3], 4, 2, 64, 16, dtype=dtype)
    kw = dict(cap=30.0 if form == "cap" else 0.0, slopes=torch.full((4,), 0.02, device="cuda") if form == "bias" else None)
    want, want_lse = s.run(bank, **kw)
    assert np.isfinite(want).all() and np.isfinite(want_lse).all()
    kept = s.q.clone()
    for value in (float("nan"), float("inf")):
        if value == float("inf") and form == "cap":
            continue  # capped: a finite score
        s.q.copy_(kept)
        s.q[2, 1, 5] = value  # +inf times a key of either sign: +inf, -inf and so NaN among the scores
        got, lse = s.run(bank, **kw)
        assert np.isnan(got[2, 1]).all() and np.isnan(lse[2, 1])
        got[2, 1], lse[2, 1] = want[2, 1], want_lse[2, 1]
        assert np.array_equal(got, want) and np.array_equal(lse, want_lse)
    # one key of head 0, in the prefix: every row of its two query heads
    s.q.copy_(kept)
    slot = L // 2
    s.pages.k[0, int(s.table[0, slot // 16]), 0, slot % 16, 9] = float("nan")
    got, lse = s.run(bank, **kw)
    assert np.isnan(got[:, :2]).all() and np.isnan(lse[:, :2]).all()
    assert np.array_equal(got[:, 2:], want[:, 2:]) and np.array_equal(lse[:, 2:], want_lse[:, 2:])


@pytest.mark.parametrize("L", [90, 6000])
@pytest.mark.parametrize("window", [0, 3])
def test_a_plan_of_another_bank(bank, L, window):
    """Requests whose tree the call's bank lacks, or has with other nodes, are reported and left out, whether one CTA
    has their unit or several; the others are served."""
    s = Scene(L, [L, 40, L, 70, 9], [0, 9, 7, 3, 1], 4, 2, 64, 16)
    s.run(bank, window=window)
    at = np.concatenate([[0], np.cumsum(s.n)])

    def left_out(trees, served):
        other = tv.Bank(len(trees), 0)
        for t in trees:
            other.add(s.trees[t])
        ws = tv.make_workspace(tv.tb_workspace_size(0, 1, s.H, s.Hq, s.d, 0, 0))
        out, lse = torch.full_like(s.out, 5.0), torch.full_like(s.lse, 5.0)
        tv.paged_tree_attention(other, s.req, s.pages, s.plan, s.q, out, ws, lse=lse)
        torch.cuda.synchronize()
        assert tv.tb_workspace_status(ws) == (tv.TB_OK if all(served) else tv.TB_EINVAL)
        for b, known in enumerate(served):
            rows = slice(at[b], at[b + 1])
            for got, was in ((out, s.out), (lse, s.lse)):
                assert torch.equal(got[rows], was[rows] if known else torch.full_like(was[rows], 5.0))
        other.close()

    left_out((0, 1, 5, 3), (True, False, False, True, True))
    left_out((0,), (True, False, False, False, False))
    left_out((0, 1, 2, 4, 4, 5, 6, 7, 8, 9), (True, True, True, False, True))
    left_out(range(10), (True,) * 5)


@pytest.mark.parametrize("P", [16, 128, 512])
@pytest.mark.parametrize("entry", [-1, -2 ** 31, "past", 2 ** 31 - 1])
def test_holes_in_the_table(bank, P, entry):
    """A page that is not there, where rows look: reported, its keys and values zeros.  Where none looks: nothing."""
    def scene(**kw):
        s = Scene(P, [1700, 300], [5, 3], 4, 2, 64, P, **kw)
        return s, s.pages.k.shape[1] if entry == "past" else entry

    def run(s, reported, **kw):
        real = tv.tb_workspace_status
        tv.tb_workspace_status = lambda ws: 0  # (the scene's own check)
        try:
            s.check(bank, **kw)
        finally:
            tv.tb_workspace_status = real
        assert tv.tb_workspace_status(s.ws) == (tv.TB_EINVAL if reported else tv.TB_OK)

    for page in (0, 1024 // P, 1699 // P):  # the first page, one in the middle, the last prefix slot's
        s, e = scene()
        s.table[0, page] = e
        for x in s.dense[0]:
            x[page * P:(page + 1) * P] = 0
        run(s, True)
        # with a window of 100 the pages before slot 1601 are looked at by the first tokens' rule alone
        run(s, page * P + P > 1601, window=100)
        run(s, page * P + P > 1601 or page * P < 20, window=100, sink=20)
    # documents that begin behind the hole, at its end, inside it
    for begin, reported in ((1024 + P, False), (1023 + P, True), (1024, True)):
        s, e = scene(begin=[begin, 0])
        s.table[0, 1024 // P] = e
        for x in s.dense[0]:
            x[1024:1024 + P] = 0
        run(s, reported)

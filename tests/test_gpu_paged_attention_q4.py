"""paged_tree_attention_q4 against 64 bits: the cases of paged_tree_attention's test
over pages of 4 bits, from single tokens (few rows per kv head) to whole trees.
Every slot that no row may see has the scale NaN and any codes."""
import time

import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2606_27550_gb300 as tv
import q4_reference as q4
from paper_2606_27550_gb300 import synth
from test_gpu_paged_attention import BF, HF, bank, i32  # noqa: F401
from test_gpu_paged_attention import Scene as Scene16

pytestmark = pytest.mark.gpu


class Scene(Scene16):
    """The 16-bit scene's batch, its keys and values replaced by ones of 4 bits."""

    def __init__(self, seed, lens, tree, Hq, H, d, P=16, dtype=BF, layers=1, layer=0, begin=None, q_std=1.5, n_extra=0):
        super().__init__(seed, lens, tree, Hq, H, d, P, "heads", dtype, 1, 0, begin, q_std, 0)
        self.layer = layer
        n_pages = self.pages.k.shape[1] + n_extra
        if n_extra:
            self.table[self.table >= 0] += n_extra
        shape = (layers, n_pages, H, tv.q4_page_bytes(P, d))
        pools = []
        for i in range(2):
            pool = torch.empty(shape, dtype=torch.uint8, device="cuda")
            codes, scales = q4.parts(pool, P, d)
            codes[:, n_extra:].random_(0, 256)
            scales[:, n_extra:] = 255
            for b, (L, n) in enumerate(zip(lens, self.n)):
                c = (torch.randn(L + n, H, d, device="cuda") * 2.5).round().clamp(-7, 7)
                byte = torch.randint(0x60, 0x6D, (L + n, H, d // 32), device="cuda")
                c8 = (c + 8).to(torch.uint8)
                slot = torch.arange(L + n, device="cuda")
                if begin:
                    slot = slot[begin[b]:]
                page, at = self.table[b].long()[slot // P], slot % P
                codes[layer].transpose(1, 2)[page, at] = (c8[..., 0::2] | (c8[..., 1::2] << 4))[slot]
                scales[layer].transpose(1, 2)[page, at] = byte.to(torch.uint8)[slot]
                s = torch.from_numpy(q4.scale_value(byte.cpu().numpy())).cuda()
                self.dense[b][i] = (c.double() * s.repeat_interleave(32, -1)).cpu().numpy()
            pools.append(pool)
        self.pages = tv.PagesQ4(*pools, P, d, dtype)

    def run(self, bank, window=0, sink=0, cap=0.0, slopes=None, scale=None, stream=None, extra_rows=0):  # noqa: F811
        B = len(self.lens)
        self.req = tv.Requests(row_start=torch.empty(B + 1, dtype=torch.int32, device="cuda"), lens=i32(self.lens),
                               table=self.table, page_size=self.P, tree=i32(self.tree),
                               key_begin=i32(self.begin) if self.begin else None)
        rows = max(1, self.R)
        slots, pos = (torch.empty(rows, dtype=t, device="cuda") for t in (torch.int64, torch.int32))
        status = torch.empty(B, dtype=torch.int32, device="cuda")
        self.plan = tv.make_paged_plan(B)
        tv.paged_plan(bank, self.req, slots, pos, status, self.plan, n_q_heads=self.Hq, n_kv_heads=self.H,
                      window=window, sink=sink)
        assert status.tolist() == [0] * B
        out = torch.full((self.R + extra_rows, self.Hq, self.d), 7.0, dtype=self.dtype, device="cuda")
        lse = torch.full((self.R + extra_rows, self.Hq), 7.0, dtype=torch.float32, device="cuda")
        q = torch.cat([self.q, self.q[:1].expand(extra_rows, -1, -1)]) if extra_rows else self.q
        self.ws = tv.make_workspace(tv.tb_workspace_size(0, 1, self.H, self.Hq, self.d, 0, 0))
        self.call = lambda **kw: tv.paged_tree_attention_q4(bank, self.req, self.pages, self.plan, q, out, self.ws,
                                                            layer=self.layer, softcap=cap, slopes=slopes, lse=lse,
                                                            scale=scale, **kw)
        self.call()
        torch.cuda.synchronize()
        self.status = tv.tb_workspace_status(self.ws)
        assert self.status == 0 or getattr(self, "may_report", False)
        if extra_rows:
            assert bool((out[self.R:] == 7).all()) and bool((lse[self.R:] == 7).all())
        self.out, self.lse = out, lse
        return out[:self.R].double().cpu().numpy(), lse[:self.R].double().cpu().numpy()

    def scales(self, i, b, slot, g):
        """The scale bytes of a slot of request b (i: 0 for K, 1 for V)."""
        pool = self.pages.k if i == 0 else self.pages.v
        return q4.parts(pool, self.P, self.d)[1][self.layer, int(self.table[b, slot // self.P]), g, slot % self.P]


MODES = ["plain", "cap", "bias", "window", "all"]


def mode_args(mode, Hq):
    slopes = 2.0 ** (-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if mode in ("bias", "all") else None
    return dict(cap=6.0 if mode in ("cap", "all") else 0.0, slopes=slopes, window=100 if mode in ("window", "all") else 0,
                sink=5 if mode == "all" else 0)


# trees by number: 0..7 the bank's (1, 2, 4, 8, 16, 26, 40, 64 nodes), 8 a chain of 20, 9 a star of 12, 10 random 37
@pytest.mark.parametrize("Hq,H,d,P,dtype", [
    (4, 4, 64, 16, BF), (8, 2, 128, 16, BF), (12, 4, 64, 32, HF), (16, 1, 128, 64, HF), (7, 1, 128, 8, BF),
    (32, 8, 128, 128, BF), (5, 5, 64, 256, HF), (6, 3, 128, 1024, HF), (64, 2, 64, 8, BF)])
@pytest.mark.parametrize("mode", MODES)
def test_ragged_batches(bank, Hq, H, d, P, dtype, mode):  # noqa: F811
    lens = [0, 1, 127, 128, 129, 300, 63, 511, 65, 1000, 17]
    tree = [0, 7, 5, 3, 10, 8, -1, 9, 6, 0, 4]
    Scene(Hq * 7 + P, lens, tree, Hq, H, d, P, dtype).check(bank, **mode_args(mode, Hq))


@pytest.mark.parametrize("Hq,H,d,P,dtype,nodes", [
    (4, 4, 64, 16, BF, (0, 1, 2)), (8, 2, 128, 16, BF, (0, 1)), (8, 1, 128, 8, HF, (0,)), (8, 1, 128, 32, BF, (0, 1)),
    (16, 1, 64, 128, HF, (0,)), (2, 2, 128, 64, HF, (0, 3)), (3, 1, 64, 1024, BF, (0, 1, 2)), (14, 2, 128, 512, BF, (0, 1)),
    (12, 12, 64, 8, BF, (0, 2, 3)), (1, 1, 128, 16, HF, (4, 3, 9))])
@pytest.mark.parametrize("mode", MODES)
def test_few_rows_per_head(bank, Hq, H, d, P, dtype, nodes, mode):  # noqa: F811
    """Single tokens and small trees: up to 16 query rows per kv head, lengths about the sizes of pieces and tiles."""
    lens = [0, 1, 7, 15, 16, 17, 31, 32, 33, 63, 96, 127, 128, 129, 255, 256, 300, 511, 640, 1000, 2500]
    tree = [nodes[i % len(nodes)] for i in range(len(lens))]
    tree[5] = -1
    Scene(Hq + P, lens, tree, Hq, H, d, P, dtype).check(bank, **mode_args(mode, Hq))


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (2, 130), (5, 0), (64, 4), (128, 128), (129, 300), (2000, 7),
                                         (400, 257)])
@pytest.mark.parametrize("few", [False, True])
def test_windows(bank, window, sink, few):  # noqa: F811
    """Windows shorter than the tree, ends inside and at tiles, first tokens that meet the window."""
    tree = [0, 1, 2, 2, 0, 0, 1] if few else [8, 7, 10, 7, 8, 0, 2]
    s = Scene(window + sink, [700, 3, 128, 1500, 0, 255, 384], tree, 8, 4, 64, 16)
    s.check(bank, window=window, sink=sink)


@pytest.mark.parametrize("sink", [0, 20])
@pytest.mark.parametrize("few", [False, True])
def test_documents_that_begin_late_and_rows_that_see_nothing(bank, sink, few):  # noqa: F811
    lens = [300, 40, 256, 500, 130, 0, 64]
    tree = [0, 1, 2, 2, 0, 1, 2] if few else [5, 8, 7, 10, 0, 4, 9]
    begin = [77, 40, 128, 0, 131, 3, 200]
    s = Scene(90 + sink, lens, tree, 8, 2, 128, 16, begin=[min(b, x + len(ref.trees()[t])) for b, x, t in
                                                          zip(begin, lens, tree)])
    s.check(bank)
    s.begin = begin
    s.check(bank, window=60, sink=sink)


def test_one_token_for_many_requests(bank):  # noqa: F811
    """Plain decoding, batch larger than the SM count, empty slots between."""
    g = synth.rng(5)
    B = 200
    lens = [int(x) for x in g.integers(0, 400, B)]
    tree = [0 if g.random() < 0.8 else -1 for _ in range(B)]
    Scene(5, lens, tree, 8, 2, 64, 16).check(bank)


def test_many_units_per_cta(bank):  # noqa: F811
    """More (request, kv head) units per CTA than are laid out at a time, one tile each; a tree among the tokens."""
    B = 1500
    s = Scene(6, [i % 90 for i in range(B)], [0] * (B - 1) + [5], 16, 16, 64, 16)
    s.check(bank, only=set(range(0, B, 97)) | {B - 1, B - 2})


@pytest.mark.parametrize("L,Hq,H,tree", [(20000, 4, 2, 7), (9000, 2, 1, 0), (5000, 1, 1, 5), (70000, 8, 1, 0),
                                         (30000, 16, 4, 2)])
def test_few_long_units_are_split(bank, L, Hq, H, tree):  # noqa: F811
    Scene(L, [L], [tree], Hq, H, 128, 64).check(bank)
    Scene(L + 1, [L], [tree], Hq, H, 64, 16, dtype=HF).check(bank, cap=20.0, window=L // 2, sink=300)


@pytest.mark.parametrize("tree", [5, 0])
def test_large_scores_and_weights(bank, tree):  # noqa: F811
    """Scores of several hundred, increasing along the keys so that the running maximum keeps growing."""
    s = Scene(11, [900], [tree], 4, 4, 64, 16, q_std=1.0)
    n = 900 + s.n[0]
    # key r: 7 s_r in the first element, s_r a power of two times 8 to 15 sixteenths
    codes, scales = q4.parts(s.pages.k, 16, 64)
    slot = torch.arange(n, device="cuda")
    page, at = s.table[0].long()[slot // 16], slot % 16
    byte = (0x50 + slot * 60 // n).to(torch.uint8)
    scales[0].transpose(1, 2)[page, at, :, 0] = byte[:, None]
    codes[0].transpose(1, 2)[page, at, :, 0] = 0x8F  # 7 and 0
    codes[0].transpose(1, 2)[page, at, :, 1:16] = 0x88
    x = s.dense[0][0]
    x[:, :, :32] = 0
    x[:, :, 0] = 7 * q4.scale_value(byte.cpu().numpy())[:, None]
    s.q[..., 0] = 8.0
    s.check(bank)
    s.q[..., 0] = -8.0
    s.check(bank)


@pytest.mark.parametrize("tree", [(5, 7), (0, 1)])
def test_layers_strides_and_side_by_side_pools(bank, tree):  # noqa: F811
    """K and V in one tensor, layers innermost, gaps between the heads; the second of three layers."""
    s = Scene(77, [200, 90], list(tree), 8, 4, 64, 16, layers=3, layer=1)
    n, size = s.pages.k.shape[1], tv.q4_page_bytes(16, 64)
    both = torch.full((n, 4, 2, 3, size + 48), 255, dtype=torch.uint8, device="cuda")
    for i, x in enumerate((s.pages.k, s.pages.v)):
        both[:, :, i, :, :size] = x.permute(1, 2, 0, 3)
    s.pages = tv.PagesQ4(*(both[:, :, i, :, :size].permute(2, 0, 1, 3) for i in range(2)), 16, 64, BF)
    s.check(bank)


@pytest.mark.parametrize("tree", [(2, -1, 3), (0, -1, 1)])
def test_rows_past_the_batch_and_scale(bank, tree):  # noqa: F811
    Scene(15, [100, 0, 30], list(tree), 4, 2, 128, 16).check(bank, scale=0.3, extra_rows=9)


@pytest.mark.parametrize("lens,tree,keep", [([5000, 40, 9], (0, 1, 2), 2), ([5000, 40], (7, 5), 63), ([30], (5,), 7),
                                            ([20000, 300], (1, 7), 1)])
def test_fewer_rows_than_the_plan_has(bank, lens, tree, keep):  # noqa: F811
    """Rows of the plan past the call's n_rows are left out, in whole units and in split ones."""
    s = Scene(16, lens, list(tree), 4, 2, 64, 16)
    s.run(bank)
    out, lse = torch.full_like(s.out, 3.0), torch.full_like(s.lse, 3.0)
    tv.paged_tree_attention_q4(bank, s.req, s.pages, s.plan, s.q[:keep], out[:keep], s.ws, lse=lse[:keep])
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_OK
    assert torch.equal(out[:keep], s.out[:keep]) and torch.equal(lse[:keep], s.lse[:keep])
    assert bool((out[keep:] == 3).all()) and bool((lse[keep:] == 3).all())


@pytest.mark.parametrize("tree", [(5, 0), (0, 0)])
def test_offsets_past_32_bits(bank, tree):  # noqa: F811
    n = (1 << 32) // (2 * tv.q4_page_bytes(128, 128)) + 40
    s = Scene(19, [300, 700], list(tree), 4, 2, 128, 128, n_extra=n)
    assert s.pages.k.stride(1) * n > 2**32
    s.check(bank)


@pytest.mark.parametrize("tree", [(7, 5, 0), (0, 1, 0), (0, 7, 2)])
def test_streams_graphs_and_repeats(bank, tree):  # noqa: F811
    s = Scene(23, [600, 4000, 20], list(tree), 8, 2, 128, 32)
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


def test_a_replayed_graph_follows_the_lengths(bank):  # noqa: F811
    """Plan and attention captured once: the batch's lengths and trees change between replays."""
    s = Scene(24, [900, 300], [7, 7], 4, 2, 128, 16)
    s.run(bank)
    slots, pos = torch.empty(s.R, dtype=torch.int64, device="cuda"), torch.empty(s.R, dtype=torch.int32, device="cuda")
    status = torch.empty(2, dtype=torch.int32, device="cuda")

    def step():
        tv.paged_plan(bank, s.req, slots, pos, status, s.plan, n_q_heads=4, n_kv_heads=2)
        s.call()

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens, tree in (([500, 300], [0, 0]), ([900, 1], [0, 7]), ([0, 250], [5, 1])):
        s.req.lens.copy_(i32(lens))
        s.req.tree.copy_(i32(tree))
        s.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = s.out.clone()
        s.out.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, s.out)
        n = [len(s.trees[t]) for t in tree]
        q = s.q.double().cpu().numpy()
        for b in range(2):
            rows = slice(sum(n[:b]), sum(n[:b + 1]))
            k, v = (s.dense[b][i][:lens[b] + n[b]] for i in range(2))
            o, _, absv, big = ref.attend(q[rows], k, v, s.trees[tree[b]], lens[b], s.d ** -0.5)
            bound = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -21 * big[..., None]) * absv + 1e-7
            assert (np.abs(got[rows].double().cpu().numpy() - o) <= bound).all()
        assert bool((got[sum(n):] == 3).all())


def test_a_plan_of_other_heads_is_refused_on_the_device(bank):  # noqa: F811
    s = Scene(29, [50], [2], 4, 2, 64, 16)
    s.run(bank)
    out = torch.full((s.R, 8, 64), 3.0, dtype=BF, device="cuda")
    q = torch.zeros_like(out)
    tv.paged_tree_attention_q4(bank, s.req, s.pages, s.plan, q, out, s.ws)
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_EINVAL and bool((out == 3).all())


@pytest.mark.parametrize("seed", range(36))
def test_random_batches(bank, seed):  # noqa: F811
    g = synth.rng(2000 + seed)
    B = int(g.integers(1, 12))
    H, group = int(g.choice([1, 2, 3, 4, 8])), int(g.choice([1, 1, 2, 3, 4, 8]))
    d, P = int(g.choice([64, 128])), int(g.choice([8, 16, 32, 64, 128, 512]))
    lens = [int(g.integers(0, int(g.choice([4, 200, 3000])))) for _ in range(B)]
    tree = [int(g.integers(-1, 3 if seed % 2 else 11)) for _ in range(B)]
    if all(t < 0 for t in tree):
        tree[0] = 1
    begin = [int(g.integers(0, L + 1)) for L in lens] if g.random() < 0.3 else None
    s = Scene(seed, lens, tree, H * group, H, d, P, BF if g.random() < 0.5 else HF, begin=begin)
    window = int(g.choice([0, 0, int(g.integers(1, 600))]))
    slopes = torch.rand(H * group, device="cuda") if g.random() < 0.3 else None
    s.check(bank, window=window, sink=int(g.integers(0, 200)) if window else 0,
            cap=float(g.choice([0.0, 0.0, 5.0, 50.0])), slopes=slopes)


@pytest.mark.parametrize("tree", [(7, 5, 8, 0), (0, 1, 2, 0)])
@pytest.mark.parametrize("cap", [0.01, 0.5, 50.0, 1024.0])
@pytest.mark.parametrize("biased", [False, True])
def test_caps_from_saturated_to_hardly_bent(bank, tree, cap, biased):  # noqa: F811
    """Scores far past the cap in both directions, and caps far past the scores; hidden slots hold NaN."""
    s = Scene(int(cap) + 3, [130, 5, 0, 260], list(tree), 6, 3, 64, 16, q_std=20.0 if cap < 100 else 2.0)
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


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("tree", [3, 1])
@pytest.mark.parametrize("L", [70, 9000])
def test_a_score_that_is_not_finite_shows(bank, form, dtype, tree, L):  # noqa: F811
    """NaN or infinity in a query, the scale NaN in one visible key: output and log-sum-exp of those rows are NaN, in
    units of one CTA and of several, and all others are as they were."""
    s = Scene(L, [L], [tree], 4, 2, 64, 16, dtype=dtype)
    kw = dict(cap=30.0 if form == "cap" else 0.0, slopes=torch.full((4,), 0.02, device="cuda") if form == "bias" else None)
    want, want_lse = s.run(bank, **kw)
    assert np.isfinite(want).all() and np.isfinite(want_lse).all()
    kept = s.q.clone()
    for value in (float("nan"), float("inf")):
        if value == float("inf") and form == "cap":
            continue  # capped: a finite score
        s.q.copy_(kept)
        s.q[1, 1, 5] = value
        got, lse = s.run(bank, **kw)
        assert np.isnan(got[1, 1]).all() and np.isnan(lse[1, 1])
        got[1, 1], lse[1, 1] = want[1, 1], want_lse[1, 1]
        assert np.array_equal(got, want) and np.array_equal(lse, want_lse)
    # one key of head 0, in the prefix: every row of its two query heads
    s.q.copy_(kept)
    s.scales(0, 0, L // 2, 0)[1] = 255
    got, lse = s.run(bank, **kw)
    assert np.isnan(got[:, :2]).all() and np.isnan(lse[:, :2]).all()
    assert np.array_equal(got[:, 2:], want[:, 2:]) and np.array_equal(lse[:, 2:], want_lse[:, 2:])


@pytest.mark.parametrize("trees", [(0, 9, 7, 3, 1), (0, 1, 2, 1, 0)])
@pytest.mark.parametrize("L", [90, 6000])
@pytest.mark.parametrize("window", [0, 3])
def test_a_plan_of_another_bank(bank, trees, L, window):  # noqa: F811
    """Requests whose tree the call's bank lacks, or has with other nodes, are reported and left out, whether one CTA
    has their unit or several; the others are served."""
    s = Scene(L, [L, 40, L, 70, 9], list(trees), 4, 2, 64, 16)
    s.run(bank, window=window)
    at = np.concatenate([[0], np.cumsum(s.n)])

    def left_out(held):
        """held: the bank's trees; a tree is served where it stands at its number with its own nodes."""
        served = [t < len(held) and len(s.trees[held[t]]) == len(s.trees[t]) for t in trees]
        other = tv.Bank(len(held), 0)
        for t in held:
            other.add(s.trees[t])
        ws = tv.make_workspace(tv.tb_workspace_size(0, 1, s.H, s.Hq, s.d, 0, 0))
        out, lse = torch.full_like(s.out, 5.0), torch.full_like(s.lse, 5.0)
        tv.paged_tree_attention_q4(other, s.req, s.pages, s.plan, s.q, out, ws, lse=lse)
        torch.cuda.synchronize()
        assert tv.tb_workspace_status(ws) == (tv.TB_OK if all(served) else tv.TB_EINVAL)
        for b, known in enumerate(served):
            rows = slice(at[b], at[b + 1])
            for got, was in ((out, s.out), (lse, s.lse)):
                assert torch.equal(got[rows], was[rows] if known else torch.full_like(was[rows], 5.0))
        other.close()

    left_out((0, 1, 5, 3))
    left_out((0,))
    left_out((0, 1, 2, 4, 4, 5, 6, 7, 8, 9))
    left_out((0, 2, 1))
    left_out(tuple(range(10)))


@pytest.mark.parametrize("P", [16, 128, 512])
@pytest.mark.parametrize("entry", [-1, -2 ** 31, "past", 2 ** 31 - 1])
@pytest.mark.parametrize("tree", [(5, 3), (0, 1)])
def test_holes_in_the_table(bank, P, entry, tree):  # noqa: F811
    """A page that is not there, where rows look: reported, its keys and values zeros.  Where none looks: nothing."""
    def scene(**kw):
        s = Scene(P, [1700, 300], list(tree), 4, 2, 64, P, **kw)
        s.may_report = True
        return s, s.pages.k.shape[1] if entry == "past" else entry

    def run(s, reported, **kw):
        s.check(bank, **kw)
        assert s.status == (tv.TB_EINVAL if reported else tv.TB_OK)

    for page in (0, 1024 // P, 1699 // P):  # the first page, one in the middle, the last prefix slot's
        s, e = scene()
        s.table[0, page] = e
        for i in range(2):
            s.dense[0][i][page * P:(page + 1) * P] = 0
        run(s, True)
        # with a window of 100 the pages before slot 1601 are looked at by the first tokens' rule alone
        run(s, page * P + P > 1601, window=100)
        run(s, page * P + P > 1601 or page * P < 20, window=100, sink=20)
    # documents that begin behind the hole, at its end, inside it
    for begin, reported in ((1024 + P, False), (1023 + P, True), (1024, True)):
        s, e = scene(begin=[begin, 0])
        s.table[0, 1024 // P] = e
        for i in range(2):
            s.dense[0][i][1024:1024 + P] = 0
        run(s, reported)


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
def test_a_wait_that_runs_out(bank, form, d, dtype):  # noqa: F811
    # units of several CTAs (one long request), of one, several in one CTA, few rows and many
    lens = [9000, 100, 0, 400] + [30] * 300
    tree = [7, 5, 8, -1] + [0, 2, 3] * 100
    s = Scene(d, lens, tree, 4, 2, d, 16, dtype=dtype)
    s.run(bank, cap=30.0 if form == "cap" else 0.0,
          slopes=torch.full((4,), 0.02, device="cuda") if form == "bias" else None)
    want = [s.out.clone(), s.lse.clone()]
    s.out.fill_(5.0), s.lse.fill_(5.0)
    t0 = time.time()
    s.layer = tv.TB_DEBUG_EXPIRE_WAIT
    s.call()
    torch.cuda.synchronize()
    assert time.time() - t0 < 20.0
    assert tv.tb_workspace_status(s.ws) == tv.TB_ETIMEOUT
    assert bool((s.out == 5).all()) and bool((s.lse == 5).all())
    tv.tb_workspace_init(s.ws)
    s.layer = 0
    s.call()
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_OK
    assert torch.equal(s.out, want[0]) and torch.equal(s.lse, want[1])

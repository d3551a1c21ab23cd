"""The attention over 4-bit pages where units have few rows (single tokens, short chains): the way through the
kernel that it takes for up to 8 rows per kv head in CTAs of more than two tiles, against 64 bits.  Every case is
made as large as this GPU's SMs need for that, and looks into the step's plan that its CTAs do go that way."""
import os
import re
import threading
import time

import numpy as np
import pytest
import torch

import paged_reference as ref
import paper_2606_27550_gb300 as tv
import q4_reference as q4
from paper_2606_27550_gb300 import synth
from test_gpu_paged_attention import BF, HF, bank, i32  # noqa: F401
from test_gpu_paged_attention_q4 import MODES, mode_args
from test_gpu_paged_attention_q4 import Scene as SceneQ4

pytestmark = pytest.mark.gpu

TILE, MAX_CTAS = 128, 512
REQ = np.dtype([("base", "i8"), *((x, "i4") for x in ("L", "n", "row0", "tree", "T", "a0", "n1", "b0", "begin", "far_end",
                                                        "b", "pad"))])
CTA = np.dtype([("t0", "i8"), ("t1", "i8"), ("rb", "i4"), ("idx", "i4"), ("req", REQ)])


def rule():
    """(rows of a unit at most, tiles of a CTA that are too few), from the kernel's source."""
    path = os.path.join(os.path.dirname(tv.__file__), "csrc", "paged_attention_few.cuh")
    with open(path) as f:
        text = f.read()
    return tuple(int(re.search(rf"{name} = (\d+);", text)[1]) for name in ("kFewRows", "kFewTiles"))


def ways(plan, group):
    """[(few, t0, t1, begins inside a unit)] of a plan's CTAs that have tiles."""
    rows_max, too_few = rule()
    raw = plan.cpu().numpy()
    ctas = raw[64:64 + MAX_CTAS * CTA.itemsize].view(CTA)
    reqs = raw[64 + MAX_CTAS * (CTA.itemsize + 32):]
    reqs = reqs[:len(reqs) // REQ.itemsize * REQ.itemsize].view(REQ)
    out = []
    for c in ctas[:torch.cuda.get_device_properties(0).multi_processor_count]:
        if c["t1"] <= c["t0"]:
            continue
        rows, i = 0, int(c["idx"])
        while reqs[i]["base"] < c["t1"]:  # (behind the last request a record that begins at the end)
            rows = max(rows, int(reqs[i]["n"]) * group - int(c["rb"]) * 128)
            i += 1
        inside = (int(c["t0"]) - int(c["req"]["base"])) % int(c["req"]["T"]) != 0
        out.append((rows <= rows_max and c["t1"] - c["t0"] > too_few, int(c["t0"]), int(c["t1"]), inside))
    return out


def tiles_of(L, n, begin, window, sink):
    """Key tiles of a request: what its rows may see, the kept first tokens apart from the window if they lie apart."""
    if n == 0:
        return 0
    end = L + n
    lo = max(begin, L - window + 1) if window else begin
    first, kept = min(lo, end - 1) // TILE, 0
    far = min(begin + sink, lo)
    if window and far > begin:
        a0, a1 = begin // TILE, -(-far // TILE)
        if a1 >= first:
            first = a0
        else:
            kept = a1 - a0
    return kept + (end - 1) // TILE - first + 1


def fill(lens, tree, H, per_cta=3, begin=None, window=0, sink=0):
    """(lens, tree, begin) repeated, each time a little longer, until every SM has per_cta tiles and one more."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    nodes = [0 if t < 0 else len(ref.trees()[t]) for t in range(-1, 11)]
    out, total, i = ([], [], []), 0, 0
    while total < sms * per_cta + sms // 2:
        k, again = i % len(lens), i // len(lens)
        L, t, b = lens[k] + 5 * again, tree[k], begin[k] if begin else 0
        n = nodes[t + 1]
        b = min(b, L + n)
        total += H * tiles_of(L, n, b, window, sink)
        for x, y in zip(out, (L, t, b)):
            x.append(y)
        i += 1
    return out[0], out[1], out[2] if begin else None


def attend64(q, k, v, parent, L, scale, cap, slopes, window, sink, begin):
    """(out, lse, |V| average, largest |z| that matters) of one request, all heads at once in 64 bits (torch)."""
    n, Hq, d = q.shape
    H = k.shape[1]
    dep = torch.as_tensor(np.asarray(synth.depth_of(parent)), device="cuda").long()
    s = torch.arange(L + n, device="cuda")
    pos = torch.cat([s[:L], L + dep])
    dist = (L + dep)[:, None] - pos[None]
    see = torch.cat([torch.ones(n, L, dtype=torch.bool, device="cuda"),
                     torch.as_tensor(ref.ancestors(parent), device="cuda")], 1)
    if window:
        see &= (dist < window) | (s < begin + sink)
    see &= s >= begin
    see = see[:, None, None]
    z = torch.einsum("nhgd,khd->nhgk", q.view(n, H, Hq // H, d), k) * scale
    if cap:
        z = cap * torch.tanh(z / cap)
    if slopes is not None:
        z = z - slopes.double().view(H, Hq // H, 1) * dist[:, None, None].double()
    z = torch.where(see, z, -torch.inf)
    m = z.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
    p = torch.exp(z - m)
    total = p.sum(-1, keepdim=True)
    w = torch.where(total > 0, p / total, 0.0)
    out, absv = (torch.einsum("nhgk,khd->nhgd", w, x).reshape(n, Hq, d) for x in (v, v.abs()))
    big = torch.where(p > 2.0 ** -30, z.abs(), 0.0).amax(-1).reshape(n, Hq)
    return out, (m + total.log()).reshape(n, Hq), absv, big


class Scene(SceneQ4):
    """A 4-bit scene (every slot that no row may see has the scale NaN and any codes) that has to go the few-row way:
    all of its CTAs, or (some_few) some of them.  Keys and values of all requests are made at once and stay on the GPU."""

    some_few = False

    def __init__(self, seed, lens, tree, Hq, H, d, P=16, dtype=BF, layers=1, layer=0, begin=None, q_std=1.5, n_extra=0):
        torch.manual_seed(seed)
        g = synth.rng(seed)
        self.trees = ref.trees()
        self.lens, self.tree, self.P, self.H, self.Hq, self.d, self.dtype = lens, tree, P, H, Hq, d, dtype
        self.begin, self.layer = begin, layer
        self.n = [0 if t < 0 else len(self.trees[t]) for t in tree]
        self.R = sum(self.n)
        ends = np.add(lens, self.n)
        counts = -(-ends // P)
        n_pages = n_extra + int(counts.sum()) + 2
        ids = n_extra + g.permutation(n_pages - n_extra)  # the pool's last pages
        table = np.full((len(lens), int(counts.max()) + 1), -1, np.int32)
        table[np.arange(table.shape[1])[None] < counts[:, None]] = ids[:counts.sum()]
        self.table = torch.from_numpy(table).cuda()
        request = np.repeat(np.arange(len(lens)), ends)
        first = np.concatenate([[0], np.cumsum(ends)])
        slot = np.arange(len(request)) - first[request]
        page, at = (torch.from_numpy(x).cuda() for x in (table[request, slot // P].astype(np.int64), slot % P))
        there = torch.from_numpy(slot >= np.array(begin if begin else [0] * len(lens))[request]).cuda()
        pools, rows = [], []
        for _ in range(2):
            pool = torch.empty((layers, n_pages, H, tv.q4_page_bytes(P, d)), dtype=torch.uint8, device="cuda")
            codes, scales = q4.parts(pool, P, d)
            codes[:, n_extra:].random_(0, 256)
            scales[:, n_extra:] = 255
            c = (torch.randn(len(request), H, d, device="cuda") * 2.5).round().clamp(-7, 7)
            byte = torch.randint(0x60, 0x6D, (len(request), H, d // 32), device="cuda")
            c8 = (c + 8).to(torch.uint8)
            codes[layer].transpose(1, 2)[page[there], at[there]] = (c8[..., 0::2] | (c8[..., 1::2] << 4))[there]
            scales[layer].transpose(1, 2)[page[there], at[there]] = byte.to(torch.uint8)[there]
            s = torch.from_numpy(q4.scale_value(np.arange(0x6D))).float().cuda()[byte]
            pools.append(pool)
            rows.append(c * s.repeat_interleave(32, -1))  # 7 bits: exact
        self.dense = [[x[first[b]:first[b + 1]] for x in rows] for b in range(len(lens))]
        self.pages = tv.PagesQ4(*pools, P, d, dtype)
        self.q = (q_std * torch.randn(self.R, Hq, d, device="cuda")).to(dtype)

    def run(self, bank, *args, **kw):  # noqa: F811
        out = super().run(bank, *args, **kw)
        found = [few for few, *_ in ways(self.plan, self.Hq // self.H)]
        assert any(found) and (self.some_few or all(found)), f"{sum(found)} of {len(found)} CTAs"
        return out

    def check(self, bank, window=0, sink=0, cap=0.0, slopes=None, scale=None, extra_rows=0, cap_error=False):  # noqa: F811
        """As the scene of any rows is checked: weights and outputs are each rounded once to the type, 2^-12 for the
        32-bit steps, and a score of size z carries a rounding of 2^-22 z into its weight.  cap_error: also the
        documented cap 2^-20 of every score (once in the weight, once in the sum)."""
        self.run(bank, window, sink, cap, slopes, scale, extra_rows=extra_rows)
        self.compare(window, sink, cap, slopes, scale, cap_error)

    def compare(self, window=0, sink=0, cap=0.0, slopes=None, scale=None, cap_error=False, lens=None):
        eps = 2.0 ** -8 if self.dtype == BF else 2.0 ** -11
        q, out, lse = (x.double() for x in (self.q, self.out, self.lse))
        at, fine = 0, []
        for b, n in enumerate(self.n):
            if n == 0:
                continue
            L = self.lens[b] if lens is None else lens[b]
            k, v = (x[:L + n].double() for x in self.dense[b])
            rows = slice(at, at + n)
            at += n
            o, ls, absv, big = attend64(q[rows], k, v, self.trees[self.tree[b]], L, self.d ** -0.5 if scale is None else scale,
                                        cap, slopes, window, sink, self.begin[b] if self.begin else 0)
            z = 2.0 ** -21 * big[..., None]
            if cap_error:
                z = 2 * (z + 2.0 ** -20 * cap)
            bound = eps * o.abs() + (eps + 2.0 ** -12 + z) * absv + 1e-7
            empty = torch.isneginf(ls)
            tol = 1e-5 + 2.0 ** -21 * torch.maximum(ls.abs(), big) + (2.0 ** -20 * cap if cap_error else 0.0)
            fine.append(torch.stack([
                ((out[rows] - o).abs() <= bound).all(), ((lse[rows] - ls).abs() <= tol)[~empty].all(),
                torch.isneginf(lse[rows])[empty].all(), (out[rows][empty] == 0).all()]))
        fine = torch.stack(fine).cpu()
        assert bool(fine.all()), f"requests with rows, by (output, lse, lse of empty rows, output of empty rows): {fine.tolist()}"


# lengths about the sizes of pieces and tiles; a slot without a request
LENS = [0, 1, 7, 15, 16, 300, 17, 31, 32, 33, 63, 96, 127, 128, 129, 255, 256, 511, 640, 1000, 2500]


# trees by number: 0..3 of 1, 2, 4 and 8 nodes
@pytest.mark.parametrize("Hq,H,d,P,dtype,nodes,per_cta", [
    (8, 8, 128, 8, BF, (0, 1, 2), 5), (8, 8, 128, 16, HF, (3, 0), 3), (16, 8, 128, 32, BF, (0, 1, 2), 21),
    (32, 8, 128, 64, HF, (0, 1), 9), (32, 4, 128, 128, BF, (0,), 6), (12, 4, 128, 256, HF, (0, 1), 4),
    (21, 3, 128, 512, BF, (0,), 7), (8, 8, 128, 1024, HF, (0, 2), 30), (16, 4, 64, 8, HF, (0, 1), 4),
    (8, 8, 64, 16, BF, (3, 1), 9), (24, 6, 64, 32, HF, (0, 1), 32), (16, 2, 64, 64, BF, (0,), 3),
    (6, 6, 64, 128, HF, (3,), 7), (10, 2, 64, 256, BF, (0,), 5), (8, 4, 64, 512, HF, (0, 2), 11),
    (5, 5, 64, 1024, BF, (1, 2), 16)])
@pytest.mark.parametrize("mode", MODES)
def test_forms(bank, Hq, H, d, P, dtype, nodes, per_cta, mode):  # noqa: F811
    kw = mode_args(mode, Hq)
    tree = [nodes[i % len(nodes)] for i in range(len(LENS))]
    tree[5] = -1
    # (a window leaves a tile or two of each request)
    lens, tree, _ = fill(LENS, tree, H, min(per_cta, 5) if kw["window"] else per_cta, window=kw["window"], sink=kw["sink"])
    Scene(Hq + P, lens, tree, Hq, H, d, P, dtype).check(bank, **kw)


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (2, 130), (5, 0), (64, 4), (128, 128), (129, 300), (2000, 7),
                                         (400, 257)])
@pytest.mark.parametrize("d,P,dtype", [(128, 16, BF), (64, 64, HF)])
def test_windows(bank, window, sink, d, P, dtype):  # noqa: F811
    """Windows shorter than the chain, ends inside and at tiles, first tokens that meet the window."""
    lens, tree, _ = fill([700, 3, 128, 1500, 0, 255, 384], [0, 1, 2, 2, 0, 0, 1], 8, window=window, sink=sink)
    Scene(window + sink, lens, tree, 16, 8, d, P, dtype).check(bank, window=window, sink=sink)


@pytest.mark.parametrize("window,sink", [(0, 0), (60, 0), (60, 20)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (128, HF), (64, BF)])
def test_documents_that_begin_late_and_rows_that_see_nothing(bank, window, sink, d, dtype):  # noqa: F811
    lens, tree, begin = fill([300, 40, 256, 500, 130, 0, 64, 900], [0, 1, 2, 2, 0, 1, 2, 3], 8,
                             begin=[77, 40, 128, 0, 131, 3, 200, 897], window=window, sink=sink)
    Scene(90 + sink, lens, tree, 8, 8, d, 16, dtype, begin=begin).check(bank, window=window, sink=sink)


@pytest.mark.parametrize("d,dtype", [(128, HF), (64, BF)])
def test_large_scores(bank, d, dtype):  # noqa: F811
    """Scores of several hundred, increasing along the keys so that the running maximum keeps growing, or falling."""
    lens, tree, _ = fill([900], [1], 4, per_cta=6)
    s = Scene(11, lens, tree, 8, 4, d, 16, dtype, q_std=1.0)
    codes, scales = q4.parts(s.pages.k, 16, d)
    for b, (L, n) in enumerate(zip(lens, s.n)):
        # key r: 7 s_r in the first element, s_r a power of two times 8 to 15 sixteenths
        slot = torch.arange(L + n, device="cuda")
        page, at = s.table[b].long()[slot // 16], slot % 16
        byte = (0x50 + slot * 60 // (L + n)).to(torch.uint8)
        scales[0].transpose(1, 2)[page, at, :, 0] = byte[:, None]
        codes[0].transpose(1, 2)[page, at, :, 0] = 0x8F  # 7 and 0
        codes[0].transpose(1, 2)[page, at, :, 1:16] = 0x88
        s.dense[b][0][:, :, :32] = 0
        s.dense[b][0][:, :, 0] = 7 * torch.from_numpy(q4.scale_value(byte.cpu().numpy())).float().cuda()[:, None]
    for x in (8.0, -8.0):
        s.q[..., 0] = x
        s.check(bank)


@pytest.mark.parametrize("cap", [0.01, 0.5, 50.0, 1024.0])
@pytest.mark.parametrize("biased", [False, True])
def test_caps_from_saturated_to_hardly_bent(bank, cap, biased):  # noqa: F811
    lens, tree, _ = fill([130, 5, 0, 260], [0, 1, 2, 0], 8)
    s = Scene(int(cap) + 3, lens, tree, 16, 8, 128, 16, BF if cap < 1 else HF, q_std=20.0 if cap < 100 else 2.0)
    s.check(bank, cap=cap, slopes=torch.full((16,), 0.05, device="cuda") if biased else None, cap_error=True)


def test_many_units_per_warp(bank):  # noqa: F811
    """More units of one tile in a warp's run, a 16th of its CTA's tiles, than the 8 that it lays out at a time."""
    B = 8 * torch.cuda.get_device_properties(0).multi_processor_count
    s = Scene(6, [i % 90 for i in range(B)], ([0, 0, 0, 1, -1, 0] * B)[:B], 40, 20, 128, 16, HF)
    s.check(bank)
    found = ways(s.plan, 2)
    assert min(t1 - t0 for _, t0, t1, _ in found) > 16 * 8


@pytest.mark.parametrize("L,Hq,H,tree", [(70000, 8, 1, 0), (30000, 16, 4, 1), (131000, 4, 2, 2)])
@pytest.mark.parametrize("d,dtype", [(128, BF), (128, HF), (64, BF)])
def test_long_units_are_split(bank, L, Hq, H, tree, d, dtype):  # noqa: F811
    lens, trees, _ = fill([L], [tree], H)
    Scene(L, lens, trees, Hq, H, d, 64, dtype).check(bank, cap=20.0)
    kw = dict(window=L // 2, sink=300)
    lens, trees, _ = fill([L], [tree], H, **kw)
    Scene(L + 1, lens, trees, Hq, H, d, 64, dtype).check(bank, **kw)


@pytest.mark.parametrize("d,dtype", [(128, BF), (128, HF), (64, HF)])
def test_units_that_few_row_and_many_row_ctas_share(bank, d, dtype):  # noqa: F811
    """A tree between long chains: the CTAs at the tree go the other way, and join the chains' units with the others."""
    s = Scene(31, [30000, 700, 21000, 500, 26000], [1, 5, 0, 7, 2], 8, 4, d, 32, dtype)
    s.some_few = True
    s.check(bank)
    found = ways(s.plan, 2)
    shared = [(a[0], b[0]) for a, b in zip(found, found[1:]) if b[3]]
    assert (True, False) in shared and (False, True) in shared
    s.check(bank, cap=30.0, window=12000, sink=500)


@pytest.mark.parametrize("d", [64, 128])
def test_layers_strides_and_side_by_side_pools(bank, d):  # noqa: F811
    """K and V in one tensor, layers innermost, gaps between the heads; the second of three layers."""
    lens, tree, _ = fill([200, 90, 350], [0, 1, 0], 4)
    s = Scene(77, lens, tree, 8, 4, d, 16, layers=3, layer=1)
    n, size = s.pages.k.shape[1], tv.q4_page_bytes(16, d)
    both = torch.full((n, 4, 2, 3, size + 48), 255, dtype=torch.uint8, device="cuda")
    for i, x in enumerate((s.pages.k, s.pages.v)):
        both[:, :, i, :, :size] = x.permute(1, 2, 0, 3)
    s.pages = tv.PagesQ4(*(both[:, :, i, :, :size].permute(2, 0, 1, 3) for i in range(2)), 16, d, BF)
    s.check(bank)


def test_rows_past_the_batch_and_scale(bank):  # noqa: F811
    lens, tree, _ = fill([100, 0, 330], [0, -1, 1], 8)
    Scene(15, lens, tree, 16, 8, 128, 16).check(bank, scale=0.3, extra_rows=9)


@pytest.mark.parametrize("lens,tree,keep", [([20000, 40, 9000], (0, 1, 2), 2), ([9000, 20000, 300], (2, 1, 0), 5)])
def test_fewer_rows_than_the_plan_has(bank, lens, tree, keep):  # noqa: F811
    """Rows of the plan past the call's n_rows are left out, in whole units and in split ones."""
    lens, tree, _ = fill(lens, tree, 2)
    s = Scene(16, lens, tree, 4, 2, 128, 16, HF)
    s.run(bank)
    out, lse = torch.full_like(s.out, 3.0), torch.full_like(s.lse, 3.0)
    tv.paged_tree_attention_q4(bank, s.req, s.pages, s.plan, s.q[:keep], out[:keep], s.ws, lse=lse[:keep])
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_OK
    assert torch.equal(out[:keep], s.out[:keep]) and torch.equal(lse[:keep], s.lse[:keep])
    assert bool((out[keep:] == 3).all()) and bool((lse[keep:] == 3).all())


@pytest.mark.parametrize("d,dtype", [(128, BF), (64, HF)])
def test_offsets_past_32_bits(bank, d, dtype):  # noqa: F811
    lens, tree, _ = fill([300, 700], [0, 1], 4)
    n = (1 << 32) // (4 * tv.q4_page_bytes(128, d)) + 40
    s = Scene(19, lens, tree, 8, 4, d, 128, dtype, n_extra=n)
    assert s.pages.k.stride(1) * n > 2**32
    s.check(bank)


def test_streams_graphs_repeats_and_threads(bank):  # noqa: F811
    lens, tree, _ = fill([600, 4000, 20], [0, 1, 0], 4, per_cta=7)
    scenes = [Scene(23 + i, lens, tree, 8, 4, 128, 32) for i in range(2)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for s in scenes:
            s.check(bank, cap=30.0)
    side.synchronize()
    firsts = [(s.out.clone(), s.lse.clone()) for s in scenes]
    s, first = scenes[0], firsts[0]
    for _ in range(5):
        s.out.zero_()
        s.call()
        torch.cuda.synchronize()
        assert torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    s.out.zero_(), s.lse.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])
    failed = []

    def work(s, first):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    s.out.zero_(), s.lse.zero_()
                    s.call()
                    torch.cuda.current_stream().synchronize()
                    if not (torch.equal(s.out, first[0]) and torch.equal(s.lse, first[1])):
                        failed.append(s)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=x) for x in zip(scenes, firsts)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_a_replayed_graph_follows_the_lengths(bank):  # noqa: F811
    """Plan and attention captured once: lengths grow and shrink between replays, from and to CTAs of too few tiles."""
    lens, tree, _ = fill([900, 300, 2000, 40], [0, 1, 2, 0], 4, per_cta=5)
    s = Scene(24, lens, tree, 8, 4, 128, 16)
    s.run(bank)
    slots, pos = torch.empty(s.R, dtype=torch.int64, device="cuda"), torch.empty(s.R, dtype=torch.int32, device="cuda")
    status = torch.empty(len(lens), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tv.paged_plan(bank, s.req, slots, pos, status, s.plan, n_q_heads=8, n_kv_heads=4)
        s.call()
    seen = set()
    for f in (1.0, 0.7, 0.1, 0.9, 0.0):
        now = [int(L * f) for L in lens]
        s.req.lens.copy_(i32(now))
        s.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert status.tolist() == [0] * len(lens) and tv.tb_workspace_status(s.ws) == tv.TB_OK
        seen.add(all(few for few, *_ in ways(s.plan, 2)))
        # the tree's keys and values are those that lie behind the shorter prefix
        s.compare(lens=now)
    assert seen == {True, False}


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("d,dtype", [(128, BF), (128, HF), (64, BF)])
@pytest.mark.parametrize("long", [False, True])
def test_a_score_that_is_not_finite_shows(bank, form, d, dtype, long):  # noqa: F811
    """NaN or infinity in a query, the scale NaN in one visible key: output and log-sum-exp of those rows are NaN, in
    units of one CTA and of several, and all others are as they were."""
    lens, tree, _ = fill([31000] if long else [70, 300], [1] if long else [1, 0], 4)
    s = Scene(len(lens), lens, tree, 8, 4, d, 16, dtype)
    kw = dict(cap=30.0 if form == "cap" else 0.0, slopes=torch.full((8,), 0.02, device="cuda") if form == "bias" else None)
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
    # one key of head 0 of the first request, in the prefix: both rows of its two query heads
    s.q.copy_(kept)
    s.scales(0, 0, lens[0] // 2, 0)[1] = 255
    got, lse = s.run(bank, **kw)
    assert np.isnan(got[:2, :2]).all() and np.isnan(lse[:2, :2]).all()
    got[:2, :2], lse[:2, :2] = want[:2, :2], want_lse[:2, :2]
    assert np.array_equal(got, want) and np.array_equal(lse, want_lse)


@pytest.mark.parametrize("L", [90, 9000])
@pytest.mark.parametrize("window", [0, 3])
def test_a_plan_of_another_bank(bank, L, window):  # noqa: F811
    """Requests whose tree the call's bank lacks, or has with other nodes, are reported and left out, whether one CTA
    has their unit or several; the others are served."""
    lens, trees, _ = fill([L, 40, L, 70, 9], [0, 1, 2, 1, 0], 8, window=window)
    s = Scene(L, lens, trees, 16, 8, 128, 16)
    s.run(bank, window=window)
    for held in ((0, 1, 5), (0,), (0, 2, 1), (0, 1, 2)):
        served = [t < len(held) and len(s.trees[held[t]]) == len(s.trees[t]) for t in trees]
        other = tv.Bank(len(held), 0)
        for t in held:
            other.add(s.trees[t])
        ws = tv.make_workspace(tv.tb_workspace_size(0, 1, s.H, s.Hq, s.d, 0, 0))
        out, lse = torch.full_like(s.out, 5.0), torch.full_like(s.lse, 5.0)
        tv.paged_tree_attention_q4(other, s.req, s.pages, s.plan, s.q, out, ws, lse=lse)
        torch.cuda.synchronize()
        assert tv.tb_workspace_status(ws) == (tv.TB_OK if all(served) else tv.TB_EINVAL)
        keep = torch.tensor(np.repeat(served, s.n), device="cuda")
        assert torch.equal(out[keep], s.out[keep]) and torch.equal(lse[keep], s.lse[keep])
        assert bool((out[~keep] == 5).all()) and bool((lse[~keep] == 5).all())
        other.close()


@pytest.mark.parametrize("P,entry", [(8, -1), (32, "past"), (128, 2 ** 31 - 1), (512, -2 ** 31)])
def test_holes_in_the_table(bank, P, entry):  # noqa: F811
    """A page that is not there, where rows look: reported, its keys and values zeros.  Where none looks: nothing."""
    def scene(window=0, sink=0, first=0, **kw):
        begin = [first, 0] if first else None
        lens, tree, begin = fill([1700, 300], [0, 1], 8, begin=begin, window=window, sink=sink)
        if begin:
            begin[2:] = [0] * (len(begin) - 2)
        s = Scene(P, lens, tree, 8, 8, 128 if P != 32 else 64, P, HF if P == 8 else BF, begin=begin)
        s.may_report = True
        return s, s.pages.k.shape[1] if entry == "past" else entry

    def hole(s, e, page):
        s.table[0, page] = e
        for i in range(2):
            s.dense[0][i][page * P:(page + 1) * P] = 0

    def run(s, reported, **kw):
        s.check(bank, **kw)
        assert s.status == (tv.TB_EINVAL if reported else tv.TB_OK)

    for page in (0, 1024 // P, 1699 // P):  # the first page, one in the middle, the last prefix slot's
        s, e = scene()
        hole(s, e, page)
        run(s, True)
        for sink in (0, 20):
            # with a window of 100 the pages before slot 1601 are looked at by the first tokens' rule alone
            s, e = scene(window=100, sink=sink)
            hole(s, e, page)
            run(s, page * P + P > 1601 or page * P < sink, window=100, sink=sink)
    for first, reported in ((1024 + P, False), (1023 + P, True), (1024, True)):
        s, e = scene(first=first)
        hole(s, e, 1024 // P)
        run(s, reported)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(bank, seed):  # noqa: F811
    g = synth.rng(5000 + seed)
    group = int(g.choice([1, 1, 2, 3, 4, 8]))
    H = int(g.choice([1, 2, 3, 4, 8]))
    d, P = int(g.choice([64, 128])), int(g.choice([8, 16, 32, 64, 128, 256, 512, 1024]))
    most = int(np.searchsorted([1, 2, 4, 8], 8 // group, side="right"))  # trees of at most 8 rows
    window = int(g.choice([0, 0, int(g.integers(1, 600))]))
    sink = int(g.integers(0, 200)) if window else 0
    reach = int(g.choice([200, 1200] if window else [200, 3000, 20000]))
    B = int(g.integers(3, 40))
    lens = [int(g.integers(0, reach)) for _ in range(B)]
    tree = [0] + [int(g.integers(-1, most)) for _ in range(B - 1)]
    begin = [int(g.integers(0, L + 1)) for L in lens] if g.random() < 0.3 else None
    lens, tree, begin = fill(lens, tree, H, int(g.choice([3, 4, 7, 12])), begin, window, sink)
    s = Scene(seed, lens, tree, H * group, H, d, P, BF if g.random() < 0.5 else HF, begin=begin)
    slopes = torch.rand(H * group, device="cuda") if g.random() < 0.3 else None
    s.check(bank, window=window, sink=sink, cap=float(g.choice([0.0, 0.0, 5.0, 50.0])), slopes=slopes)


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
def test_a_wait_that_runs_out(bank, form, d, dtype):  # noqa: F811
    """All CTAs go the few-row way: units of several CTAs, of one, of one warp."""
    lens, tree, _ = fill([9000, 100, 0, 400] + [30] * 40, [1, 0, 2, -1] + [0, 1] * 20, 4, per_cta=6)
    s = Scene(d, lens, tree, 8, 4, d, 16, dtype)
    s.run(bank, cap=30.0 if form == "cap" else 0.0,
          slopes=torch.full((8,), 0.02, device="cuda") if form == "bias" else None)
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

"""logits_process: processed logits bit for bit against the documented 32-bit
steps, statistics against 64 bits."""
import numpy as np
import pytest
import torch

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


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def pack_bits(allowed):
    n, V = allowed.shape
    words = -(-V // 32)
    full = np.zeros((n, words * 32), bool)
    full[:, :V] = allowed
    return np.packbits(full, axis=1, bitorder="little").view(np.uint32).view(np.int32)


class Scene:
    def __init__(self, seed, tree, V, dtype=torch.float32, hist_max=300, pad=0, mask_share=0.7, biases=5, free_rows=None):
        g = self.g = synth.rng(seed)
        self.trees, self.tree, self.V = ref.trees(), tree, V
        B = len(tree)
        self.n = free_rows or [0 if t < 0 else len(self.trees[t]) for t in tree]
        self.start = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        R = self.R = int(self.start[-1])
        z = (3 * g.standard_normal((R, V + pad))).astype(np.float32)
        if R and V > 40:
            z[:, 7] = z[:, 30] = z.max() + 1  # ties: the lowest index
        self.logits = dev(z, dtype)[:, :V]
        self.z = self.logits.float().cpu().numpy()
        self.hist = g.integers(-2, max(1, min(V, 50)) + 2, (B, hist_max)).astype(np.int32)
        self.hist_len = g.integers(0, hist_max + 1, B).astype(np.int32)
        self.hist_len[0] = 0
        self.prompt = np.array([g.integers(0, x + 1) for x in self.hist_len], np.int32)
        self.draft = g.integers(-1, max(1, min(V, 60)) + 1, R).astype(np.int32)
        self.rep = (1 + g.random(B)).astype(np.float32)
        self.pres, self.freq = g.standard_normal(B).astype(np.float32), g.standard_normal(B).astype(np.float32)
        counts = g.integers(0, biases * 2 + 1, B)
        self.bstart = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.btok = g.integers(-1, V + 1, self.bstart[-1]).astype(np.int32)
        self.bval = (5 * g.standard_normal(self.bstart[-1])).astype(np.float32)
        self.allowed = g.random((R, V)) < mask_share
        if R > 2:
            self.allowed[1] = False  # a row without an allowed token
        self.T = 0.7

    def run(self, bank, rules=("history", "penalty", "bias", "mask", "draft"), in_place=False, mask_row=None, out_pad=0):
        B, R, V = len(self.tree), self.R, self.V
        trees = None if bank is None else dev(np.array(self.tree, np.int32))
        req = tv.Requests(row_start=dev(self.start), tree=trees)
        out = self.logits if in_place else torch.empty((R, V + out_pad), device="cuda")[:, :V]
        ws = tv.make_workspace(tv.tb_logits_workspace_size(B, R, V))
        kw = {}
        if "history" in rules:
            kw.update(history=dev(self.hist), history_len=dev(self.hist_len), prompt_len=dev(self.prompt))
        if "penalty" in rules:
            kw.update(repetition=dev(self.rep), presence=dev(self.pres), frequency=dev(self.freq))
        if "bias" in rules:
            kw.update(bias_start=dev(self.bstart), bias_token=dev(self.btok), bias_value=dev(self.bval))
        if "draft" in rules:
            kw.update(draft=dev(self.draft))
        allowed = None
        if "mask" in rules:
            allowed = self.allowed
            bits = pack_bits(allowed)
            if mask_row is not None:
                kw.update(mask_row=dev(mask_row))
                allowed = np.where(mask_row[:, None] >= 0, allowed[mask_row.clip(0)], True)
            kw.update(mask=dev(bits))
        st = {k: torch.full((R,), 55, dtype=torch.int32 if k == "argmax" else torch.float32, device="cuda")
              for k in ("argmax", "top1", "entropy", "logz_t", "entropy_t")}
        if "draft" in rules and bank is not None:
            st["draft_logit"] = torch.full((R,), 55.0, device="cuda")
        self.call = lambda: tv.logits_process(bank, req, self.logits, out, ws, temperature=self.T, **kw, **st)
        self.out, self.st = out, st
        self.call()
        torch.cuda.synchronize()
        self.check(rules, bank is not None, allowed)
        return ws

    def check(self, rules, with_trees, allowed):
        out = self.out.cpu().numpy()
        for b in range(len(self.tree)):
            lo, hi = self.start[b], self.start[b + 1]
            if lo == hi:
                continue
            h = self.hist[b, :self.hist_len[b]].tolist() if "history" in rules else []
            paths = [[] for _ in range(hi - lo)]
            parent = None
            if with_trees and self.tree[b] >= 0:
                parent = self.trees[self.tree[b]]
                if "draft" in rules:
                    anc = ref.ancestors(parent)
                    paths = [[int(self.draft[lo + j]) for j in range(1, len(parent)) if anc[i, j]]
                             for i in range(hi - lo)]
            pen = "penalty" in rules
            bias = list(zip(self.btok[self.bstart[b]:self.bstart[b + 1]], self.bval[self.bstart[b]:self.bstart[b + 1]]))
            want = ref.process(self.z[lo:hi], self.rep[b] if pen else 1, self.freq[b] if pen else 0,
                               self.pres[b] if pen else 0, h[:self.prompt[b]], h[self.prompt[b]:], paths,
                               bias if "bias" in rules else [], None if allowed is None else allowed[lo:hi])
            got = out[lo:hi]
            assert np.array_equal(got, want), f"request {b}: {np.argwhere(got != want)[:4]}"
            st = {k: v.cpu().numpy() for k, v in self.st.items()}
            for i in range(hi - lo):
                a, top1, ent, lz, et = ref.stats(want[i], self.T)
                assert st["argmax"][lo + i] == a
                # sums of 2^17 terms and fewer, exponents to 2^-24 of up to 40 each: 1e-5 relative
                assert abs(st["top1"][lo + i] - top1) <= 1e-5 * top1
                assert abs(st["entropy"][lo + i] - ent) <= 3e-5 * (1 + ent)
                assert abs(st["entropy_t"][lo + i] - et) <= 3e-5 * (1 + et)
                if a < 0:
                    assert st["logz_t"][lo + i] == -np.inf
                else:
                    assert abs(st["logz_t"][lo + i] - lz) <= 2e-5 + 1e-6 * abs(lz)
            if "draft_logit" in st:
                for j in range(hi - lo):
                    tok = int(self.draft[lo + j])
                    if parent is None or j == 0 or not 0 <= tok < self.V:
                        assert st["draft_logit"][lo + j] == 55
                    else:
                        assert st["draft_logit"][lo + j] == want[parent[j]][tok]


@pytest.mark.parametrize("V", [1, 2, 31, 33, 255, 257, 1000, 4099, 32000, 50001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rules_and_statistics(bank, V, dtype):
    Scene(V, [5, -1, 0, 8, 3], V, dtype).run(bank)


@pytest.mark.parametrize("rules", [(), ("history",), ("penalty",), ("history", "penalty"), ("bias",), ("mask",),
                                   ("draft",), ("draft", "penalty"), ("mask", "draft", "penalty")])
def test_each_rule_alone(bank, rules):
    Scene(len(rules) + 70, [7, 9], 3001).run(bank, rules)


def test_many_requests_and_large_chunks(bank):
    g = synth.rng(4)
    Scene(5, [int(g.integers(-1, 4)) for _ in range(150)], 5003, hist_max=900, biases=40).run(bank)


def test_large_vocabulary(bank):
    Scene(6, [5, 10, 0, 7], 128256, hist_max=4000, biases=200).run(bank)
    Scene(7, [3] * 5, 152064, torch.bfloat16).run(bank)


def test_rows_without_trees_and_more_than_a_tree_has(bank):
    Scene(8, [-1, -1, -1], 2000, free_rows=[1, 200, 0]).run(None, ("history", "penalty", "bias", "mask"))


def test_in_place_strided_and_shared_masks(bank):
    Scene(9, [5, 4], 4099).run(bank, in_place=True)
    Scene(10, [5, 4], 999, pad=7).run(bank, in_place=True)
    Scene(11, [5, 4], 2048, pad=5).run(bank, out_pad=3)
    s = Scene(12, [5, 4], 700)
    s.run(bank, mask_row=s.g.integers(-1, 3, s.R).astype(np.int32))


def test_duplicates_add_up_in_list_order(bank):
    s = Scene(13, [2], 100, biases=60)
    s.btok[:] = s.btok % 3
    s.run(bank, ("bias",))


def test_masked_nan_and_infinities(bank):
    s = Scene(14, [3, 3], 1500)
    s.allowed[:] = True
    z = s.z
    bad = s.g.random(z.shape) < 0.3
    z[bad] = s.g.choice(np.array([np.nan, np.inf, -np.inf], np.float32), int(bad.sum()))
    s.allowed[bad] = False
    z[2, 100] = -np.inf  # allowed, never likely
    s.allowed[2, 100] = True
    s.logits.copy_(dev(z))
    s.run(bank)


def test_an_allowed_nan_shows_in_the_statistics(bank):
    s = Scene(15, [1], 600)
    s.run(bank, ())
    s.logits[0, 333] = float("nan")
    s.call()
    st = {k: v.cpu().numpy() for k, v in s.st.items()}
    for k in ("top1", "entropy", "logz_t", "entropy_t"):
        assert np.isnan(st[k][0]) and np.isfinite(st[k][1])


def test_temperature_one_and_a_graph(bank):
    s = Scene(16, [5, 0], 3000)
    s.T = 1.0
    s.run(bank)
    first = s.out.clone(), {k: v.clone() for k, v in s.st.items()}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.call()
    s.out.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.out, first[0]) and all(torch.equal(s.st[k], v) for k, v in first[1].items())


def test_an_empty_list_of_biases(bank):
    s = Scene(17, [3, 0], 500, biases=0)
    assert s.btok.size == 0
    s.run(bank)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hist_max", [4096, 4097, 6145, 8193, 21000])
def test_long_histories_and_many_biases(bank, dtype, hist_max):
    """Histories past what is fetched at once, prompts that end anywhere in them, hundreds of biases; ids at
    the ends of their type."""
    s = Scene(hist_max, [3, 0, 4], 1500, dtype, hist_max=hist_max, biases=900)
    s.hist_len[:] = hist_max, hist_max - 1, hist_max
    s.prompt[:] = hist_max // 3, hist_max - 2, 0
    s.hist[:, ::97] = 2 ** 31 - 1
    s.hist[:, ::89] = -2 ** 31
    s.btok[::50] = 2 ** 31 - 1
    s.btok[::61] = -2 ** 31
    s.run(bank)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_more_work_than_the_gpu_holds(bank, dtype):
    """Several CTAs per SM one after the other; the statistics as of the same rows alone."""
    g = synth.rng(40)
    s = Scene(41, [int(g.integers(-1, 4)) for _ in range(70)], 50001, dtype, hist_max=200)
    s.run(bank)
    whole = {k: v.clone() for k, v in s.st.items()}
    one = Scene(41, s.tree, 50001, dtype, hist_max=200)
    lo, hi = int(one.start[5]), int(one.start[8])
    keep = [None] * 3
    for i, b in enumerate((5, 6, 7)):
        keep[i] = slice(one.bstart[b], one.bstart[b + 1])
    one.tree, one.n, one.R = one.tree[5:8], one.n[5:8], hi - lo
    one.start = one.start[5:9] - lo
    one.logits, one.z, one.allowed, one.draft = one.logits[lo:hi], one.z[lo:hi], one.allowed[lo:hi], one.draft[lo:hi]
    for k in ("hist", "hist_len", "prompt", "rep", "pres", "freq"):
        setattr(one, k, getattr(one, k)[5:8])
    one.btok, one.bval = (np.concatenate([x[k] for k in keep]) for x in (one.btok, one.bval))
    one.bstart = one.bstart[5:9] - one.bstart[5]
    one.logits = one.logits.clone(memory_format=torch.contiguous_format)
    one.run(bank)
    # other slices, other sums: the outputs are the same, the statistics within their own bounds
    assert torch.equal(one.out, s.out[lo:hi]) and torch.equal(one.st["argmax"], whole["argmax"][lo:hi])


@pytest.mark.parametrize("T", [0.01, 0.3, 50.0])
def test_temperatures(bank, T):
    s = Scene(18, [4, 2], 2500)
    s.T = T
    s.run(bank)


def test_a_long_root_path(bank, monkeypatch):
    """64 nodes in a chain: more draft tokens in one chunk than a warp has lanes, some of them twice."""
    trees = ref.trees() + [synth.chain(64)]
    monkeypatch.setattr(ref, "trees", lambda: trees)
    bid, _ = bank.add(trees[-1])
    assert bid == len(trees) - 1
    for dtype in (torch.float32, torch.bfloat16):
        for V, rules in ((500, ("draft", "penalty")), (500, ("history", "penalty", "bias", "mask", "draft")),
                         (60, ("history", "penalty", "draft")), (1300, ("bias", "draft", "penalty"))):
            s = Scene(V, [bid, 5], V, dtype, hist_max=40)
            s.draft = s.g.integers(-1, V + 1, s.R).astype(np.int32)
            s.run(bank, rules)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,pad,out_pad", [(5001, 0, 0), (5002, 0, 0), (5000, 1, 0), (5003, 4, 1), (4096, 2, 2), (513, 0, 3),
                                           (511, 1, 1), (3585, 0, 0), (7170, 1, 0)])
def test_rows_of_any_alignment(bank, dtype, V, pad, out_pad):
    s = Scene(V + pad, [5, 3], V, dtype, pad=pad)
    s.run(bank, out_pad=out_pad)
    s.run(bank, ("mask",), out_pad=out_pad)
    s.run(bank, (), out_pad=out_pad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,lo,hi", [(513, 0, 512), (700, 512, 700), (6000, 0, 3600), (6000, 4000, 6000), (5001, 0, 5000),
                                     (128256, 128000, 128256), (131072, 128256, 131072), (50001, 1024, 50000)])
def test_logits_of_the_types_lowest_value(bank, dtype, V, lo, hi):
    """The lowest value of a type in place of -inf, over whole chunks, parts and slices: it weighs nothing, and the
    entropies stay numbers."""
    s = Scene(V + lo, [2, -1, 1], V, dtype, biases=3)
    low = torch.finfo(dtype).min
    s.z[:, lo:hi] = low
    s.z[3] = low  # a row of nothing else: all tokens alike
    s.logits.copy_(dev(s.z))
    s.T = 2.0
    s.run(bank, ())
    s.run(bank, ("mask", "draft"))
    s.z[3] = s.z[0]
    s.logits.copy_(dev(s.z))
    s.T = 1.7  # (below 1, ln Z of a row whose mask leaves only the lowest value is past 32 bits)
    s.run(bank)


@pytest.mark.parametrize("T", [1e-30, 4e-38])
def test_temperatures_next_to_zero(bank, T):
    """1 / T is a number, a difference of two logits over T need not be: the largest logit has all the weight."""
    s = Scene(19, [2, 1], 6000)
    s.z[:] = s.z - 50
    s.z[:, 2500] = 0.5
    s.logits.copy_(dev(s.z))
    s.T = T
    s.run(bank, ())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [5932, 5931, 3584 + 513])
@pytest.mark.parametrize("rules", [(), ("mask",), ("bias",), ("history", "penalty", "bias", "mask", "draft")])
def test_without_statistics(bank, dtype, V, rules):
    """Logits alone, in slices of several whole chunks and the rest of one: the same bits as with statistics."""
    s = Scene(V, [3] * 300, V, dtype, hist_max=30)
    s.run(bank, rules)
    kw = dict(history=dev(s.hist), history_len=dev(s.hist_len), prompt_len=dev(s.prompt)) if "history" in rules else {}
    if "penalty" in rules:
        kw.update(repetition=dev(s.rep), presence=dev(s.pres), frequency=dev(s.freq), draft=dev(s.draft))
    if "bias" in rules:
        kw.update(bias_start=dev(s.bstart), bias_token=dev(s.btok), bias_value=dev(s.bval))
    if "mask" in rules:
        kw.update(mask=dev(pack_bits(s.allowed)))
    req = tv.Requests(row_start=dev(s.start), tree=dev(np.array(s.tree, np.int32)))
    ws = tv.make_workspace(tv.tb_logits_workspace_size(len(s.tree), s.R, V))
    for _ in range(3):
        out = torch.full((s.R, V), 3.0, device="cuda")
        tv.logits_process(bank, req, s.logits, out, ws, **kw)
        assert torch.equal(out, s.out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [700, 5001])
def test_mask_rows_that_there_are_not(bank, dtype, V):
    """A row that names a mask past the last is allowed nothing and reported; -1 stands for no mask as before."""
    s = Scene(V, [5, -1, 2], V, dtype)
    known = s.g.integers(-1, s.R, s.R).astype(np.int32)
    assert tv.tb_workspace_status(s.run(bank, mask_row=known)) == tv.TB_OK
    first, st = s.out.clone(), {k: v.clone() for k, v in s.st.items()}
    rows = known.copy()
    rows[4], rows[7], rows[-1] = s.R, 2 ** 31 - 1, s.R + 3
    req = tv.Requests(row_start=dev(s.start), tree=dev(np.array(s.tree, np.int32)))
    ws = tv.make_workspace(tv.tb_logits_workspace_size(3, s.R, V))
    tv.logits_process(bank, req, s.logits, s.out, ws, temperature=s.T, draft=dev(s.draft), history=dev(s.hist),
                      history_len=dev(s.hist_len), prompt_len=dev(s.prompt), repetition=dev(s.rep), presence=dev(s.pres),
                      frequency=dev(s.freq), bias_start=dev(s.bstart), bias_token=dev(s.btok), bias_value=dev(s.bval),
                      mask=dev(pack_bits(s.allowed)), mask_row=dev(rows), **s.st)
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(ws) == tv.TB_EINVAL
    bad = [4, 7, s.R - 1]
    assert bool((s.out[bad] == -np.inf).all()) and s.st["argmax"][bad].tolist() == [-1] * 3
    assert s.st["entropy"][bad].tolist() == [0.0] * 3 and s.st["logz_t"][bad].tolist() == [-np.inf] * 3
    good = [i for i in range(s.R) if i not in bad]
    assert torch.equal(s.out[good], first[good]) and all(torch.equal(s.st[k][good], st[k][good]) for k in ("argmax", "entropy"))


def test_bias_offsets_past_the_list(bank):
    """Offsets that name entries past the last: those are left out and the call says so; the others count."""
    s = Scene(71, [5, 2, 3], 1500, biases=30)
    assert tv.tb_workspace_status(s.run(bank)) == tv.TB_OK
    n = s.btok.size
    assert s.bstart[1] < n
    want = s.out.clone()
    req = tv.Requests(row_start=dev(s.start), tree=dev(np.array(s.tree, np.int32)))
    for end in (n + 1, n + 5000, 2 ** 31 - 1):
        start = s.bstart.copy()
        start[-1] = end  # of the last request
        ws = tv.make_workspace(tv.tb_logits_workspace_size(3, s.R, s.V))
        tv.logits_process(bank, req, s.logits, s.out, ws, temperature=s.T, draft=dev(s.draft), history=dev(s.hist),
                          history_len=dev(s.hist_len), prompt_len=dev(s.prompt), repetition=dev(s.rep), presence=dev(s.pres),
                          frequency=dev(s.freq), bias_start=dev(start), bias_token=dev(s.btok), bias_value=dev(s.bval),
                          mask=dev(pack_bits(s.allowed)), **s.st)
        torch.cuda.synchronize()
        assert tv.tb_workspace_status(ws) == tv.TB_EINVAL and torch.equal(s.out, want)

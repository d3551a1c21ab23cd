"""paged_accept_q4: the same acceptance as paged_accept's, codes and scales of the
accepted rows moved byte for byte, everything else left alone."""
import numpy as np
import pytest
import torch

import paper_2606_27550_gb300 as tv
import q4_reference as q4
from paper_2606_27550_gb300 import synth
from test_gpu_paged_accept import Scene as Scene16
from test_gpu_paged_accept import bank, i32  # noqa: F401

pytestmark = pytest.mark.gpu


class Scene(Scene16):
    """A batch over 4-bit pages of any bytes."""

    def __init__(self, seed, lens, tree, layers, H, d, P, layout, **kw):
        super().__init__(seed, lens, tree, 1, 1, 64, P, "heads", **kw)
        n_pages, n = self.pools[0].shape[1], tv.q4_page_bytes(P, d)
        self.d = d
        if layout == "heads":
            self.pools = [torch.randint(0, 256, (layers, n_pages, H, n), dtype=torch.uint8, device="cuda") for _ in range(2)]
        else:  # K and V side by side, layers innermost
            both = torch.randint(0, 256, (n_pages, H, layers, 2, n), dtype=torch.uint8, device="cuda")
            self.pools = [both[:, :, :, i].permute(2, 0, 1, 3) for i in range(2)]
        self.pages = tv.PagesQ4(*self.pools, P, d, torch.bfloat16)

    def moved(self, paths):
        want = [p.cpu().numpy().copy() for p in self.pools]
        for b, path in paths.items():
            L, t = self.lens[b], self.table[b]
            for new, pool in zip(want, self.pools):
                old = pool.cpu().numpy()
                for to, src in zip(q4.parts(new, self.P, self.d), q4.parts(old, self.P, self.d)):
                    for j, u in enumerate(path):
                        to[:, t[(L + j) // self.P], :, (L + j) % self.P] = src[:, t[(L + u) // self.P], :, (L + u) % self.P]
        return want


@pytest.mark.parametrize("seed,B,layers,H,d,P,layout,in_place", [
    (1, 1, 1, 1, 64, 8, "heads", True), (2, 9, 3, 4, 128, 16, "side", True), (3, 40, 2, 8, 64, 32, "heads", False),
    (4, 5, 33, 3, 128, 16, "heads", True), (5, 60, 1, 2, 64, 128, "side", True), (6, 4, 2, 40, 128, 1024, "side", False)])
@pytest.mark.parametrize("match", [0.0, 0.7, 1.0])
def test_accept(bank, seed, B, layers, H, d, P, layout, in_place, match):  # noqa: F811
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
    tv.paged_accept_q4(bank, s.req, s.pages, s.results, draft=i32(s.draft), argmax=i32(s.argmax), vocab=s.vocab,
                       lens_out=out)
    torch.cuda.synchronize()
    assert s.results.tolist() == results
    assert (s.req.lens if in_place else out).tolist() == [r[2] for r in results]
    for pool, w in zip(s.pools, want):
        assert np.array_equal(pool.cpu().numpy(), w)


def test_results_of_another_rule_and_no_pages(bank):  # noqa: F811
    s = Scene(31, [100, 20, 0, 64], [5, 8, -1, 10], 2, 2, 64, 16, "heads")
    paths = {0: [0, 1, 5], 1: [0], 3: [0, 2, 7, 9]}
    for b, p in paths.items():
        s.results[b, 0] = len(p)
        s.results[b, 4:4 + len(p)] = i32(np.array(p))
    want = s.moved(paths)
    tv.paged_accept_q4(bank, s.req, s.pages, s.results)
    torch.cuda.synchronize()
    for pool, w in zip(s.pools, want):
        assert np.array_equal(pool.cpu().numpy(), w)
    assert s.req.lens.tolist() == [103, 21, 0, 68]
    tv.paged_accept_q4(bank, s.req, None, s.results)
    torch.cuda.synchronize()
    for pool, w in zip(s.pools, want):
        assert np.array_equal(pool.cpu().numpy(), w)


@pytest.mark.parametrize("entry", [-1, 10**6])
def test_rows_that_cannot_move_are_reported(bank, entry):  # noqa: F811
    s = Scene(41, [14], [10], 2, 2, 128, 16, "heads", match=1.0)
    k, path, _ = s.expected(0)
    assert any((14 + u) // 16 >= 2 for u in path) and k > 2
    table = s.table.copy()
    table[0, 2] = entry  # slots 32 to 47
    s.req = tv.Requests(row_start=s.req.row_start, lens=s.req.lens, table=i32(table), page_size=16, tree=s.req.tree)
    want = [p.cpu().numpy().copy() for p in s.pools]
    for w, pool in zip(want, s.pools):
        old = pool.cpu().numpy()
        for to, src in zip(q4.parts(w, 16, 128), q4.parts(old, 16, 128)):
            for j, u in enumerate(path):
                if (14 + u) // 16 != 2 and (14 + j) // 16 != 2:
                    to[:, s.table[0, (14 + j) // 16], :, (14 + j) % 16] = src[:, s.table[0, (14 + u) // 16], :, (14 + u) % 16]
    tv.paged_accept_q4(bank, s.req, s.pages, s.results, draft=i32(s.draft), argmax=i32(s.argmax), vocab=s.vocab)
    torch.cuda.synchronize()
    assert s.results[0, 3].item() == tv.TB_EINVAL and s.results[0, 0].item() == k
    for pool, w in zip(s.pools, want):
        assert np.array_equal(pool.cpu().numpy(), w)

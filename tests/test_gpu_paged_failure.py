"""A bounded wait of the paged attention that runs out: with the test hook the
second product waits on a barrier that nothing arrives on, and every other role
of the kernel runs into that one.  The call ends by itself, reports the time-out
and writes nothing; after tb_workspace_init the same context computes as before."""
import time

import pytest
import torch

import paged_reference as ref
import paper_2606_27550_gb300 as tv
from test_gpu_paged_attention import BF, HF, Scene

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bank():
    b = tv.Bank(16, 0)
    for t in ref.trees():
        b.add(t)
    yield b
    b.close()


@pytest.mark.parametrize("form", ["plain", "cap", "bias"])
@pytest.mark.parametrize("d,dtype", [(64, HF), (128, BF)])
def test_a_wait_that_runs_out(bank, form, d, dtype):
    # units of several CTAs (one long request), of one, several in one CTA, and rows that are cut off by documents
    lens = [9000, 100, 0, 400] + [30] * 300
    tree = [7, 5, 8, -1] + [0, 2, 3] * 100
    s = Scene(d, lens, tree, 4, 2, d, 16, dtype=dtype)
    kw = dict(softcap=30.0 if form == "cap" else 0.0, slopes=torch.full((4,), 0.02, device="cuda") if form == "bias" else None)
    s.run(bank, cap=kw["softcap"], slopes=kw["slopes"])
    out, lse = torch.full_like(s.out, 5.0), torch.full_like(s.lse, 5.0)
    t0 = time.time()
    tv.paged_tree_attention(bank, s.req, s.pages, s.plan, s.q, out, s.ws, layer=tv.TB_DEBUG_EXPIRE_WAIT, lse=lse, **kw)
    torch.cuda.synchronize()
    assert time.time() - t0 < 20.0
    assert tv.tb_workspace_status(s.ws) == tv.TB_ETIMEOUT
    assert bool((out == 5).all()) and bool((lse == 5).all())
    tv.tb_workspace_init(s.ws)
    tv.paged_tree_attention(bank, s.req, s.pages, s.plan, s.q, out, s.ws, lse=lse, **kw)
    torch.cuda.synchronize()
    assert tv.tb_workspace_status(s.ws) == tv.TB_OK
    assert torch.equal(out, s.out) and torch.equal(lse, s.lse)

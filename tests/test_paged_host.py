"""The paged serving calls without a GPU: every refusal of their argument checks,
what they launch, and the binding's own checks (the library's objects linked
with a stand-in for the CUDA runtime)."""
import ctypes

import pytest
import torch

import fake_cuda
import paper_2606_27550_gb300 as tv

STREAM = 7
BF = torch.bfloat16


@pytest.fixture(scope="module")
def fake_path(tmp_path_factory):
    return fake_cuda.build_lib(tmp_path_factory.mktemp("fake_paged"))


@pytest.fixture
def lib(fake_path, monkeypatch):
    monkeypatch.setattr(tv, "_lib", None)
    lib = tv.load(fake_path)
    fake_cuda.launches(lib)
    yield lib


class Setup:
    def __init__(self, B=3, P=16, heads=4, H=2, d=64, R=9, dtype=BF):
        self.bank = tv.Bank(2, 0)
        self.bank.add([-1, 0, 0])
        z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t)  # noqa: E731
        self.req = tv.Requests(row_start=z(B + 1), tree=z(B), lens=z(B), table=z(B, 5), page_size=P)
        self.pages = tv.Pages(z(2, 6, H, P, d, t=dtype), z(2, 6, H, P, d, t=dtype))
        self.slots, self.positions, self.status = z(R, t=torch.int64), z(R), z(B)
        self.plan = tv.make_paged_plan(B, "cpu")
        self.pool = tv.make_page_pool(6, B, "cpu")
        self.q, self.out = z(R, heads, d, t=dtype), z(R, heads, d, t=dtype)
        self.kv = z(R, H, d, t=dtype)
        self.ws = tv.make_workspace(tv.tb_workspace_size(0, 1, H, heads, d, 0, 0), "cpu")
        self.logits = torch.zeros(R, 100)
        self.lws = tv.make_workspace(tv.tb_logits_workspace_size(B, R, 100), "cpu")
        self.results = tv.make_results(B, "cpu")

    def do_plan(self, **kw):
        a = dict(pool=self.pool, n_q_heads=4, n_kv_heads=2, stream=STREAM)
        a.update(kw)
        tv.paged_plan(a.pop("bank", self.bank), a.pop("req", self.req), self.slots, self.positions, a.pop("status", self.status),
                      a.pop("plan", self.plan), **a)

    def store(self, **kw):
        a = dict(q=self.q, positions=self.positions, rope_theta=1e4, stream=STREAM)
        a.update(kw)
        tv.paged_kv_store(a.pop("pages", self.pages), a.pop("slots", self.slots), a.pop("k", self.kv), self.kv, **a)

    def attend(self, **kw):
        a = dict(stream=STREAM)
        a.update(kw)
        tv.paged_tree_attention(self.bank, a.pop("req", self.req), a.pop("pages", self.pages), a.pop("plan", self.plan),
                                a.pop("q", self.q), a.pop("out", self.out), a.pop("ws", self.ws), **a)

    def process(self, **kw):
        a = dict(stream=STREAM)
        a.update(kw)
        tv.logits_process(a.pop("bank", self.bank), a.pop("req", self.req), a.pop("logits", self.logits),
                          a.pop("out", torch.zeros(9, 100)), a.pop("ws", self.lws), **a)

    def accept(self, **kw):
        a = dict(draft=self.positions, argmax=self.positions, vocab=10, stream=STREAM)
        a.update(kw)
        tv.paged_accept(self.bank, a.pop("req", self.req), a.pop("pages", self.pages), self.results, **a)


@pytest.fixture
def s(lib):
    x = Setup()
    yield x
    x.bank.close()


def refused(code, fn, **kw):
    with pytest.raises(tv.TreeVerifyError) as e:
        fn(**kw)
    assert e.value.status == code, e.value
    return str(e.value)


def test_one_launch_each(lib, s):
    for fn, kernel in ((s.do_plan, "k_paged_plan"), (s.store, "k_paged_store"), (s.process, "k_logits"),
                       (s.accept, "k_paged_accept")):
        fn()
        (launch,) = fake_cuda.launches(lib)
        assert kernel in launch.name and launch.stream == STREAM
    s.attend()
    assert all(x.stream == STREAM and "paged" in x.name for x in fake_cuda.launches(lib))


def _other(req, **kw):
    a = {f: getattr(req, f) for f in ("row_start", "tree", "lens", "table", "page_size", "n_new", "key_begin")}
    a.update(kw)
    return tv.Requests(**a)


def test_refusals_of_plan(lib, s):
    for page in (0, 4, 12, 2048):
        refused(tv.TB_EINVAL, s.do_plan, req=_other(s.req, page_size=page))
    refused(tv.TB_EINVAL, s.do_plan, bank=None)
    refused(tv.TB_EINVAL, s.do_plan, req=_other(s.req, tree=None))
    refused(tv.TB_EINVAL, s.do_plan, req=_other(s.req, lens=None))
    refused(tv.TB_EINVAL, s.do_plan, req=_other(s.req, table=None))
    refused(tv.TB_EINVAL, s.do_plan, n_q_heads=5)
    refused(tv.TB_EINVAL, s.do_plan, window=-1)
    refused(tv.TB_EINVAL, s.do_plan, sink=-3)
    refused(tv.TB_ECAPACITY, s.do_plan, plan=s.plan[:-1])
    refused(tv.TB_EINVAL, s.do_plan, req=_other(s.req, tree=None, n_new=s.req.tree), bank=None)  # heads without trees
    big = torch.zeros(tv.TB_MAX_REQUESTS + 2, dtype=torch.int32)
    refused(tv.TB_EINVAL, s.do_plan, req=tv.Requests(row_start=big, tree=big[:-1], lens=big[:-1],
                                                     table=big[:-1].view(-1, 1)), pool=None, status=big[:-1])
    assert tv.tb_paged_plan_size(0) == 0 and tv.tb_paged_plan_size(tv.TB_MAX_REQUESTS + 1) == 0
    assert fake_cuda.launches(lib) == []
    s.do_plan(req=_other(s.req, tree=None, n_new=s.req.tree), bank=None, n_q_heads=0)
    assert len(fake_cuda.launches(lib)) == 1


def test_refusals_of_store(lib, s):
    refused(tv.TB_EINVAL, s.store, layer=2)
    refused(tv.TB_EINVAL, s.store, layer=-1)
    refused(tv.TB_EINVAL, s.store, sections=(16, 8), positions=torch.zeros(2, 9, dtype=torch.int32))
    refused(tv.TB_EINVAL, s.store, sections=(40, -8), positions=torch.zeros(2, 9, dtype=torch.int32))
    refused(tv.TB_EINVAL, s.store, rope_theta=0.5)
    refused(tv.TB_EINVAL, s.store, rope_theta=float("inf"))
    refused(tv.TB_EINVAL, s.store, k=torch.zeros(9, 2, 65, dtype=BF)[..., 1:])  # misaligned rows
    with pytest.raises(ValueError):
        s.store(k=torch.zeros(8, 2, 64, dtype=BF))
    with pytest.raises(TypeError):
        s.store(k=torch.zeros(9, 2, 64))
    with pytest.raises(ValueError):
        s.store(positions=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(TypeError):
        s.store(slots=torch.zeros(9, dtype=torch.int32))
    odd = torch.zeros(1, 6, 2, 16, 68, dtype=BF)[..., :64]
    refused(tv.TB_EINVAL, s.store, pages=tv.Pages(odd, odd))  # strides not multiples of 8
    for d, status in ((96, tv.TB_EUNSUPPORTED), (256, tv.TB_EUNSUPPORTED)):
        p = torch.zeros(1, 2, 2, 16, d, dtype=BF)
        x = torch.zeros(9, 2, d, dtype=BF)
        with pytest.raises(tv.TreeVerifyError) as e:
            tv.paged_kv_store(tv.Pages(p, p), s.slots, x, x, stream=STREAM)
        assert e.value.status == status
    with pytest.raises(TypeError):
        tv.Pages(torch.zeros(1, 2, 2, 16, 64), torch.zeros(1, 2, 2, 16, 64)).as_c()
    assert fake_cuda.launches(lib) == []


def test_refusals_of_attention(lib, s):
    refused(tv.TB_EINVAL, s.attend, layer=2)
    refused(tv.TB_EINVAL, s.attend, scale=0.0)
    refused(tv.TB_EINVAL, s.attend, scale=float("nan"))
    refused(tv.TB_EINVAL, s.attend, softcap=-1.0)
    refused(tv.TB_EUNSUPPORTED, s.attend, softcap=1025.0)
    refused(tv.TB_EUNSUPPORTED, s.attend, softcap=1e-40)
    refused(tv.TB_EINVAL, s.attend, q=torch.zeros(9, 3, 64, dtype=BF), out=torch.zeros(9, 3, 64, dtype=BF))
    refused(tv.TB_EINVAL, s.attend, req=_other(s.req, page_size=32))
    refused(tv.TB_EINVAL, s.attend, req=_other(s.req, tree=None))
    refused(tv.TB_ECAPACITY, s.attend, ws=s.ws[:-16])
    refused(tv.TB_ECAPACITY, s.attend, plan=s.plan[:-1])
    with pytest.raises(ValueError):
        s.attend(out=torch.zeros(9, 4, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        s.attend(q=torch.zeros(9, 8, 64, dtype=BF)[:, ::2])
    with pytest.raises(ValueError):
        s.attend(lse=torch.zeros(9, 3))
    with pytest.raises(TypeError):
        s.attend(slopes=torch.zeros(4, dtype=torch.float64))
    assert fake_cuda.launches(lib) == []


def test_refusals_of_logits(lib, s):
    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(tv.TB_EINVAL, s.process, temperature=T)
    refused(tv.TB_EINVAL, s.process, temperature=1e-39)  # 1 / T is no number
    refused(tv.TB_ECAPACITY, s.process, ws=s.lws[:-16])
    refused(tv.TB_EINVAL, s.process, history=torch.zeros(3, 4, dtype=torch.int32))
    refused(tv.TB_EINVAL, s.process, bias_start=torch.zeros(4, dtype=torch.int32))
    refused(tv.TB_EINVAL, s.process, mask=torch.zeros(9, 3, dtype=torch.int32))
    refused(tv.TB_EINVAL, s.process, draft_logit=torch.zeros(9))
    half = torch.zeros(9, 100, dtype=torch.float16)
    with pytest.raises(TypeError):
        s.process(out=half)
    with pytest.raises(TypeError):
        s.process(logits=half.double())
    with pytest.raises(ValueError):
        s.process(logits=torch.zeros(100, 9).T)
    with pytest.raises(ValueError):
        s.process(mask=torch.zeros(8, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        s.process(argmax=torch.zeros(8, dtype=torch.int32))
    with pytest.raises(TypeError):
        s.process(repetition=torch.zeros(3, dtype=torch.float64))
    assert fake_cuda.launches(lib) == []
    # in place with another type: through the C call, the binding never gets there
    a = s.logits
    rc = lib.logits_process(s.bank.handle, ctypes.byref(s.req.as_c()), a.data_ptr(), tv.TB_BF16, 100, 9, 100, None, 1.0,
                            a.data_ptr(), 100, None, s.lws.data_ptr(), s.lws.numel(), STREAM)
    assert rc == tv.TB_EINVAL
    assert tv.tb_logits_workspace_size(0, 1, 1) == 0


def test_refusals_of_accept(lib, s):
    refused(tv.TB_EINVAL, s.accept, vocab=0)
    refused(tv.TB_EINVAL, s.accept, req=_other(s.req, tree=None))
    refused(tv.TB_EINVAL, s.accept, req=_other(s.req, page_size=32))
    with pytest.raises(ValueError):
        s.accept(lens_out=torch.zeros(2, dtype=torch.int32))
    assert fake_cuda.launches(lib) == []
    s.accept(pages=None)
    s.accept(draft=None, argmax=None, vocab=0)
    assert len(fake_cuda.launches(lib)) == 2


def test_another_devices_bank_is_refused(lib, s):
    lib.fake_set_device(1)
    try:
        for fn in (s.do_plan, s.attend, s.accept, s.process):
            refused(tv.TB_EINVAL, fn)
    finally:
        lib.fake_set_device(0)
    assert fake_cuda.launches(lib) == []


def test_a_pool_of_what_is_held_alone(lib, s):
    """The form of a step's further plans launches; any other pool without a ring, or without `held`, is refused."""
    s.do_plan(pool=s.pool.held_only())
    assert len(fake_cuda.launches(lib)) == 1
    z = torch.zeros(3, dtype=torch.int32)
    for bad in (tv.PagePool(None, z, z), tv.PagePool(None, None, z, state_out=z), tv.PagePool(None, None, z, held_out=z),
                tv.PagePool(None, None, None), tv.PagePool(z, None, z), tv.PagePool(z, z, None)):
        refused(tv.TB_EINVAL, s.do_plan, pool=bad)
    assert fake_cuda.launches(lib) == []


def test_mask_rows_need_their_number(lib, s):
    """mask_row indexes the mask's rows on the device: the C call wants to know how many there are."""
    words, rows = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)
    rules = tv.TbLogitRules()
    rules.mask, rules.mask_stride, rules.mask_row = words.data_ptr(), 4, rows.data_ptr()
    out = torch.zeros(9, 100)

    def call():
        return lib.logits_process(s.bank.handle, ctypes.byref(s.req.as_c()), s.logits.data_ptr(), tv.TB_F32, 100, 9, 100,
                                  ctypes.byref(rules), 1.0, out.data_ptr(), 100, None, s.lws.data_ptr(), s.lws.numel(), STREAM)

    assert call() == tv.TB_EINVAL and fake_cuda.launches(lib) == []
    rules.mask_rows = 2
    assert call() == tv.TB_OK and len(fake_cuda.launches(lib)) == 1
    s.process(mask=words, mask_row=rows)
    assert len(fake_cuda.launches(lib)) == 1


def test_steps_without_rows(lib, s):
    """Empty tensors have no address: no call refuses them, and those that have only rows to work on launch nothing."""
    none = torch.zeros(0, 2, 64, dtype=BF)
    s.slots, s.positions = s.slots[:0], s.positions[:0]
    s.do_plan()
    assert len(fake_cuda.launches(lib)) == 1
    s.kv = none
    s.store(k=none, q=torch.zeros(0, 4, 64, dtype=BF), q_out=torch.zeros(0, 4, 64, dtype=BF))
    s.store(k=none, q=None, positions=torch.zeros(3, 0, dtype=torch.int32), sections=(8, 12, 12))
    s.store(k=none, q=None, rope_theta=0.0)
    s.attend(q=s.q[:0], out=s.out[:0], lse=torch.zeros(0, 4))
    s.process(logits=s.logits[:0], out=torch.zeros(0, 100), draft=s.positions, argmax=s.positions, top1=torch.zeros(0),
              draft_logit=torch.zeros(0), mask=torch.zeros(0, 4, dtype=torch.int32))
    assert fake_cuda.launches(lib) == []
    s.accept(draft=s.positions, argmax=s.positions)
    assert len(fake_cuda.launches(lib)) == 1
    refused(tv.TB_EINVAL, s.accept, draft=s.positions, argmax=s.positions, vocab=0)  # greedy, not results given


def test_the_attention_and_its_join(lib, s):
    """Exactly two launches, on the call's stream, the join behind the attention as its dependent."""
    s.attend()
    first, second = fake_cuda.launches(lib)
    assert "k_paged_attention" in first.name and "k_paged_merge" in second.name
    for launch in (first, second):
        assert launch.stream == STREAM and launch.pdl and launch.cluster == 1 and launch.device == 0
    assert first.grid == (152, 1, 1) and first.block == 512 and second.block == 256


def test_bias_offsets_need_the_lists_length(lib, s):
    """bias_start indexes the bias lists on the device: the C call wants to know how long they are."""
    start, token, value = torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int32), torch.zeros(5)
    rules = tv.TbLogitRules()
    rules.bias_start, rules.bias_token, rules.bias_value = start.data_ptr(), token.data_ptr(), value.data_ptr()
    out = torch.zeros(9, 100)

    def call():
        return lib.logits_process(s.bank.handle, ctypes.byref(s.req.as_c()), s.logits.data_ptr(), tv.TB_F32, 100, 9, 100,
                                  ctypes.byref(rules), 1.0, out.data_ptr(), 100, None, s.lws.data_ptr(), s.lws.numel(), STREAM)

    for n in (0, -1, 2 ** 31):
        rules.n_bias = n
        assert call() == tv.TB_EINVAL and fake_cuda.launches(lib) == []
    rules.n_bias = 5
    assert call() == tv.TB_OK and len(fake_cuda.launches(lib)) == 1
    s.process(bias_start=start, bias_token=token, bias_value=value)
    s.process(bias_start=start, bias_token=token[:0], bias_value=value[:0])
    assert len(fake_cuda.launches(lib)) == 2
    with pytest.raises(ValueError):
        s.process(bias_start=start, bias_token=token, bias_value=value[:4])

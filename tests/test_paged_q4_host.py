"""The calls over 4-bit pages and the store with norms without a GPU: every refusal
of their argument checks, what they launch, and the binding's own checks."""
import ctypes

import pytest
import torch

import fake_cuda
import paper_2606_27550_gb300 as tv
from test_paged_host import BF, STREAM, _other, fake_path, lib, refused  # noqa: F401
from test_paged_host import Setup as Setup16


class Setup(Setup16):
    def __init__(self):
        super().__init__()
        self.pages16 = self.pages
        self.pages = tv.make_pages_q4(2, 6, 2, 16, 64, BF, device="cpu")
        self.w = torch.zeros(64, dtype=BF)

    def _store(self, fn, own, **kw):
        a = dict(q=self.q, positions=self.positions, rope_theta=1e4, q_norm=self.w, k_norm=self.w, stream=STREAM)
        a.update(kw)
        fn(a.pop("pages", own), a.pop("slots", self.slots), a.pop("k", self.kv), a.pop("v", self.kv), **a)

    def store_norm(self, **kw):
        self._store(tv.paged_kv_store_norm, self.pages16, **kw)

    def store_q4(self, **kw):
        self._store(tv.paged_kv_store_q4, self.pages, **kw)

    def load(self, **kw):
        a = dict(k=self.kv, v=self.kv.clone(), slots=self.slots, pages=self.pages, stream=STREAM)
        a.update(kw)
        tv.paged_kv_load_q4(a.pop("pages"), a.pop("slots"), a.pop("k"), a.pop("v"), **a)

    def attend(self, **kw):
        a = dict(stream=STREAM)
        a.update(kw)
        tv.paged_tree_attention_q4(self.bank, a.pop("req", self.req), a.pop("pages", self.pages),
                                   a.pop("plan", self.plan), a.pop("q", self.q), a.pop("out", self.out),
                                   a.pop("ws", self.ws), **a)

    def accept(self, **kw):
        a = dict(draft=self.positions, argmax=self.positions, vocab=10, stream=STREAM)
        a.update(kw)
        tv.paged_accept_q4(self.bank, a.pop("req", self.req), a.pop("pages", self.pages), self.results, **a)


@pytest.fixture
def s(lib):  # noqa: F811
    x = Setup()
    yield x
    x.bank.close()


def test_launches(lib, s):  # noqa: F811
    for fn, kernel in ((s.store_norm, "k_paged_rows"), (s.store_q4, "k_paged_rows"), (s.load, "k_paged_load"),
                       (s.accept, "k_paged_accept")):
        fn()
        (launch,) = fake_cuda.launches(lib)
        assert kernel in launch.name and launch.stream == STREAM and launch.pdl
    s.attend()
    first, second = fake_cuda.launches(lib)
    assert "k_paged_attention" in first.name and "k_paged_merge" in second.name
    for launch in (first, second):
        assert launch.stream == STREAM and launch.pdl and launch.cluster == 1 and launch.device == 0
    assert first.grid == (152, 1, 1)
    s.store_q4(q=None, q_norm=None, k_norm=None, rope_theta=0.0, positions=None)
    s.load(k=torch.zeros(2, 9, 2, 64, dtype=BF), v=torch.zeros(2, 9, 2, 64, dtype=BF))
    assert len(fake_cuda.launches(lib)) == 2


@pytest.mark.parametrize("name", ["store_norm", "store_q4"])
def test_refusals_of_the_stores(lib, s, name):  # noqa: F811
    fn = getattr(s, name)
    refused(tv.TB_EINVAL, fn, layer=2)
    refused(tv.TB_EINVAL, fn, layer=-1)
    refused(tv.TB_EINVAL, fn, sections=(16, 8), positions=torch.zeros(2, 9, dtype=torch.int32))
    refused(tv.TB_EINVAL, fn, rope_theta=0.5)
    refused(tv.TB_EINVAL, fn, k=torch.zeros(9, 2, 65, dtype=BF)[..., 1:])
    for eps in (-1e-6, float("nan"), float("inf")):
        refused(tv.TB_EINVAL, fn, eps=eps)
    refused(tv.TB_EINVAL, fn, weight_offset=float("inf"))
    refused(tv.TB_EINVAL, fn, q_norm=torch.zeros(65, dtype=BF)[1:])  # off 16 bytes
    with pytest.raises(ValueError):
        fn(k_norm=s.w[:32])
    with pytest.raises(TypeError):
        fn(k_norm=s.w.float())
    with pytest.raises(TypeError):
        fn(k=torch.zeros(9, 2, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        fn(v=torch.zeros(8, 2, 64, dtype=BF))
    with pytest.raises(ValueError):
        fn(positions=torch.zeros(5, dtype=torch.int32))
    with pytest.raises(TypeError):
        fn(slots=torch.zeros(9, dtype=torch.int32))
    assert fake_cuda.launches(lib) == []


def test_packed_operands_are_the_c_structs():
    assert tv._ROWS(1 << 40, -8, 1 << 33) == bytes(tv.TbRows(1 << 40, -8, 1 << 33))
    assert tv._ROPE(1e4, 3, 16, 24, 24, 0, 77, 9) == bytes(tv.TbRope(1e4, 3, (16, 24, 24, 0), 77, 9))
    assert tv._NORM(0, 1 << 50, 1e-6, 1.0) == bytes(tv.TbHeadNorm(None, 1 << 50, 1e-6, 1.0))


def test_too_many_heads_for_a_store(lib, s):  # noqa: F811
    pages = tv.make_pages_q4(2, 6, 2, 16, 64, BF, device="cpu").as_c()
    pages.n_kv_heads, pages.layer_stride, pages.page_stride = (1 << 20) + 1, 1 << 40, 1 << 36
    rows = tv.TbRows(s.kv.data_ptr(), 0, 0)
    rc = lib.paged_kv_store_q4(ctypes.byref(pages), 0, s.slots.data_ptr(), 9, ctypes.byref(rows), ctypes.byref(rows), None,
                               None, 0, None, None, STREAM)
    assert rc == tv.TB_EUNSUPPORTED and fake_cuda.launches(lib) == []


@pytest.mark.parametrize("rows,Hq,H,block,grid", [
    (1, 16, 8, 256, 1), (9, 32, 8, 192, 9), (760, 32, 8, 192, 760), (1000, 32, 8, 128, 1000), (2400, 32, 8, 128, 1200),
    (8191, 32, 32, 256, 1171), (9, 40, 8, 224, 9), (9, 64, 8, 160, 9), (9, 33, 3, 256, 9), (40000, 32, 32, 256, 5000)])
def test_the_shape_of_a_store(lib, s, rows, Hq, H, block, grid):  # noqa: F811
    """CTAs as wide as the 16-byte places of a row, of one row while the SMs hold as many, of 8 at most: 1024 threads on
    each of 152 SMs are 608 CTAs of 256, 760 of 192 and 1216 of 128, of which 1000 rows take one each."""
    kv, q = (torch.zeros(128, dtype=BF).expand(rows, h, 128) for h in (H, Hq))
    pages = tv.make_pages_q4(1, 2, H, 16, 128, BF, device="cpu")
    tv.paged_kv_store_q4(pages, torch.full((rows,), -1, dtype=torch.int64), kv, kv, q=q, q_out=q, stream=STREAM)
    (launch,) = fake_cuda.launches(lib)
    assert launch.block == block and launch.grid == (grid, 1, 1)


def test_refusals_of_load(lib, s):  # noqa: F811
    refused(tv.TB_EINVAL, s.load, layer=2)
    refused(tv.TB_EINVAL, s.load, layer=-1)
    two = torch.zeros(2, 9, 2, 64, dtype=BF)
    refused(tv.TB_EINVAL, s.load, layer=1, k=two, v=two)  # layers 1 and 2 of 2
    refused(tv.TB_EINVAL, s.load, k=torch.zeros(9, 2, 65, dtype=BF)[..., 1:])
    odd = torch.zeros(9 * 2 * 64 * 2 + 20, dtype=BF).as_strided((2, 9, 2, 64), (9 * 128 + 4, 128, 64, 1))
    refused(tv.TB_EINVAL, s.load, k=odd, v=odd)
    for k, v in ((two, s.kv), (two, two[:1]), (two, torch.zeros(2, 10, 2, 64, dtype=BF)), (two[:0], two[:0])):
        with pytest.raises(ValueError):
            s.load(k=k, v=v)
    with pytest.raises(ValueError):
        s.load(k=s.kv[:8])
    with pytest.raises(TypeError):
        s.load(v=s.kv.half())
    with pytest.raises(TypeError):
        s.load(slots=s.positions)
    # more rows than a launch counts
    rows = tv.TbRows(s.kv.data_ptr(), 0, 0)
    rc = lib.paged_kv_load_q4(ctypes.byref(s.pages.as_c()), 0, 1, s.slots.data_ptr(), (1 << 30) + 1, ctypes.byref(rows),
                              ctypes.byref(rows), 0, STREAM)
    assert rc == tv.TB_EUNSUPPORTED and fake_cuda.launches(lib) == []


def test_refusals_of_attention_and_accept(lib, s):  # noqa: F811
    refused(tv.TB_EINVAL, s.attend, layer=2)
    refused(tv.TB_EINVAL, s.attend, scale=0.0)
    refused(tv.TB_EINVAL, s.attend, softcap=-1.0)
    refused(tv.TB_EUNSUPPORTED, s.attend, softcap=1025.0)
    refused(tv.TB_EINVAL, s.attend, q=torch.zeros(9, 3, 64, dtype=BF), out=torch.zeros(9, 3, 64, dtype=BF))
    refused(tv.TB_EUNSUPPORTED, s.attend, q=torch.zeros(9, 130, 64, dtype=BF), out=torch.zeros(9, 130, 64, dtype=BF))
    refused(tv.TB_EINVAL, s.attend, req=_other(s.req, page_size=32))
    refused(tv.TB_EINVAL, s.attend, req=_other(s.req, tree=None))
    refused(tv.TB_ECAPACITY, s.attend, ws=s.ws[:-16])
    refused(tv.TB_ECAPACITY, s.attend, plan=s.plan[:-1])
    with pytest.raises(ValueError):
        s.attend(out=torch.zeros(9, 4, 64, dtype=torch.float16))
    refused(tv.TB_EINVAL, s.accept, vocab=0)
    refused(tv.TB_EINVAL, s.accept, req=_other(s.req, tree=None))
    refused(tv.TB_EINVAL, s.accept, req=_other(s.req, page_size=32))
    assert fake_cuda.launches(lib) == []
    s.accept(pages=None)
    s.accept(draft=None, argmax=None, vocab=0)
    assert len(fake_cuda.launches(lib)) == 2


def test_another_devices_bank_is_refused(lib, s):  # noqa: F811
    lib.fake_set_device(1)
    try:
        for fn in (s.attend, s.accept):
            refused(tv.TB_EINVAL, fn)
    finally:
        lib.fake_set_device(0)
    assert fake_cuda.launches(lib) == []


def test_bad_pages(lib, s):  # noqa: F811
    """Shapes, strides, types and kinds that a call must not read as 4-bit pages."""
    n = tv.q4_page_bytes(16, 64)
    assert n == 16 * 34
    k = torch.zeros(2, 6, 2, n, dtype=torch.uint8)

    def pages(k=k, v=None, page=16, d=64, dtype=BF):
        return tv.PagesQ4(k, k if v is None else v, page, d, dtype)

    for bad in (dict(k=k[..., :-1]), dict(k=k[0]), dict(v=k[:1]), dict(v=k.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(page=32), dict(d=128), dict(k=torch.zeros(2, 6, n, 2, dtype=torch.uint8).transpose(2, 3))):
        with pytest.raises(ValueError):
            pages(**bad)
    for bad in (dict(k=k.view(torch.int8)), dict(dtype=torch.float32), dict(dtype=torch.uint8)):
        with pytest.raises(TypeError):
            pages(**bad)
    calls = (s.store_q4, s.load, s.attend, s.accept)
    for fn in calls:  # 16-bit pages where 4-bit ones belong, and the other way round
        with pytest.raises(TypeError):
            fn(pages=s.pages16)
    with pytest.raises(TypeError):
        s.store_norm(pages=s.pages)
    with pytest.raises(TypeError):
        Setup16.store(s, pages=s.pages)
    with pytest.raises(TypeError):
        Setup16.attend(s, pages=s.pages)
    with pytest.raises(TypeError):
        Setup16.accept(s, pages=s.pages)
    off = torch.zeros(2 * 6 * 2 * n + 16, dtype=torch.uint8)[8:8 + 2 * 6 * 2 * n].view(2, 6, 2, n)
    odd = torch.zeros(2, 6, 2, n + 8, dtype=torch.uint8)[..., :n]
    tight = torch.zeros(2 * 6 * 2 * n, dtype=torch.uint8).as_strided((2, 6, 2, n), (12 * n, 2 * n, n - 16, 1))
    for x in (off, odd, tight):
        for fn in calls:
            refused(tv.TB_EINVAL, fn, pages=pages(k=x))
    c = s.pages.as_c()
    for field, value, status in (("head_dim", 96, tv.TB_EUNSUPPORTED), ("dtype", tv.TB_F32, tv.TB_EUNSUPPORTED),
                                 ("page_size", 12, tv.TB_EINVAL), ("n_pages", 0, tv.TB_EINVAL), ("k", None, tv.TB_EINVAL)):
        kept = getattr(c, field)
        setattr(c, field, value)
        refused(status, s.accept)
        setattr(c, field, kept)
    assert fake_cuda.launches(lib) == []


def test_steps_without_rows(lib, s):  # noqa: F811
    none = torch.zeros(0, 2, 64, dtype=BF)
    s.slots, s.positions = s.slots[:0], s.positions[:0]
    q0 = torch.zeros(0, 4, 64, dtype=BF)
    for fn in (s.store_norm, s.store_q4):
        fn(k=none, v=none, q=q0, q_out=q0)
        fn(k=none, v=none, q=None, rope_theta=0.0)
    s.load(k=none, v=none)
    s.attend(q=s.q[:0], out=s.out[:0], lse=torch.zeros(0, 4))
    assert fake_cuda.launches(lib) == []
    s.accept(draft=s.positions, argmax=s.positions)
    assert len(fake_cuda.launches(lib)) == 1

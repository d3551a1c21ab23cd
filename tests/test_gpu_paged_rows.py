"""paged_kv_store_norm, paged_kv_store_q4 and paged_kv_load_q4: norms, rotation and
rounding to 4 bits bit by bit, axes, strides, types, padding, numbers at the ends
of the range, what stays untouched.

The documented 32-bit steps take sines, cosines and reciprocal roots that are right
to half a unit in the last place but for one in a thousand; such a unit moves a
result by 2^-23 of the head's size, which changes a number rounded to 16 bits (spaced
2^-7 to 2^-11) or a code (spaced a seventh of the largest) in fewer than 1 of 10^7
elements.  The cases have 10^6: all bits are the same as the reference's."""
import numpy as np
import pytest
import torch

import paper_2606_27550_gb300 as tv
import q4_reference as q4

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
THETA = 10000.0


def f32(t):
    return t.float().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.int16).cpu()


def rows_like(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)


class Scene:
    """Rows of a projection's output (q, k, v and something else side by side), slots with two of padding."""

    def __init__(self, rows, Hq, H, d, P, dtype, sections, norm, seed=0):
        torch.manual_seed(rows + seed)
        self.n_pages = rows // P + 4
        self.Hq, self.H, self.d, self.P, self.dtype, self.sections = Hq, H, d, P, dtype, sections
        self.slots = torch.randperm(self.n_pages * P, device="cuda")[:rows].contiguous()
        if rows > 5:
            self.slots[3], self.slots[5] = -1, self.n_pages * P
        qkv = torch.randn(rows, Hq + 2 * H + 1, d, device="cuda") * torch.randn(Hq + 2 * H + 1, d, device="cuda").exp()
        self.qkv = qkv.to(dtype)
        self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + H], self.qkv[:, Hq + H:Hq + 2 * H]
        self.q_out = torch.empty((rows, Hq, d), dtype=dtype, device="cuda") if Hq else None
        self.args = {}
        self.weights = {}
        if sections:
            self.pos = torch.randint(0, 100000, (len(sections), rows), device="cuda", dtype=torch.int32)
            self.args.update(positions=self.pos, sections=sections, rope_theta=THETA)
        self.offset = 1.0 if norm == "offset" else 0.0
        for name in {"both": ("q", "k"), "offset": ("q", "k"), "q": ("q",), "k": ("k",)}.get(norm, ()):
            self.weights[name] = (torch.randn(d, device="cuda") * 0.3 + 1 - self.offset).to(dtype)
            self.args[name + "_norm"] = self.weights[name]
        if norm:
            self.args.update(eps=1e-5, weight_offset=self.offset)
        if Hq:
            self.args.update(q=self.q, q_out=self.q_out)

    def expected(self, name):
        """32-bit rows after norm and rotation."""
        x = f32(getattr(self, name))
        if name in self.weights:
            x = q4.head_norm(x, f32(self.weights[name]), 1e-5, self.offset)
        return q4.turn(x, self.pos.cpu().numpy(), self.sections, THETA) if self.sections else x

    def places(self):
        good = (self.slots >= 0) & (self.slots < self.n_pages * self.P)
        return good.cpu().numpy(), (self.slots[good] // self.P).cpu(), (self.slots[good] % self.P).cpu()


CASES = [(1, 4, 4, 64, 16, BF, (32,), "both"), (7, 6, 2, 128, 8, HF, (16, 24, 24), "offset"),
         (301, 8, 8, 128, 64, BF, (10, 54), "both"), (2500, 2, 3, 64, 1024, BF, (8, 12, 12), "k"),
         (1300, 3, 1, 128, 16, HF, (0, 60, 4, 0), None), (40, 5, 5, 64, 32, HF, None, "q"),
         (13, 0, 2, 64, 16, BF, (32,), "both"), (129, 1, 2, 128, 128, BF, None, None), (9731, 1, 1, 64, 8, BF, (32,), "both")]


@pytest.mark.parametrize("rows,Hq,H,d,P,dtype,sections,norm", CASES)
@pytest.mark.parametrize("layout", ["heads", "slots"])
def test_store_norm(rows, Hq, H, d, P, dtype, sections, norm, layout):
    s = Scene(rows, Hq, H, d, P, dtype, sections, norm)
    kept = s.qkv.clone()
    shape = (3, s.n_pages, H, P, d) if layout == "heads" else (3, s.n_pages, P, H, d)
    pools = [torch.randn(shape, device="cuda").to(dtype) for _ in range(2)]
    pools = [t if layout == "heads" else t.transpose(2, 3) for t in pools]
    want = [t.cpu().clone() for t in pools]
    tv.paged_kv_store_norm(tv.Pages(*pools), s.slots, s.k, s.v, layer=1, **s.args)
    torch.cuda.synchronize()
    assert torch.equal(bits(s.qkv), bits(kept))
    good, page, at = s.places()
    want[0][1].transpose(1, 2)[page, at] = rows_like(s.expected("k")[good], dtype)
    want[1][1].transpose(1, 2)[page, at] = s.v.cpu()[torch.from_numpy(good)]
    for pool, w in zip(pools, want):  # the rows, and nothing else
        assert torch.equal(bits(pool), bits(w))
    if Hq:
        assert torch.equal(bits(s.q_out), bits(rows_like(s.expected("q"), dtype)))


@pytest.mark.parametrize("rows,Hq,H,d,P,dtype,sections,norm", CASES)
@pytest.mark.parametrize("side", [False, True])
def test_store_q4_and_load(rows, Hq, H, d, P, dtype, sections, norm, side):
    s = Scene(rows, Hq, H, d, P, dtype, sections, norm, seed=1)
    n = tv.q4_page_bytes(P, d)
    if side:  # K and V of a head side by side, pages outermost
        both = torch.randint(0, 256, (s.n_pages, 3, H, 2, n), dtype=torch.uint8, device="cuda")
        pools = [both[:, :, :, i].transpose(0, 1) for i in range(2)]
    else:
        pools = [torch.randint(0, 256, (3, s.n_pages, H, n), dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [t.cpu().numpy().copy() for t in pools]
    pages = tv.PagesQ4(*pools, P, d, dtype)
    tv.paged_kv_store_q4(pages, s.slots, s.k, s.v, layer=2, **s.args)
    torch.cuda.synchronize()
    good, page, at = (np.asarray(x) for x in s.places())
    stored = {}
    for name, x, w in (("k", s.expected("k"), want[0]), ("v", f32(s.v), want[1])):
        codes, scales = q4.parts(w, P, d)  # views of w
        c, b = q4.quantize(x[good])
        codes[2, page, :, at], scales[2, page, :, at] = c, b
        stored[name] = q4.values(c, b)
    for pool, w in zip(pools, want):
        assert np.array_equal(pool.cpu().numpy(), w)
    if Hq:
        assert torch.equal(bits(s.q_out), bits(rows_like(s.expected("q"), dtype)))
    # and back: exact, padding left alone
    out = [torch.full((rows, H, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    tv.paged_kv_load_q4(pages, s.slots, *out, layer=2)
    torch.cuda.synchronize()
    for x, name in zip(out, "kv"):
        got = x.double().cpu().numpy()
        assert np.array_equal(got[good], stored[name]) and (got[~good] == 7.0).all()


# (query heads, kv heads, head_dim): 16-byte places of a row that fill 256, 192, 224, 160 or 128 threads, or whole rows
# of which do, or none
@pytest.mark.parametrize("Hq,H,d", [(16, 8, 128), (32, 8, 128), (40, 8, 128), (24, 8, 128), (0, 8, 128), (4, 1, 64),
                                    (33, 1, 128), (1, 1, 64)])
@pytest.mark.parametrize("rows", [3, 700, 5003])
def test_shapes_of_the_work(Hq, H, d, rows):
    s = Scene(rows, Hq, H, d, 16, BF, (d // 2,), "both" if Hq else "k", seed=2)
    pages = tv.make_pages_q4(1, s.n_pages, H, 16, d, BF)
    tv.paged_kv_store_q4(pages, s.slots, s.k, s.v, **s.args)
    got = [torch.zeros((rows, H, d), dtype=BF, device="cuda") for _ in range(2)]
    tv.paged_kv_load_q4(pages, s.slots, *got)
    torch.cuda.synchronize()
    good, _, _ = s.places()
    at = np.unique(np.concatenate([np.arange(min(rows, 10)), np.arange(rows - 3, rows), np.arange(0, rows, 97)]))
    for name, x in (("k", got[0]), ("v", got[1]), ("q", s.q_out)):
        if x is None:
            continue
        part = Scene.__new__(Scene)
        part.__dict__.update(s.__dict__)
        part.pos, part.k, part.q, part.v = s.pos[:, at], s.k[at], s.q[at], s.v[at]
        want = part.expected(name) if name != "v" else f32(part.v)
        if name == "q":
            assert torch.equal(bits(x[at]), bits(rows_like(want, BF)))
        else:
            want = q4.values(*q4.quantize(want)) * good[at][:, None, None]
            assert np.array_equal(x[at].double().cpu().numpy(), want)


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, HF), (128, BF)])
def test_load_of_layers(d, dtype):
    torch.manual_seed(d)
    layers, n_pages, H, P = 5, 9, 3, 32
    pools = [torch.randint(0, 256, (layers, n_pages, H, tv.q4_page_bytes(P, d)), dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    for p in pools:
        q4.parts(p, P, d)[1].clamp_(max=240)  # numbers
    slots = torch.randint(0, n_pages * P, (77,), device="cuda")
    slots[5], slots[9], slots[10] = slots[4], -1, n_pages * P + 3  # one twice, padding
    wide = torch.full((3, 80, 2 * H + 1, d), 7.0, dtype=dtype, device="cuda")
    k, v = wide[:, 1:78, :H], wide[:, 1:78, H:2 * H]
    tv.paged_kv_load_q4(tv.PagesQ4(*pools, P, d, dtype), slots, k, v, layer=1)
    torch.cuda.synchronize()
    good = (slots >= 0) & (slots < n_pages * P)
    page, at, good = (slots[good] // P).cpu().numpy(), (slots[good] % P).cpu().numpy(), good.cpu().numpy()
    want = np.full((3, 80, 2 * H + 1, d), 7.0)
    for i, p in enumerate(pools):
        codes, scales = q4.parts(p.cpu().numpy(), P, d)
        x = q4.values(codes, scales)[1:4]                       # [layers][pages][heads][slots][d]
        rows = x.transpose(0, 1, 3, 2, 4)[:, page, at]
        want[:, 1:78][:, good, i * H:(i + 1) * H] = rows
    with np.errstate(over="ignore"):
        want = rows_like(want, torch.float64).to(dtype).double().numpy()  # 15 * 57344 is past fp16: an infinity
    assert np.array_equal(wide.double().cpu().numpy(), want)


def test_every_scale_and_code():
    """A group for every scale byte that is written and every code: values times 1, 1/2 beside them (ties), and the
    last bit above."""
    rows = []
    for byte in range(1, 226):
        s = q4.scale_value(byte)
        for bump in (0, 1):
            top = np.float32(7 * s)
            top = np.nextafter(top, np.float32(np.inf)) if bump else top
            half = (np.arange(31) - 15) * 0.5 * s
            rows.append(np.concatenate([[top], half[:31]]))
    x = np.array(rows, np.float32).reshape(-1, 1, 32)
    x = np.concatenate([x, -x], -1)  # d 64
    # through a rotation by nothing: 16-bit operands cannot hold these, so that halves of them go in as they round
    for dtype in (BF, HF):
        t = torch.from_numpy(x).to(dtype).cuda()
        pages = tv.make_pages_q4(1, len(rows) // 8 + 1, 1, 8, 64, dtype)
        slots = torch.arange(len(rows), device="cuda")
        tv.paged_kv_store_q4(pages, slots, t, t.flip(0).contiguous())
        torch.cuda.synchronize()
        for pool, y in ((pages.k, t), (pages.v, t.flip(0))):
            codes, scales = q4.parts(pool.cpu().numpy(), 8, 64)
            c, b = q4.quantize(f32(y)[:, 0])
            assert np.array_equal(codes.reshape(-1, 32)[:len(rows)], c)
            assert np.array_equal(scales.reshape(-1, 2)[:len(rows)], b)


@pytest.mark.parametrize("norm", [False, True])
def test_the_ends_of_the_range(norm):
    """Zeros, numbers whose squares leave 32 bits, the largest ones, infinities and NaN, each in a head of its own."""
    torch.manual_seed(4)
    d, P = 128, 16
    x = torch.randn(12, 1, d)
    x[0] = 0
    x[1] *= 1e25
    x[2] *= 1e-25
    x[3] *= 3e-39
    x[4, 0, 3] = float("inf")
    x[5, 0, 70] = float("nan")
    x[6] = 3.3e38
    x[7] *= 60000
    x[8, 0, 1:] = 0
    x[9] *= 1e-6
    x[10, 0, 40] = -float("inf")
    x = x.to(BF).cuda()
    pages = tv.make_pages_q4(1, 1, 1, P, d, BF)
    slots = torch.arange(12, device="cuda")
    w = torch.linspace(0.5, 1.5, d).to(BF).cuda()
    q_out = torch.empty_like(x)
    args = dict(q_norm=w, k_norm=w, eps=1e-6) if norm else {}
    tv.paged_kv_store_q4(pages, slots, x, x, q=x, q_out=q_out, **args)
    torch.cuda.synchronize()
    y = f32(x)
    if norm:
        y = q4.head_norm(y, f32(w), 1e-6)
    assert torch.equal(torch.isnan(q_out), torch.isnan(rows_like(y, BF).cuda()))
    assert torch.equal(q_out.nan_to_num(1.5), rows_like(y, BF).cuda().nan_to_num(1.5))
    for pool, z in ((pages.k, y), (pages.v, f32(x))):
        codes, scales = q4.parts(pool.cpu().numpy(), P, d)
        c, b = q4.quantize(z[:, 0])
        assert np.array_equal(scales[0, 0, 0, :12], b)
        assert np.array_equal(codes[0, 0, 0, :12], c)


def test_in_place_queries_a_graph_and_a_stream():
    torch.manual_seed(3)
    pages = tv.make_pages_q4(1, 9, 2, 16, 64, BF)
    q, k, v = (torch.randn(50, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    w = torch.rand(64, device="cuda").bfloat16()
    pos = torch.arange(50, device="cuda", dtype=torch.int32) * 37
    slots = torch.arange(50, device="cuda") * 2
    want, rows = torch.empty_like(q), [torch.empty_like(k) for _ in range(2)]
    tv.paged_kv_store_q4(pages, slots, k, v, q=q, q_out=want, q_norm=w, k_norm=w, positions=pos, rope_theta=500000.0)
    first = [pages.k.clone(), pages.v.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pages.k.zero_(), pages.v.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tv.paged_kv_store_q4(pages, slots, k, v, q=q, q_norm=w, k_norm=w, positions=pos, rope_theta=500000.0)
        tv.paged_kv_load_q4(pages, slots, *rows)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, want) and torch.equal(pages.k, first[0]) and torch.equal(pages.v, first[1])
    with torch.cuda.stream(side):
        again = [torch.empty_like(k) for _ in range(2)]
        tv.paged_kv_load_q4(pages, slots, *again)
    torch.cuda.synchronize()
    assert torch.equal(again[0], rows[0]) and torch.equal(again[1], rows[1])


def test_offsets_past_32_bits():
    """A pool of more than 4 GB of 4-bit pages: its last pages."""
    d, P, H = 128, 16, 8
    n_pages = (5 << 30) // (H * tv.q4_page_bytes(P, d))
    pages = tv.PagesQ4(*(torch.empty((1, n_pages, H, tv.q4_page_bytes(P, d)), dtype=torch.uint8, device="cuda")
                         for _ in range(2)), P, d, BF)
    slots = torch.arange(n_pages * P - 40, n_pages * P, device="cuda")
    k, v = (torch.randn(40, H, d, device="cuda").bfloat16() for _ in range(2))
    tv.paged_kv_store_q4(pages, slots, k, v)
    rows = [torch.empty_like(k) for _ in range(2)]
    tv.paged_kv_load_q4(pages, slots, *rows)
    torch.cuda.synchronize()
    for x, got in ((k, rows[0]), (v, rows[1])):
        assert np.array_equal(got.double().cpu().numpy(), q4.values(*q4.quantize(f32(x))))


def test_norms_against_64_bits():
    """Queries against the formulas in 64 bits: three 32-bit roundings in the norm, two and the sines' in the
    rotation, each 2^-24 of at most the head's largest element, two such terms; then half a step of the type."""
    s = Scene(200, 4, 2, 128, 16, HF, (64,), "both")
    pages = tv.make_pages_q4(1, s.n_pages, 2, 16, 128, HF)
    tv.paged_kv_store_q4(pages, s.slots, s.k, s.v, **s.args)
    torch.cuda.synchronize()
    x = s.q.double().cpu().numpy()
    x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + np.float64(np.float32(1e-5))) * s.weights["q"].double().cpu().numpy()
    a = s.pos.double().cpu().numpy()[0][:, None] * THETA ** (-2.0 * np.arange(64) / 128)
    c, n = np.cos(a)[:, None], np.sin(a)[:, None]
    want = np.concatenate([x[..., :64] * c - x[..., 64:] * n, x[..., 64:] * c + x[..., :64] * n], -1)
    size = np.abs(x).max(-1, keepdims=True)
    slack = size * 2 * 6 * 2.0 ** -24 + np.abs(want) * 2.0 ** -11 + 2.0 ** -25
    assert (np.abs(s.q_out.double().cpu().numpy() - want) <= slack).all()

"""paged_kv_store against the rotation in 64 bits: axes, strides, types, padding."""
import numpy as np
import pytest
import torch

import paper_2606_27550_gb300 as tv

pytestmark = pytest.mark.gpu


def turn(x, pos, sections, theta):
    """[rows][heads][d] in 64 bits."""
    x = x.double()
    d = x.shape[2]
    axis = np.repeat(np.arange(len(sections)), sections)
    f = theta ** (-2.0 * np.arange(d // 2) / d)
    a = pos.double().cpu().numpy()[axis].T * f  # [rows][d / 2]
    c, s = (torch.from_numpy(fn(a)).to(x.device)[:, None] for fn in (np.cos, np.sin))
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def pools(layers, n_pages, H, P, d, dtype, layout):
    shape = (layers, n_pages, H, P, d) if layout == "heads" else (layers, n_pages, P, H, d)
    out = [torch.randn(shape, device="cuda").to(dtype) for _ in range(2)]
    return [t if layout == "heads" else t.transpose(2, 3) for t in out]


@pytest.mark.parametrize("rows,Hq,H,d,P,layout,dtype,sections,layer", [
    (1, 4, 4, 64, 16, "heads", torch.bfloat16, (32,), 0), (7, 6, 2, 128, 8, "slots", torch.float16, (16, 24, 24), 1),
    (301, 32, 8, 128, 64, "heads", torch.bfloat16, (10, 54), 2), (2500, 8, 8, 64, 1024, "slots", torch.bfloat16, (8, 12, 12), 0),
    (9731, 3, 1, 128, 16, "heads", torch.float16, (0, 60, 4, 0), 0), (40, 5, 5, 64, 32, "slots", torch.float16, None, 0),
    (13, 0, 2, 64, 16, "heads", torch.bfloat16, (32,), 0)])
def test_store(rows, Hq, H, d, P, layout, dtype, sections, layer):
    torch.manual_seed(rows)
    n_pages, layers, theta = rows // P + 4, 3, 10000.0
    k_pages, v_pages = pools(layers, n_pages, H, P, d, dtype, layout)
    first = [t.clone() for t in (k_pages, v_pages)]
    slots = torch.randperm(n_pages * P, device="cuda")[:rows].contiguous()
    if rows > 5:
        slots[3], slots[5] = -1, n_pages * P  # padding
    qkv = torch.randn(rows, Hq + 2 * H + 1, d, device="cuda").to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:Hq + 2 * H]
    kept = qkv.clone()
    q_out = torch.empty((rows, Hq, d), dtype=dtype, device="cuda") if Hq else None
    args = {}
    if sections:
        # positions up to what 31 bits hold: the fraction of a turn must survive
        pos = torch.randint(0, 2**31 - 1, (len(sections), rows), device="cuda", dtype=torch.int32)
        pos[:, ::2] %= 5000
        args = dict(positions=pos, sections=sections, rope_theta=theta)
    if Hq:
        args.update(q=q, q_out=q_out)
    tv.paged_kv_store(tv.Pages(k_pages, v_pages), slots, k, v, layer=layer, **args)
    torch.cuda.synchronize()
    assert torch.equal(qkv, kept)
    kt = turn(k, args["positions"], sections, theta) if sections else k.double()
    qt = turn(q, args["positions"], sections, theta) if sections else q.double()
    # 32-bit angles and products: sin and cos are off by less than 2^-21 (the angle's rounding to 24
    # bits of pi, sincospif's 2 ulp), four such terms of the largest element; then one rounding to the
    # type, which is monotone: the result lies between the rounded ends of that interval

    def near(got, want, size):
        slack = size * 2.0 ** -19
        lo, hi = (want - slack).to(dtype), (want + slack).to(dtype)
        assert bool(((got >= lo) & (got <= hi)).all())

    if Hq:
        near(q_out, qt, q.double().abs().amax())
    good = (slots >= 0) & (slots < n_pages * P)
    page, at = slots[good] // P, slots[good] % P
    got_k, got_v = k_pages[layer].transpose(1, 2)[page, at], v_pages[layer].transpose(1, 2)[page, at]
    near(got_k, kt[good], k.double().abs().amax())
    assert torch.equal(got_v, v[good])
    # nothing else moves
    for pool, was, new in ((k_pages, first[0], got_k), (v_pages, first[1], got_v)):
        want = was.clone()
        want[layer].transpose(1, 2)[page, at] = new
        assert torch.equal(pool, want)


def test_in_place_queries_and_a_graph():
    torch.manual_seed(3)
    k_pages, v_pages = pools(1, 9, 2, 16, 64, torch.bfloat16, "heads")
    q, k, v = (torch.randn(50, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
    pos = torch.arange(50, device="cuda", dtype=torch.int32) * 37
    slots = torch.arange(50, device="cuda") * 2
    want = torch.empty_like(q)
    pages = tv.Pages(k_pages, v_pages)
    tv.paged_kv_store(pages, slots, k, v, q=q, q_out=want, positions=pos, rope_theta=500000.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tv.paged_kv_store(pages, slots, k, v, q=q, positions=pos, rope_theta=500000.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, want)


def test_no_rows():
    k_pages, v_pages = pools(1, 2, 2, 16, 64, torch.bfloat16, "heads")
    none = torch.empty(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    before = k_pages.clone()
    x = torch.randn(1, 2, 64, device="cuda").bfloat16()
    tv.paged_kv_store(tv.Pages(k_pages, v_pages), torch.empty(0, dtype=torch.int64, device="cuda"), x, x)
    assert torch.equal(before, k_pages) and none.numel() == 0

"""Sines of small angles to their last bit, through the stores.

Where an angle is below 2^-12 its cosine rounds to 1, and the upper element of a pair is
fl(b + fl(a s)).  For each sine s two pairs (a, b) are searched whose result in bf16 is
another one with the next 32-bit number above s, and below it.  Sines whose exact value lies
nearer to the middle of two 32-bit numbers than the angle is known to (4 units of 2^-64 of a turn
a position) or than 2^-33 of themselves are left out."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2606_27550_gb300 as tv

BF = torch.bfloat16
TURN = Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563281257241799725607")
POSITIONS = (1, 2, 3, 4, 5, 7, 50, 1000, 65535, -1, -2, -3, -5)


def exact_sine(x):
    """x below 2^-12: five terms leave less than 2^-150."""
    y, t = x, x
    for k in range(2, 10, 2):
        t = -t * x * x / (k * (k + 1))
        y += t
    return y


def bf16(x):
    """32-bit floats rounded to bf16, to even."""
    u = x.view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def telling_pair(s, other):
    """(a, b) of 8 bits each for which fl(b + fl(a s)) rounds otherwise than with `other`, or None."""
    a = (np.arange(128, 256, dtype=np.float32) / 128)[:, None, None]
    size = np.float32(2.0) ** np.floor(np.log2(np.abs(s)))
    b = (np.arange(128, 256, dtype=np.float32) / 128)[None, :, None] * size
    b = b * np.array([-2, -1, -0.5, 0.5, -0.25, 0.25, -0.125, 0.125], np.float32)
    hit = np.argwhere(bf16(b + a * s) != bf16(b + a * other))
    return None if not len(hit) else (a[hit[0][0], 0, 0], b[0, hit[0][1], hit[0][2]])


def cases(theta, d):
    """[(row, pair, [(a, b) for the number above, (a, b) for the one below], s)]"""
    getcontext().prec = 60
    found = []
    for row, pos in enumerate(POSITIONS):
        for i in range(d // 2):
            x = pos * ((-2 * i / Decimal(d)) * Decimal(theta).ln()).exp()
            if abs(x) >= Decimal(2) ** -12:
                continue
            y = exact_sine(x)
            s = np.float32(float(y))
            beside = [np.nextafter(s, np.float32(e)) for e in (1, -1)]
            slack = abs(pos) * 4 * TURN / 2 ** 64 + abs(y) / 2 ** 33
            if any(abs(y - (Decimal(float(s)) + Decimal(float(o))) / 2) <= slack for o in beside):
                continue
            pairs = [telling_pair(s, o) for o in beside]
            if None not in pairs:
                found.append((row, i, pairs, s))
    return found


def test_the_search():
    """What is told apart: most pairs of the case below, each by a last bit."""
    found = cases(1e9, 64)
    assert len(found) > 60
    for _, _, pairs, s in found[::7]:
        for (a, b), other in zip(pairs, (np.nextafter(s, np.float32(1)), np.nextafter(s, np.float32(-1)))):
            assert bf16(np.float32([b + a * s])) != bf16(np.float32([b + a * other]))


@pytest.mark.gpu
@pytest.mark.parametrize("theta,d", [(1e9, 128), (2e9, 128), (3e9, 128), (4e9, 128), (5e9, 128), (3e9, 64), (5e6, 64)])
def test_sines_of_small_angles(theta, d):
    found = cases(theta, d)
    assert len(found) > 60
    rows, H = len(POSITIONS), 2
    k = np.zeros((rows, H, d), np.float32)
    want = np.zeros((rows, H, d), np.float32)
    told = np.zeros((rows, H, d), bool)
    for row, i, pairs, s in found:
        for h, (a, b) in enumerate(pairs):
            k[row, h, i], k[row, h, i + d // 2] = a, b
            want[row, h, i + d // 2] = bf16(np.float32([b + a * s]))[0]
            told[row, h, i + d // 2] = True
    x = torch.from_numpy(k).to(BF).cuda()
    assert np.array_equal(x.float().cpu().numpy(), k)
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device="cuda")
    pages = tv.Pages(*(torch.zeros((1, 2, H, 16, d), dtype=BF, device="cuda") for _ in range(2)))
    q = torch.empty_like(x)
    tv.paged_kv_store_norm(pages, torch.arange(rows, device="cuda"), x, x, q=x, q_out=q, positions=pos, rope_theta=theta)
    q4 = tv.make_pages_q4(1, 2, H, 16, d, BF)
    q_too = torch.empty_like(x)
    tv.paged_kv_store_q4(q4, torch.arange(rows, device="cuda"), x, x, q=x, q_out=q_too, positions=pos, rope_theta=theta)
    torch.cuda.synchronize()
    for got in (pages.k[0, 0].transpose(0, 1)[:rows], q, q_too):
        wrong = (got.float().cpu().numpy() != want) & told
        assert not wrong.any(), f"{wrong.sum()} of {told.sum()}"

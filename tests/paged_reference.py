"""Plain references of the paged serving calls (loops, 64 bits) and the inputs
of their tests.  They share nothing with the library but synth's tree shapes."""
from __future__ import annotations

import numpy as np

import oracle
from paper_2606_27550_gb300 import synth

EINVAL, ECAPACITY = -1, -5


def trees():
    """Topologies in canonical order: the bank's trees, a chain, a star, a random one."""
    g = synth.rng(41)
    rnd = np.array([-1] + sorted(int(g.integers(0, i)) for i in range(1, 37)), np.int32)
    return [*synth.bank_trees(), synth.chain(20), np.array([-1] + [0] * 11, np.int32), rnd]


def ancestors(parent):
    n = len(parent)
    a = np.zeros((n, n), bool)
    for i in range(n):
        u = i
        while u >= 0:
            a[i, u] = True
            u = parent[u]
    return a


def plan(lens, n_new, held, state, ring, table, page, max_rows, bad=()):
    """(status, row_start, slots, positions offsets i, held, state, ring, table) of a step, one
    request after the other; bad: requests with an unknown tree."""
    B, n_pages = len(lens), len(ring)
    head, free = state
    ring, table, held = ring.copy(), table.copy(), list(held)
    status, n = [0] * B, list(n_new)
    need = [0] * B
    for b in range(B):
        if b in bad or lens[b] < 0 or n[b] < 0:
            status[b] = EINVAL
        elif -(-(lens[b] + n[b]) // page) > table.shape[1]:
            status[b] = ECAPACITY
        if status[b]:
            n[b] = 0
            need[b] = held[b]
        else:
            need[b] = -(-(lens[b] + n[b]) // page)
    rows = 0
    fits = []
    for b in range(B):
        rows += n[b]
        fits.append(not (n[b] > 0 and rows > max_rows))
    for b in range(B):
        if not fits[b]:
            status[b], n[b], need[b] = ECAPACITY, 0, held[b]
    taken = 0
    for b in range(B):
        want = max(0, need[b] - held[b])
        taken += want
        if want and taken > free:
            status[b], n[b], need[b] = ECAPACITY, 0, held[b]
    given = []
    taken = 0
    for b in range(B):
        for p in range(held[b], need[b]):
            table[b, p] = ring[(head + taken) % n_pages]
            taken += 1
    for b in range(B):
        given += [table[b, p] for p in range(need[b], held[b])]
    for i, x in enumerate(given):
        ring[(head + free + i) % n_pages] = x
    row_start = np.concatenate([[0], np.cumsum(n)])
    slots = np.full(max_rows, -1, np.int64)
    at = np.zeros((max_rows, 2), np.int64)  # (request, index) of each row
    for b in range(B):
        for i in range(n[b]):
            s = lens[b] + i
            pg = table[b, s // page]
            slots[row_start[b] + i] = pg * page + s % page if pg >= 0 else -1
            at[row_start[b] + i] = b, i
    return status, row_start, slots, at, need, ((head + taken) % n_pages, free - taken + len(given)), ring, table


def attend(q, k, v, parent, L, scale, cap=0.0, slopes=None, window=0, sink=0, begin=0):
    """(out, lse, |V| average, largest |z| that matters) of one request: q [n][Hq][d],
    k, v [L + n][Hkv][d], 64-bit."""
    n, Hq, d = q.shape
    Hkv = k.shape[1]
    dep = synth.depth_of(parent)
    anc = ancestors(parent)
    pos = np.concatenate([np.arange(L), L + dep])
    out, absv = np.zeros((n, Hq, d)), np.zeros((n, Hq, d))
    lse, big = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    for i in range(n):
        see = np.concatenate([np.ones(L, bool), anc[i]])
        dist = L + dep[i] - pos
        s = np.arange(L + n)
        if window:
            see &= (dist < window) | (s < begin + sink)
        see &= s >= begin
        if not see.any():
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            z = (k[see, g] @ q[i, h]) * scale
            if cap:
                z = cap * np.tanh(z / cap)
            if slopes is not None:
                z = z - slopes[h] * dist[see]
            m = z.max()
            p = np.exp(z - m)
            out[i, h] = p @ v[see, g] / p.sum()
            absv[i, h] = p @ np.abs(v[see, g]) / p.sum()
            lse[i, h] = m + np.log(p.sum())
            big[i, h] = np.abs(z[p > 2.0 ** -30]).max()
    return out, lse, absv, big


def process(z, rep, freq, pres, prompt, made, paths, bias, allowed):
    """Penalties, biases and masks of one request's rows [n][V] in 32-bit steps (numpy), in the
    documented order; prompt, made: token lists; paths: a list of tokens per row; bias: (token, value)s."""
    z = z.astype(np.float32).copy()
    n, V = z.shape
    ok = lambda ts: [t for t in ts if 0 <= t < V]  # noqa: E731
    base_p = np.bincount(ok(prompt), minlength=V)
    base_m = np.bincount(ok(made), minlength=V)
    b = np.zeros(V, np.float32)
    for t, x in bias:
        if 0 <= t < V:
            b[t] = np.float32(b[t] + np.float32(x))
    with np.errstate(all="ignore"):
        for i in range(n):
            count = base_m + np.bincount(ok(paths[i]), minlength=V)
            seen = (count > 0) | (base_p > 0)
            r = np.float32(rep)
            z[i] = np.where(seen, np.where(z[i] > 0, z[i] / r, z[i] * r), z[i])
            c = count.astype(np.float32)
            z[i] = np.where(count > 0, (z[i] - np.float32(freq) * c).astype(np.float32) - np.float32(pres), z[i])
            z[i] = z[i] + b
            if allowed is not None:
                z[i] = np.where(allowed[i], z[i], -np.inf)
    return z


def stats(z, T):
    """(argmax, top1, entropy, logz_t, entropy_t) of one 32-bit row, in 64 bits."""
    z = z.astype(np.float64)
    m = z.max()
    if m == -np.inf:
        return -1, 0.0, 0.0, -np.inf, 0.0
    res = []
    for t in (1.0, T):
        x = (z - m) / t
        e = np.exp(x)
        s = e.sum()
        res.append((m / t + np.log(s), np.log(s) - np.where(e > 0, e * np.where(e > 0, x, 0), 0).sum() / s, 1 / s))
    return int(np.argmax(z)), res[0][2], res[0][1], res[1][0], res[1][1]


def accept(parent, draft, argmax):
    return oracle.accept(parent, draft, argmax)

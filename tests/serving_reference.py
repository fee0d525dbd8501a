"""Plain forms in 64 bits (and whole numbers) of the operators for packed prompts and paged caches, written from their
definitions: loops over sequences, layers and heads."""
import math

import numpy as np


def pages_of(n, ps):
    return -(-n // ps)


def resize(lens, target, table, ring, state, ps):
    """-> (accepted status, lens, table, ring, state) after every segment has its target length; all or nothing."""
    P, width = len(ring), table.shape[2]
    head, count = int(state[0]), int(state[1])
    lens, table, ring = lens.copy(), table.copy(), ring.copy()
    old_ring = ring.copy()
    bad = (lens < 0).any() or (target < 0).any() or (lens > width * ps).any() or (target > width * ps).any()
    if bad or not 0 <= head < P or not 0 <= count <= P:
        return 2, lens, table, ring, np.array(state)
    held = [[pages_of(int(x), ps) for x in row] for row in lens]
    want = [[pages_of(int(x), ps) for x in row] for row in target]
    more = sum(max(0, w - h) for a, b in zip(held, want) for h, w in zip(a, b))
    less = sum(max(0, h - w) for a, b in zip(held, want) for h, w in zip(a, b))
    status = (1 if more > count else 0) | (2 if count - more + less > P else 0)
    if status:
        return status, lens, table, ring, np.array(state)
    take, give = head, head + count
    for s in range(lens.shape[0]):
        for l in range(lens.shape[1]):
            for j in range(held[s][l], want[s][l]):
                table[s, l, j] = old_ring[take % P]
                take += 1
            for j in range(want[s][l], held[s][l]):
                ring[give % P] = table[s, l, j]
                give += 1
    return 0, target.copy(), table, ring, np.array([take % P, count - more + less])


def append(lens, row_off, T, table, ring, state, ps):
    n = np.diff(row_off)
    S, layers = lens.shape
    slots = np.full((layers, T), -1, dtype=np.int64)
    if row_off[0] < 0 or (n < 0).any() or row_off[-1] > T:
        return 2, lens.copy(), table.copy(), np.array(state), slots
    status, new, table, _, state = resize(lens, lens + n[:, None], table, ring, state, ps)
    if status == 0:
        for s in range(S):
            for l in range(layers):
                for i in range(n[s]):
                    pos = lens[s, l] + i
                    slots[l, row_off[s] + i] = table[s, l, pos // ps] * ps + pos % ps
    return status, new, table, state, slots


def rope(x, pos, axis, theta, rot, interleaved):
    """x [L,h,T,D] f64, pos [axes,T] -> rotated."""
    y = x.copy()
    for i in range(rot // 2):
        angle = pos[axis[i]].astype(np.float64) * theta ** (-2.0 * i / rot)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = np.cos(angle), np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def attend(q, k, v, scale, first_limit):
    """Row i of q [n,D] sees keys 0 ... first_limit + i of k, v [m,D] -> (out, sum of p*|v|, lse).  Values that no row sees
    never enter a sum."""
    n, D = q.shape
    out, mag, lse = np.zeros((n, D)), np.zeros((n, D)), np.full(n, -math.inf)
    for i in range(n):
        c = min(first_limit + i + 1, k.shape[0])
        if c <= 0:
            continue
        z = (k[:c] @ q[i]) * scale
        m = z.max()
        if m == -math.inf:
            continue
        e = np.exp(z - m)
        p = e / e.sum()
        out[i], mag[i], lse[i] = p @ v[:c], p @ np.abs(v[:c]), m + math.log(e.sum())
    return out, mag, lse


def prompt(q, k, v, row_off, scale):
    """q [L,H,T,D], k,v [L,Hkv,T,D] f64 -> (out, mag, lse packed as [L,H,n] per sequence); rows of nobody are NaN."""
    L, H, T, D = q.shape
    grp = H // k.shape[1]
    out, mag, lse = (np.full(q.shape, np.nan), np.full(q.shape, np.nan), np.full(L * H * T, np.nan))
    for a, b in zip(row_off[:-1], row_off[1:]):
        for l in range(L):
            for h in range(H):
                o, m, z = attend(q[l, h, a:b], k[l, h // grp, a:b], v[l, h // grp, a:b], scale[l], 0)
                out[l, h, a:b], mag[l, h, a:b] = o, m
                at = L * H * a + (l * H + h) * (b - a)
                lse[at:at + b - a] = z
    return out, mag, lse


def cached(pool, table_row, size, g, ps):
    """Entries 0 ... size-1 of one KV head; those on pages outside the pool are left out -> (rows, their entries)."""
    keep = [j for j in range(size) if 0 <= table_row[j // ps] < pool.shape[0]]
    return np.array([pool[table_row[j // ps], g, j % ps] for j in keep]).reshape(-1, pool.shape[3]), np.array(keep, dtype=int)


def chunk(q, row_off, kp, vp, table, lens, scale, l0=0, max_rows=None):
    L, H, T, D = q.shape
    grp, ps = H // kp.shape[1], kp.shape[2]
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s, (a, b) in enumerate(zip(row_off[:-1], row_off[1:])):
        stop = b if max_rows is None else min(b, a + max_rows)
        for l in range(L):
            size = int(lens[s, l0 + l])
            for h in range(H):
                ks, keep = cached(kp, table[s, l0 + l], size, h // grp, ps)
                vs, _ = cached(vp, table[s, l0 + l], size, h // grp, ps)
                for t in range(a, stop):
                    c = int((keep <= size - (b - a) + (t - a)).sum())
                    o, m, _ = attend(q[l, h, t:t + 1], ks[:c], vs[:c], scale[l], c - 1)
                    out[l, h, t], mag[l, h, t] = o[0], m[0]
    return out, mag

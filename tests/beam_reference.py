"""Plain forms in 64 bits (and whole numbers) of beam search over a paged cache and of attention to states of another length,
written from their definitions: loops over prompts, places, layers and heads."""
import math

import numpy as np

from serving_reference import attend, pages_of

LARGEST = float(np.finfo(np.float32).max)


def cleaned(x):
    return np.where(np.isnan(x), -np.inf, np.minimum(x, LARGEST))


def candidates(logits, scores, ended, end):
    """All continuations of one prompt, logits [W,V] f64 -> [(score, place w * V + v)], best first."""
    W, V = logits.shape
    logits, scores = cleaned(logits), cleaned(scores)
    found = []
    for w in range(W):
        if ended is not None and ended[w]:
            if scores[w] > -np.inf:
                found.append((scores[w], w * V + end))
            continue
        if scores[w] == -np.inf:
            continue
        m = logits[w].max()
        if m == -np.inf:
            continue
        lse = m + math.log(np.exp(logits[w] - m).sum())
        keep = np.nonzero(logits[w] > -np.inf)[0]
        order = keep[np.argsort(-logits[w][keep], kind="stable")][:W + 1]
        found += [((logits[w, v] - lse) + scores[w], w * V + int(v)) for v in order]
    return sorted(found, key=lambda c: (-c[0], c[1]))


def select(logits, scores, ended, end):
    """logits [S,W,V] f64 -> (tokens, parents, scores, ended, the smallest difference that a choice or an order hangs on between
    beams)."""
    S, W, V = logits.shape
    tokens, parents = np.full((S, W), -1), np.full((S, W), -1)
    best, over = np.full((S, W), -np.inf), np.zeros((S, W), dtype=bool)
    gap = np.inf
    for s in range(S):
        found = candidates(logits[s], scores[s], None if ended is None else ended[s], end)
        for i, (score, at) in enumerate(found[:W]):
            w, v = divmod(at, V)
            tokens[s, i], parents[s, i], best[s, i] = v, w, score
            over[s, i] = end is not None and (v == end or (ended is not None and ended[s][w]))
        for (a, x), (b, y) in zip(found[:W], found[1:W + 1]):
            if x // V != y // V and a != b:
                gap = min(gap, a - b)
    return tokens, parents, best, over, gap


def reorder(parents, table, lens, ring, state, ps, pools=()):
    """-> (status, table, lens, ring, state, pools); place by place.  Pages are followed by who holds them."""
    G, W = parents.shape
    S, layers, width = table.shape
    P, (head, count) = len(ring), (int(x) for x in state)
    same = (table.copy(), lens.copy(), ring.copy(), np.array(state), [x.copy() for x in pools])
    if ((parents < -1) | (parents >= W)).any() or ((lens < 0) | (lens > width * ps)).any() or not 0 <= head < P or not 0 <= count <= P:
        return (2, *same)
    new_table, new_lens, new_ring, _, new_pools = (x if isinstance(x, list) else x.copy() for x in same)
    taken, copies = 0, []
    for s in range(S):
        g, i = divmod(s, W)
        p = parents[g, i]
        again = p >= 0 and p in parents[g, :i]
        for l in range(layers):
            n = int(lens[g * W + p, l]) if p >= 0 else 0
            new_lens[s, l] = n
            new_table[s, l, :pages_of(n, ps)] = table[g * W + p, l, :pages_of(n, ps)] if p >= 0 else 0
            if again and n % ps:
                copies.append((s, l, n // ps, table[g * W + p, l, n // ps], n % ps, taken))
                taken += 1
    for s, l, j, _, _, k in copies:
        new_table[s, l, j] = ring[(head + k) % P]
    given = []
    for s in range(S):
        g = s // W * W
        for l in range(layers):
            for j in range(pages_of(int(lens[s, l]), ps)):
                page = table[s, l, j]
                kept = any(new_table[x, l, j] == page and j < pages_of(int(new_lens[x, l]), ps) and
                           not any(c[0] == x and c[1] == l and c[2] == j for c in copies) for x in range(g, g + W))
                lower = any(table[x, l, j] == page and j < pages_of(int(lens[x, l]), ps) for x in range(g, s))
                if not kept and not lower and 0 <= page < P:
                    given.append(page)
    if count + len(given) > P:
        return (2, *same)
    if taken > count:
        return (1, *same)
    for k, page in enumerate(given):
        new_ring[(head + count + k) % P] = page
    for _, _, _, src, rows, k in copies:
        dst = ring[(head + k) % P]
        for pool in new_pools:
            pool[dst, :, :rows] = pool[src, :, :rows]
    return 0, new_table, new_lens, new_ring, np.array([(head + taken) % P, count - taken + len(given)]), new_pools


def cross(q, row_off, k, v, state_off, scale, seen=None, max_rows=None):
    """q [L,H,T,D], k,v [L,Hkv,M,D] f64 -> (out, sum of p*|v|); rows of nobody are NaN."""
    L, H, T, D = q.shape
    grp = H // k.shape[1]
    out, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s, (a, b) in enumerate(zip(row_off[:-1], row_off[1:])):
        stop = b if max_rows is None else min(b, a + max_rows)
        x, y = state_off[s], state_off[s + 1]
        for t in range(a, stop):
            n = y - x if seen is None else max(0, min(int(seen[t]), y - x))
            for l in range(L):
                for h in range(H):
                    o, m, _ = attend(q[l, h, t:t + 1], k[l, h // grp, x:x + n], v[l, h // grp, x:x + n], scale[l], n - 1)
                    out[l, h, t], mag[l, h, t] = o[0], m[0]
    return out, mag

"""Timed cases of the operators that carry several continuations of a prompt over the paged cache, and of attention to
states of another length.

A program that searches with beams holds W continuations of every prompt in W places of the cache, one behind the
other.  After a decoding step the W best of all beams' continuations are chosen (`select`), the places become what
their new beams continue (`reorder`: pages are shared, only the page that the next token goes into is copied), and the
new rows attend to their own cache and, in a model with an encoder, to the states of the prompt's encoder, which all
beams share (`cross`).

`kind` of a case:
  select   prefixkv_beam_select: the W best of W*V continuations of every prompt, with their scores
  reorder  prefixkv_page_reorder: the places of a group become copies of some of them
  cross    prefixkv_cross_attn: rows attend to all states of their memory, or with `seen` to the first ones

Where `own` is false the steps are computed in elementary torch operations: in 32 bits, the scores of continuations
and the logarithms that they are made of, which choices hang on, in 64.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


# ---- the cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # One prompt, four beams, a vocabulary of 32000: the step between two tokens of a single request; pure latency.
        dict(name="select_one", kind="select", dtype="bf16", S=1, W=4, V=32000, lens=1),
        # 64 requests of four beams, logits in 32 bits and a large vocabulary: bandwidth.
        dict(name="select_batch", kind="select", dtype="f32", S=64, W=4, V=128000, lens=2),
        # Wide beams over a vocabulary of odd size, whose rows begin anywhere.
        dict(name="select_wide", kind="select", dtype="bf16", S=8, W=32, V=100003, lens=3),
        # One request of four beams over the compressed cache of a 7B prompt, small pages: latency.
        dict(name="reorder_one", kind="reorder", dtype="bf16", S=1, W=4, L=32, Hkv=32, D=128, ps=16, ctx=400, new=100, lens=4),
        # Eight requests of four beams, grouped-query caches of 32 layers, larger pages: partly filled pages are copied.
        dict(name="reorder_many", kind="reorder", dtype="bf16", S=8, W=4, L=32, Hkv=8, D=128, ps=64, ctx=700, new=150, lens=5),
        # A prompt's cache is forked into eight beams, the storage type and heads of the validation shape.
        dict(name="reorder_fork", kind="reorder", dtype="f32", S=3, W=8, L=4, Hkv=2, D=64, ps=32, ctx=500, new=0, lens=6),
        # One token of one sequence over the states of a picture: latency.
        dict(name="cross_token", kind="cross", dtype="bf16", S=1, L=1, H=32, Hkv=8, rows=1, states=577, D=128, seen=False, lens=7),
        # A decoding step of 32 requests of four beams each, which share their request's states: bandwidth.
        dict(name="cross_beams", kind="cross", dtype="bf16", S=32, L=1, H=32, Hkv=32, rows=4, states=2880, D=128, seen=False,
             lens=8),
        # Prompts of up to 700 rows that see the pictures in front of them, one of them without any.
        dict(name="cross_pictures", kind="cross", dtype="bf16", S=6, L=1, H=32, Hkv=8, rows=700, states=2885, D=128, seen=True,
             lens=9),
        # One layer of two long texts over long recordings: the largest product.
        dict(name="cross_long", kind="cross", dtype="bf16", S=2, L=1, H=32, Hkv=8, rows=4001, states=6001, D=128, seen=False,
             lens=10),
        # The validation shape: a few rows in 32 bits over short states, all layers in a call.
        dict(name="cross_tiny_f32", kind="cross", dtype="f32", S=2, L=4, H=2, Hkv=2, rows=12, states=130, D=64, seen=False, lens=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    w = work(c)
    return w["bytes"] / 3e12 + w["flops"] / 4e14


def draw(rng):
    limit = {}
    for c in listed():
        limit[c["kind"]] = max(limit.get(c["kind"], 0.0), _cost(c))
    kind = rng.choice(["select", "select", "reorder", "reorder", "cross", "cross", "cross"])
    while True:
        D, seed = rng.choice([128, 128, 64]), rng.randrange(1 << 20)
        if kind == "select":
            c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), S=_log_int(rng, 1, 96), W=rng.choice([1, 2, 3, 4, 4, 5, 8, 16, 32]),
                     V=_log_int(rng, 1000, 160000), lens=seed)
        elif kind == "reorder":
            f32 = rng.random() < 0.25
            c = dict(kind=kind, dtype="f32" if f32 else "bf16", S=_log_int(rng, 1, 24), W=rng.choice([2, 3, 4, 4, 5, 8, 16]),
                     L=rng.choice([1, 4, 24, 32, 40]), Hkv=rng.choice([1, 2] if f32 else [4, 8, 8, 24, 32]), D=D,
                     ps=rng.choice([16, 16, 32, 64, 128]), ctx=_log_int(rng, 20, 2000),
                     new=rng.choice([0, _log_int(rng, 1, 400), _log_int(rng, 1, 400)]), lens=seed)
        else:
            f32 = rng.random() < 0.15
            H, Hkv = rng.choice([(2, 2), (4, 2), (4, 1)] if f32 else [(32, 32), (40, 40), (32, 8), (32, 4), (16, 8), (24, 24), (12, 4), (28, 4)])
            c = dict(kind=kind, dtype="f32" if f32 else "bf16", S=_log_int(rng, 1, 48), L=rng.choice([1, 1, 1, 4]), H=H, Hkv=Hkv,
                     rows=rng.choice([1, 4, 8, _log_int(rng, 2, 64 if f32 else 4000), _log_int(rng, 2, 64 if f32 else 4000)]),
                     states=_log_int(rng, 16, 400 if f32 else 8192), D=D, seen=rng.random() < 0.4, lens=seed)
        # a plain form holds the pool, the padded scores or the vocabulary in 64 bits several times over
        if _cost(c) <= limit[kind] and _held(c) <= 2e9:
            return c


def _held(c):
    if c["kind"] == "select":
        return 8 * c["S"] * c["W"] * c["V"]
    if c["kind"] == "reorder":
        rows = c["S"] * c["L"] * (c["ctx"] + c["W"] * (c["new"] + c["ps"]))
        return 2 * rows * c["Hkv"] * c["D"] * (4 if c["dtype"] == "f32" else 2)
    return c["S"] * c["L"] * max(c["H"] * c["rows"], c["Hkv"] * c["D"]) * c["states"]


# ---- sizes of a case: lengths are the case's own, values are the seed's ---------------------------------
def _spread(rng, n, lo, hi):
    """n whole numbers from lo to hi, evenly over the logarithm, the first of them hi."""
    got = [hi] + [int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)))))) for _ in range(n - 1)]
    return [min(max(x, lo), hi) for x in got]


def _rows(c):
    """Rows that attend to every memory: beams are as many everywhere, texts differ."""
    if c["rows"] <= 8:
        return [c["rows"]] * c["S"]
    return _spread(random.Random(c["lens"]), c["S"], max(1, c["rows"] // 20), c["rows"])


def _states(c):
    return _spread(random.Random(c["lens"] + 1), c["S"], max(1, c["states"] // 4), c["states"])


def _seen(c):
    """How many states of its memory a row sees: pictures lie between the rows, and the first rows have none in front."""
    r = random.Random(c["lens"] + 2)
    got = []
    for i, (n, m) in enumerate(zip(_rows(c), _states(c))):
        pictures = max(1, m // 577)
        at = sorted(r.randrange(n + 1) for _ in range(pictures))
        if i == 1:
            at = [n] * pictures                          # a text without a picture in front of it
        got.append([sum(1 for a in at if a <= t) * m // pictures for t in range(n)])
    return got


def _prompt_lengths(c):
    """What the search left of every layer of a prompt: layers differ, the beams of a prompt do not."""
    r = random.Random(c["lens"] + 3)
    got = [[max(1, int(c["ctx"] * math.exp(-r.uniform(0.0, 1.5)))) for _ in range(c["L"])] for _ in range(c["S"])]
    got[0][0] = c["ctx"]
    return got


def _parents(c):
    """Which place every place continues.  A fork continues the first place everywhere; else as the best continuations of a
    step are spread: some beams have several, as many others none.  The last prompt of many has ended."""
    r = random.Random(c["lens"] + 4)
    if c["new"] == 0:
        return [[0] * c["W"] for _ in range(c["S"])]
    got = [[min(int(r.expovariate(1.0) * c["W"] / 2.5), c["W"] - 1) for _ in range(c["W"])] for _ in range(c["S"])]
    if c["S"] > 3:
        got[-1] = [-1] * c["W"]
    return got


def _pages(n, ps):
    return -(-n // ps)


def _layout(c):
    """Lengths [S*W, L] and, per (prompt, layer), how many leading pages all beams share, and how many pairs of beams."""
    n, new, ps = torch.tensor(_prompt_lengths(c)), c["new"], c["ps"]
    r = random.Random(c["lens"] + 5)
    common = torch.tensor([[int(new * r.uniform(0.0, 0.5))] for _ in range(c["S"])])
    paired = common + torch.tensor([[int(new * r.uniform(0.0, 0.4))] for _ in range(c["S"])])
    total = (n + new)[:, None, :].expand(-1, c["W"], -1).clone()
    if new == 0:
        total[:, 1:] = 0                                     # the other places are empty before a fork
    return total.reshape(-1, c["L"]), (n + common) // ps, (n + paired) // ps


def _copied(c):
    """Rows that a reordering copies, per layer and tensor, over all places, and the pages that it takes."""
    lens, _, _ = _layout(c)
    part = (lens % c["ps"]).view(c["S"], c["W"], c["L"])
    rows = pages = 0
    for g, parents in enumerate(_parents(c)):
        for p in set(parents) - {-1}:
            more = parents.count(p) - 1
            rows += more * int(part[g, p].sum())
            pages += more * int((part[g, p] > 0).sum())
    return rows, pages


def work(c):
    k = c["kind"]
    e = 4 if c["dtype"] == "f32" else 2
    if k == "select":
        rows = c["S"] * c["W"]
        return {"bytes": float(e) * rows * c["V"] + 18.0 * rows, "flops": 3.0 * rows * c["V"]}
    if k == "reorder":
        rows, pages = _copied(c)
        lens, _, _ = _layout(c)
        entries = int(((lens + c["ps"] - 1) // c["ps"]).sum())
        return {"bytes": 4.0 * e * rows * c["Hkv"] * c["D"] + 8.0 * entries + 8.0 * pages + 8.0 * lens.numel(), "flops": 0.0}
    n, m = _rows(c), _states(c)
    pairs = sum(map(sum, _seen(c))) if c["seen"] else sum(x * y for x, y in zip(n, m))
    read = sum(max(x) for x in _seen(c)) if c["seen"] else sum(m)
    return {"bytes": 2.0 * e * c["L"] * c["D"] * (c["Hkv"] * read + c["H"] * sum(n)) + (4.0 * sum(n) if c["seen"] else 0.0),
            "flops": 4.0 * c["D"] * c["H"] * c["L"] * pairs}


# ---- inputs ------------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _offsets(n):
    off = [0]
    for x in n:
        off.append(off[-1] + x)
    return _i32(off)


def prepare(c, seed):
    k, g = c["kind"], _gen(seed, 1)
    st = dict(case=c)
    if k == "select":
        S, W, V = c["S"], c["W"], c["V"]
        logits = torch.empty((S, W, V), dtype=torch.float32, device=DEV).normal_(generator=g).mul_(2.5)
        logits += torch.randn((S, 1, V), generator=g, device=DEV) * 1.5              # beams of a prompt agree in part
        logits[torch.rand((S, W, V), generator=g, device=DEV) < 0.01] = -math.inf     # tokens that the program forbids
        scores = torch.rand((S, W), generator=g, device=DEV) * -4.0 - 10.0
        ended = torch.rand((S, W), generator=g, device=DEV) < 0.15
        ended[:, 0] = False
        st.update(logits=logits.to(DTYPES[c["dtype"]]), scores=scores, ended=ended, end=min(2, V - 1),
                  tokens=torch.empty((S, W), dtype=torch.int32, device=DEV), parents=torch.empty((S, W), dtype=torch.int32, device=DEV),
                  scores_out=torch.empty_like(scores), ended_out=torch.empty_like(ended))
        if own:
            import paper_2412_03409_amd as pkv
            st["ws"] = torch.empty(pkv.beam_workspace_bytes(S, W, V, DTYPES[c["dtype"]]), dtype=torch.uint8, device=DEV)
        return st
    dt, D, L = DTYPES[c["dtype"]], c["D"], c["L"]
    if k == "reorder":
        S, W, ps, Hkv = c["S"], c["W"], c["ps"], c["Hkv"]
        lens, shared, paired = (x.to(DEV) for x in _layout(c))
        width = _pages(c["ctx"] + c["new"], ps) + 1
        held = ((lens + ps - 1) // ps).view(S, W, L, 1)
        j, w = torch.arange(width, device=DEV), torch.arange(W, device=DEV).view(1, W, 1, 1)
        owner = torch.where(j < shared.view(S, 1, L, 1), 0, torch.where(j < paired.view(S, 1, L, 1), w - w % 2, w))
        group = torch.arange(S, device=DEV).view(S, 1, 1, 1) * W
        key = ((group + owner) * L + torch.arange(L, device=DEV).view(1, 1, L, 1)) * width + j       # one for each page there is
        used = torch.zeros(S * W * L * width, dtype=torch.bool, device=DEV)
        used[key[j < held]] = True
        number = torch.cumsum(used, 0) - 1
        count = int(number[-1]) + 1
        spare = _copied(c)[1] + 8
        perm = torch.randperm(count + spare, generator=g, device=DEV).to(torch.int32)
        table = torch.where(j < held, perm[number[key].clamp(min=0)], -1).to(torch.int32).view(S * W, L, width).contiguous()
        total = count + spare
        ring = torch.full((total,), -1, dtype=torch.int32, device=DEV)
        head = total // 3
        ring[(head + torch.arange(spare, device=DEV)) % total] = perm[count:]
        st.update(table=table, lens=lens.to(torch.int32).contiguous(), ring=ring, state=_i32([head, spare]), ps=ps,
                  parents=_i32(_parents(c)), kp=torch.empty((total, Hkv, ps, D), dtype=dt, device=DEV).normal_(generator=g),
                  vp=torch.empty((total, Hkv, ps, D), dtype=dt, device=DEV).normal_(generator=g),
                  # the updated table, lengths, ring's ends and the verdict, in buffers that the program keeps
                  table_out=torch.full_like(table, -1), lens_out=torch.empty((S * W, L), dtype=torch.int32, device=DEV),
                  state_out=torch.empty(2, dtype=torch.int32, device=DEV), status=torch.empty(1, dtype=torch.int32, device=DEV))
        if own:
            import paper_2412_03409_amd as pkv
            st["cache"] = pkv.PagedCache(kp=st["kp"], vp=st["vp"], table=table, lens=st["lens"], ring=ring, state=st["state"])
            st["ws"] = torch.empty(pkv.reorder_workspace_bytes(S * W, L), dtype=torch.uint8, device=DEV)
        return st
    H, Hkv, n, m = c["H"], c["Hkv"], _rows(c), _states(c)
    T, M = sum(n), sum(m)
    # queries token by token as a projection leaves them, keys and values of the states as a joint projection does
    q = torch.empty((L, T, H, D), dtype=dt, device=DEV).normal_(generator=g).permute(0, 2, 1, 3)
    kv = torch.empty((L, M, 2 * Hkv, D), dtype=dt, device=DEV).normal_(generator=g)
    kv[:, ::100, :Hkv] *= 4                                  # states that draw attention
    kk, v = kv[:, :, :Hkv].permute(0, 2, 1, 3), kv[:, :, Hkv:].permute(0, 2, 1, 3)
    scale = ((torch.rand(L, generator=g, device=DEV) * 2.5 + 0.5) / math.sqrt(D)).float()
    st.update(q=q, k=kk, v=v, row_off=_offsets(n), state_off=_offsets(m), scale=scale, most=max(n), longest=max(m),
              seen=_i32([x for row in _seen(c) for x in row]) if c["seen"] else None,
              out=torch.empty((L, T, H, D), dtype=dt, device=DEV).permute(0, 2, 1, 3))
    if own:
        import paper_2412_03409_amd as pkv
        st["ws"] = torch.empty(pkv.cross_workspace_bytes(c["S"], L, H, Hkv, T, M, D, dt, st["most"]), dtype=torch.uint8, device=DEV)
    return st


# ---- one pass ----------------------------------------------------------------------------------------
def run(st):
    return (_OWN if own else _PLAIN)[st["case"]["kind"]](st)


def _own_select(st):
    import paper_2412_03409_amd as pkv
    return pkv.prefixkv_beam_select(st["logits"], st["scores"], ended=st["ended"], end_token=st["end"], tokens=st["tokens"],
                                    parents=st["parents"], scores_out=st["scores_out"], ended_out=st["ended_out"], ws=st["ws"])


def _own_reorder(st):
    import paper_2412_03409_amd as pkv
    pkv.prefixkv_page_reorder(st["cache"], st["parents"], status=st["status"], table_out=st["table_out"], lens_out=st["lens_out"],
                              state_out=st["state_out"], ws=st["ws"])
    return st["table_out"], st["lens_out"], st["ring"], st["state_out"], st["status"], st["kp"], st["vp"]


def _own_cross(st):
    import paper_2412_03409_amd as pkv
    return pkv.prefixkv_cross_attn(st["q"], st["k"], st["v"], st["row_off"], st["state_off"], st["scale"], st["most"],
                                   seen=st["seen"], out=st["out"], ws=st["ws"])


def _plain_select(st):
    x, scores, ended, end = st["logits"].double(), st["scores"].double(), st["ended"], st["end"]
    S, W, V = x.shape
    m = x.amax(-1, keepdim=True)
    z = (x - m).exp_().sum(-1, keepdim=True).log_() + m
    x -= z
    x += scores[..., None]
    stays = torch.full_like(x[:, :, 0], -math.inf)
    x.masked_fill_(ended[..., None], -math.inf)
    x[:, :, end] = torch.where(ended, scores, x[:, :, end])
    flat = x.view(S, W * V)
    tokens, parents, best = [], [], []
    # the best beam of each round by its best token: a row's best is looked for again only in the beam that gave one
    top = x.amax(-1)                                                                  # [S, W]
    at = torch.arange(V, device=x.device)
    beams = torch.arange(W, device=x.device)
    for _ in range(W):
        value = top.amax(-1, keepdim=True)
        beam = torch.where(top == value, beams, W).amin(-1)                           # the lowest of equal ones
        row = torch.gather(x, 1, beam.view(S, 1, 1).expand(S, 1, V))[:, 0]
        token = torch.where(row == value, at, V).amin(-1)
        none = torch.isinf(value[:, 0])
        tokens.append(torch.where(none, -1, token))
        parents.append(torch.where(none, -1, beam))
        best.append(value[:, 0])
        flat.scatter_(1, (beam * V + token.clamp(max=V - 1))[:, None], stays[:, :1])
        row.scatter_(1, token.clamp(max=V - 1)[:, None], stays[:, :1])
        top.scatter_(1, beam[:, None], row.amax(-1, keepdim=True))
    tokens, parents, best = (torch.stack(t, 1) for t in (tokens, parents, best))
    over = (tokens == end) | (torch.gather(ended, 1, parents.clamp(min=0)) & (parents >= 0))
    return tokens.int(), parents.int(), best.float(), over


def _plain_reorder(st):
    table, lens, ring, state, ps, parents = st["table"], st["lens"], st["ring"], st["state"], st["ps"], st["parents"]
    G, W = parents.shape
    (R, L, width), P = table.shape, ring.shape[0]
    head, count = state[0], state[1]
    old, n, at = table.view(G, W, L, width), lens.view(G, W, L), torch.arange(width, device=table.device)
    real, p = parents >= 0, parents.clamp(min=0).long()
    valid = ((parents >= -1) & (parents < W)).all() & ((lens >= 0) & (lens <= width * ps)).all()
    new_n = torch.gather(n, 1, p[..., None].expand(G, W, L)) * real[..., None]
    new = torch.gather(old, 1, p[..., None, None].expand(G, W, L, width))
    in_new = at < ((new_n + ps - 1) // ps)[..., None]
    in_old = at < ((n + ps - 1) // ps)[..., None]
    # the lowest place of those that continue one keeps its partly filled page
    again = ((parents[:, :, None] == parents[:, None, :]) & torch.ones(W, W, dtype=torch.bool, device=p.device).tril(-1)).any(-1) & real
    part = new_n % ps
    copies = again[..., None] & (part > 0)                                            # [G, W, L]
    take = copies.flatten().int()
    first = (take.cumsum(0) - take).view(G, W, L)
    fresh = ring[(head + first) % P]
    last = copies[..., None] & (at == (new_n // ps)[..., None])
    result = torch.where(last, fresh[..., None], new)
    # pages of places that no place of the group holds any more, named by the lowest place that had them
    held = torch.where(in_new & ~last, new, -1)
    kept = torch.zeros_like(in_old)
    lower = torch.zeros_like(in_old)
    for w in range(W):
        kept |= held[:, w:w + 1] == old
        if w + 1 < W:
            lower[:, w + 1:] |= (old[:, w + 1:] == old[:, w:w + 1]) & in_old[:, w:w + 1]
    free = (in_old & ~kept & ~lower).flatten()
    ok = valid & (take.sum() <= count)
    to = torch.where(free & ok, (head + count + free.cumsum(0) - 1) % P, P)
    pushed = torch.cat([ring, ring[:1]])
    pushed.scatter_(0, to, table.flatten())
    status = torch.where(valid, (take.sum() > count).int(), 2).int().view(1)
    table_out = torch.where(torch.where(ok, in_new, in_old), torch.where(ok, result, old), st["table_out"].view(G, W, L, width))
    state_out = torch.stack([torch.where(ok, (head + take.sum()) % P, head), torch.where(ok, count - take.sum() + free.sum(), count)])
    # rows of the copied pages
    source = torch.gather(new, 3, (new_n // ps).clamp(max=width - 1).long()[..., None])[..., 0]
    pick = (copies & ok).flatten().nonzero()[:, 0]
    src, dst, rows = source.flatten()[pick].long(), fresh.flatten()[pick].long(), part.flatten()[pick]
    used = (torch.arange(ps, device=p.device) < rows[:, None])[:, None, :, None]
    pools = []
    for pool in (st["kp"], st["vp"]):
        y = pool.clone()
        y[dst] = torch.where(used, pool[src], pool[dst])
        pools.append(y)
    return (table_out.view(R, L, width), torch.where(ok, new_n, n).view(R, L).int(), pushed[:P], state_out.int(), status, *pools)


def _padded_rows(x, off, most):
    """[L,heads,T,D] packed -> [S,L,heads,most,D] in 32 bits, and which rows are real."""
    at = off[:-1, None] + torch.arange(most, device=off.device)
    real = at < off[1:, None]
    rows = x[:, :, at.clamp(max=x.shape[2] - 1).long()]                              # [L,heads,S,most,D]
    return rows.permute(2, 0, 1, 3, 4).float(), real


def _plain_cross(st):
    q, off, dt = st["q"], st["row_off"], st["q"].dtype
    L, H, T, D = q.shape
    Hkv, S, most, longest = st["k"].shape[1], off.shape[0] - 1, st["most"], st["longest"]
    G = H // Hkv
    qf, _ = _padded_rows(q, off, most)
    kf, see = _padded_rows(st["k"], st["state_off"], longest)
    vf, _ = _padded_rows(st["v"], st["state_off"], longest)
    qf = (qf * st["scale"][None, :, None, None, None]).reshape(S * L * Hkv, G * most, D)
    s = torch.bmm(qf, kf.reshape(S * L * Hkv, longest, D).transpose(1, 2).contiguous()).view(S, L, H, most, longest)
    see = see[:, None, None, None, :]
    if st["seen"] is not None:
        at = (off[:-1, None] + torch.arange(most, device=q.device)).clamp(max=T - 1).long()
        see = see & (torch.arange(longest, device=q.device) < st["seen"][at][..., None])[:, None, None]
    s = torch.where(see, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    z = e.sum(-1, keepdim=True)
    e /= torch.where(z > 0, z, torch.ones_like(z))
    o = torch.bmm(e.view(S * L * Hkv, G * most, longest), vf.reshape(S * L * Hkv, longest, D).contiguous()).view(S, L, H, most, D)
    t = torch.arange(T, device=off.device, dtype=torch.int32)
    sq = torch.searchsorted(off, t, right=True) - 1
    return o[sq, :, :, (t - off[sq]).long()].permute(1, 2, 0, 3).to(dt)


_PLAIN = dict(select=_plain_select, reorder=_plain_reorder, cross=_plain_cross)
_OWN = dict(select=_own_select, reorder=_own_reorder, cross=_own_cross)


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def exact(c, seed):
    """The scores of the chosen continuations, prompt by prompt; attention memory by memory and head by head.  A reordering
    makes whole numbers and copies."""
    k = c["kind"]
    if k == "reorder":
        return None
    st = prepare(c, seed)
    if k == "select":
        S, W, V = st["logits"].shape
        best = torch.full((S, W), -math.inf, dtype=torch.float64, device=DEV)
        for s in range(S):
            found = []
            for w in range(W):
                score = st["scores"][s, w].double()
                if bool(st["ended"][s, w]):
                    found.append(score.view(1))
                    continue
                logp = torch.log_softmax(st["logits"][s, w].double(), dim=0)
                found.append(score + torch.sort(logp, descending=True).values[:W])
            every = torch.sort(torch.cat(found), descending=True).values[:W]
            best[s, :every.numel()] = every
        return None, None, best, None
    q, off, to = st["q"], st["row_off"].tolist(), st["state_off"].tolist()
    L, H, T, D = q.shape
    out = torch.zeros((L, H, T, D), dtype=torch.float64, device=DEV)
    for s in range(c["S"]):
        a, b = off[s], off[s + 1]
        for l in range(L):
            keys, values = st["k"][l, :, to[s]:to[s + 1]].double(), st["v"][l, :, to[s]:to[s + 1]].double()
            hidden = None
            if st["seen"] is not None:
                hidden = torch.arange(keys.shape[1], device=DEV)[None, :] >= st["seen"][a:b, None]
            for h in range(H):
                g = h // (H // c["Hkv"])
                score = (q[l, h, a:b].double() @ keys[g].t()) * st["scale"][l].double()
                if hidden is not None:
                    score.masked_fill_(hidden, -math.inf)
                p = torch.softmax(score, dim=1)
                out[l, h, a:b] = torch.where(torch.isnan(p), 0.0, p) @ values[g]
    return out

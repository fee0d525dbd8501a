"""Timed cases of the operators that serve packed prompts and paged, compressed caches.

A serving program holds requests of different lengths: their prompts are packed one behind the other, their
queries and keys are rotated by positions on several axes (time, height, width of an image or video, one axis
for text), the prompt attends to itself, the search decides what each layer keeps, and what is kept lives in
pages that belong to one (sequence, layer) each, because every layer keeps another number of positions.  New
tokens -- a chunk of a second question, or one per sequence -- get slots in those pages, are rotated and stored,
and attend to what is there.  A case is one of these steps.

`kind` of a case:
  append   prefixkv_page_append: pages and slots for the new tokens of all sequences, every layer
  resize   prefixkv_page_resize: sequences that end, shrink to what the search keeps, or start
  rope     prefixkv_rope, or with `store` prefixkv_rope_store: K and V go into the pages
  compact  prefixkv_compact_paged: the kept rows of a rectangular batch go into the pages
  prompt   prefixkv_prefill_attn_packed
  chunk    prefixkv_chunk_attn

Where `own` is false the steps are computed in elementary torch operations, in 32 bits (angles in 64).
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
        # One token for each of 64 sequences, 32 layers: before every decode step; pure latency.
        dict(name="append_decode", kind="append", S=64, L=32, ps=16, ctx=1700, new=1, lens=1),
        # A scheduler's step: some sequences end, some shrink to their configuration, some start.
        dict(name="resize_mixed", kind="resize", S=64, L=40, ps=16, ctx=8192, lens=3),
        # One layer, one new token for each of 48 sequences, rotated and stored: latency.
        dict(name="rope_store_decode", kind="rope", store=True, dtype="bf16", L=1, H=32, Hkv=8, T=48, D=128, rot=128,
             inter=False, axes=3, far=8192, ps=16, lens=4),
        # One layer of eight packed 7B prompts: bandwidth.
        dict(name="rope_prompts", kind="rope", store=False, dtype="bf16", L=1, H=32, Hkv=32, T=5440, D=128, rot=128,
             inter=False, axes=3, far=700, ps=16, lens=5),
        # The validation shape's storage type, all layers of a chunk at once, positions far out in a video.
        dict(name="rope_store_f32", kind="rope", store=True, dtype="f32", L=4, H=4, Hkv=2, T=1021, D=64, rot=32,
             inter=True, axes=2, far=1000000, ps=32, lens=6),
        # The kept 20 % of all layers of one 7B prompt.
        dict(name="compact_7b", kind="compact", dtype="bf16", B=1, L=32, Hkv=32, N=680, D=128, budget=0.2, ps=16, lens=7),
        # The kept 10 % of a long grouped-query prompt of two sequences, large pages.
        dict(name="compact_gqa_long", kind="compact", dtype="bf16", B=2, L=32, Hkv=8, N=8192, D=128, budget=0.1, ps=64,
             lens=8),
        # One 7B layer over a handful of packed prompts, one of them a single token.
        dict(name="prompt_7b_packed", kind="prompt", dtype="bf16", S=6, L=1, H=32, Hkv=32, longest=1021, shortest=1, D=128,
             lens=9),
        # One layer of two long grouped-query prompts: the largest product.
        dict(name="prompt_gqa_long", kind="prompt", dtype="bf16", S=2, L=1, H=32, Hkv=8, longest=6001, shortest=4000, D=128,
             lens=10),
        # Single tokens of 32 sequences over long grouped-query caches: bandwidth.
        dict(name="chunk_decode", kind="chunk", dtype="bf16", S=32, L=1, H=32, Hkv=8, ctx=8192, new=1, D=128, ps=16, lens=11),
        # A second question of up to 600 tokens over the compressed caches of eight sequences.
        dict(name="chunk_question", kind="chunk", dtype="bf16", S=8, L=1, H=32, Hkv=8, ctx=6000, new=600, D=128, ps=64,
             lens=12),
        # The validation shape: a few fp32 tokens over short caches, all layers in a call.
        dict(name="chunk_tiny_f32", kind="chunk", dtype="f32", S=2, L=4, H=2, Hkv=2, ctx=128, new=8, D=64, ps=16, lens=2),
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
    limit["append"] = limit["resize"]     # one operator
    kind = rng.choice(["append", "resize", "rope", "rope", "compact", "prompt", "prompt", "chunk", "chunk", "chunk"])
    while True:
        H, Hkv = rng.choice([(32, 32), (40, 40), (32, 8), (32, 4), (16, 8), (24, 24), (12, 4), (28, 4)])
        D, ps, seed = rng.choice([128, 128, 64]), rng.choice([16, 16, 32, 64, 128]), rng.randrange(1 << 20)
        if kind == "append":
            c = dict(kind=kind, S=_log_int(rng, 1, 96), L=rng.choice([1, 24, 32, 40]), ps=ps, ctx=_log_int(rng, 20, 8192),
                     new=_log_int(rng, 1, 900), lens=seed)
        elif kind == "resize":
            c = dict(kind=kind, S=_log_int(rng, 1, 96), L=rng.choice([1, 24, 32, 40]), ps=ps, ctx=_log_int(rng, 20, 8192),
                     lens=seed)
        elif kind == "rope":
            f32 = rng.random() < 0.25
            if f32:
                H, Hkv = rng.choice([(2, 2), (4, 2), (4, 1)])
            c = dict(kind=kind, store=rng.random() < 0.5, dtype="f32" if f32 else "bf16", L=rng.choice([1, 1, 4]), H=H, Hkv=Hkv,
                     T=_log_int(rng, 1, 6000), D=D, rot=rng.choice([D, D, D // 2, 48]), inter=rng.random() < 0.4,
                     axes=rng.choice([1, 2, 3]), far=rng.choice([700, 8192, 100000, 1000000]), ps=ps, lens=seed)
        elif kind == "compact":
            f32 = rng.random() < 0.15
            c = dict(kind=kind, dtype="f32" if f32 else "bf16", B=_log_int(rng, 1, 8), L=rng.choice([4, 24, 32, 40]),
                     Hkv=rng.choice([1, 2]) if f32 else Hkv, N=_log_int(rng, 48, 8192), D=D,
                     budget=round(rng.uniform(0.05, 0.6), 3), ps=ps, lens=seed)
        elif kind == "prompt":
            longest = _log_int(rng, 2, 6000)
            c = dict(kind=kind, dtype="bf16", S=_log_int(rng, 1, 24), L=1, H=H, Hkv=Hkv, longest=longest,
                     shortest=max(1, int(longest * rng.choice([0.02, 0.3, 0.9]))), D=D, lens=seed)
        else:
            f32 = rng.random() < 0.15
            if f32:
                H, Hkv = rng.choice([(2, 2), (4, 2), (4, 1)])
            c = dict(kind=kind, dtype="f32" if f32 else "bf16", S=_log_int(rng, 1, 64), L=rng.choice([1, 1, 1, 4]), H=H, Hkv=Hkv,
                     ctx=_log_int(rng, 16, 400 if f32 else 8192), new=rng.choice([1, 1, 2, 5, _log_int(rng, 8, 64 if f32 else 700)]),
                     D=D, ps=ps, lens=seed)
        # a plain form of attention holds the padded scores several times over
        if _cost(c) <= limit[kind] and _padded(c) <= 3e9:
            return c


def _padded(c):
    if c["kind"] == "prompt":
        return c["S"] * c["H"] * c["longest"] ** 2
    if c["kind"] == "chunk":
        return c["S"] * c["L"] * max(c["H"] * c["new"], c["Hkv"] * c["D"]) * (c["ctx"] + c["new"])
    return 0


# ---- sizes of a case: lengths are the case's own, values are the seed's ---------------------------------
def _spread(rng, n, lo, hi):
    """n whole numbers from lo to hi, evenly over the logarithm, the first of them hi."""
    got = [hi] + [int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)))))) for _ in range(n - 1)]
    return [min(max(x, lo), hi) for x in got]


def _rows(c):
    """New tokens of every sequence."""
    r = random.Random(c["lens"])
    if c["kind"] == "prompt":
        return _spread(r, c["S"], c["shortest"], c["longest"])
    return _spread(r, c["S"], 1, c["new"])


def _cached(c):
    """Entries cached before the call, per (sequence, layer): layers differ, as the search leaves them."""
    r = random.Random(c["lens"] + 1)
    ctx = c["ctx"]
    got = [[max(0, min(ctx, int(ctx * math.exp(-r.uniform(0.0, 2.5))))) for _ in range(c["L"])] for _ in range(c["S"])]
    got[0][0] = ctx
    if c["S"] > 2 and c["kind"] != "chunk":
        got[1] = [0] * c["L"]
    return got


def _targets(c):
    """What a scheduler's step leaves of every segment: a third of the sequences end, a third shrink, the others grow."""
    r = random.Random(c["lens"] + 2)
    got = []
    for s, row in enumerate(_cached(c)):
        what = r.randrange(3)
        got.append([0 if what == 0 else int(x * r.uniform(0.1, 0.9)) if what == 1 else min(c["ctx"], x + r.randrange(1, 300))
                    for x in row])
    return got


def _pages(n, ps):
    return -(-n // ps)


def _keeps(c):
    """Lengths of a compaction: their sum meets the budget roughly, layers differ."""
    r = random.Random(c["lens"] + 3)
    N, L = c["N"], c["L"]
    got = []
    for _ in range(c["B"]):
        w = [math.exp(r.uniform(-1.5, 1.5)) for _ in range(L)]
        f = c["budget"] * L / sum(w)
        got.append([max(1, min(N, int(N * f * x))) for x in w])
    return got


def _numbers(c):
    """Entries that the call leaves in every segment of a chunk's cache (new tokens among them)."""
    return [[x + n for x in row] for row, n in zip(_cached(c), _rows(c))]


def work(c):
    k = c["kind"]
    e = 4 if c.get("dtype") == "f32" else 2
    if k == "append":
        n, old = _rows(c), _cached(c)
        got = sum(_pages(x + m, c["ps"]) - _pages(x, c["ps"]) for row, m in zip(old, n) for x in row)
        return {"bytes": 8.0 * c["S"] * c["L"] + 8.0 * got + 8.0 * c["L"] * sum(n) + 4.0 * c["S"], "flops": 0.0}
    if k == "resize":
        moved = sum(abs(_pages(x, c["ps"]) - _pages(y, c["ps"])) for a, b in zip(_cached(c), _targets(c)) for x, y in zip(a, b))
        return {"bytes": 12.0 * c["S"] * c["L"] + 8.0 * moved, "flops": 0.0}
    if k == "rope":
        rows = c["L"] * c["T"]
        b = 2.0 * e * rows * (c["H"] + c["Hkv"]) * c["D"] + 4.0 * c["axes"] * c["T"]
        b += (2.0 * e * rows * c["Hkv"] * c["D"] + 8.0 * rows) if c["store"] else 0.0
        return {"bytes": b, "flops": 3.0 * rows * (c["H"] + c["Hkv"]) * c["rot"]}
    if k == "compact":
        kept = sum(map(sum, _keeps(c)))
        return {"bytes": 4.0 * e * kept * c["Hkv"] * c["D"] + 8.0 * kept, "flops": 0.0}
    if k == "prompt":
        n = _rows(c)
        return {"bytes": sum(n) * c["L"] * (2.0 * e * (c["H"] + c["Hkv"]) * c["D"] + 4.0 * c["H"]),
                "flops": 4.0 * c["D"] * c["H"] * c["L"] * sum(x * (x + 1) / 2 for x in n)}
    n, tot = _rows(c), _numbers(c)
    seen = sum(m * x - m * (m - 1) / 2 for row, m in zip(tot, n) for x in row)
    return {"bytes": 2.0 * e * c["Hkv"] * c["D"] * sum(map(sum, tot)) + 2.0 * e * c["H"] * c["D"] * sum(n) * c["L"],
            "flops": 4.0 * c["D"] * c["H"] * seen}


# ---- inputs ------------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _row_off(n):
    off = [0]
    for x in n:
        off.append(off[-1] + x)
    return _i32(off)


def _projected(c, L, T, g):
    """Queries, keys and values as a fused projection leaves them: token by token, heads side by side."""
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    x = torch.empty((L, T, H + 2 * Hkv, D), dtype=DTYPES[c["dtype"]], device=DEV).normal_(generator=g)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    return tuple(t.permute(0, 2, 1, 3) for t in (q, k, v))


def _paging(lens, L, ps, width, spare, g):
    """A pool's page tables for segments of these lengths: pages in no order, the others in the ring."""
    lens = torch.tensor(lens, dtype=torch.int64)
    held = (lens + ps - 1) // ps
    used = int(held.sum())
    total = used + spare
    perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    at = torch.arange(width)
    mask = (at < held[..., None]).to(DEV)
    first = (torch.cumsum(held.flatten(), 0) - held.flatten()).view(held.shape).to(DEV)
    index = (first[..., None] + at.to(DEV)).clamp(max=total - 1)
    table = torch.where(mask, perm[index], torch.full_like(perm[index], -1)).contiguous()
    ring = torch.full((total,), -1, dtype=torch.int32, device=DEV)
    head = total // 3
    ring[(head + torch.arange(spare, device=DEV)) % total] = perm[used:]
    return dict(lens=lens.to(torch.int32).to(DEV), table=table, ring=ring, state=_i32([head, spare]), pages=total, ps=ps)


def _cache(st, Hkv=1, D=64, dtype=torch.bfloat16, pools=None):
    import paper_2412_03409_amd as pkv
    if pools is None:   # the page operators look at the tables alone
        pools = [torch.empty((1, Hkv, st["ps"], D), dtype=dtype, device=DEV).expand(st["pages"], -1, -1, -1)] * 2
    return pkv.PagedCache(kp=pools[0], vp=pools[1], table=st["table"], lens=st["lens"], ring=st["ring"], state=st["state"])


def prepare(c, seed):
    k, g = c["kind"], _gen(seed, 1)
    st = dict(case=c)
    if k in ("append", "resize"):
        old = _cached(c)
        if k == "append":
            n = _rows(c)
            need = sum(_pages(x + m, c["ps"]) - _pages(x, c["ps"]) for row, m in zip(old, n) for x in row)
            st.update(row_off=_row_off(n), T=sum(n), slots=torch.empty((c["L"], sum(n)), dtype=torch.int64, device=DEV))
            width = _pages(c["ctx"] + c["new"], c["ps"])
        else:
            to = _targets(c)
            need = sum(max(0, _pages(y, c["ps"]) - _pages(x, c["ps"])) for a, b in zip(old, to) for x, y in zip(a, b))
            st.update(target=_i32(to))
            width = _pages(c["ctx"], c["ps"])
        st.update(_paging(old, c["L"], c["ps"], width, need + 64, g))
        # the updated lengths, the ring's ends and the verdict, in buffers that the program keeps
        st.update(lens_out=torch.empty_like(st["lens"]), state_out=torch.empty_like(st["state"]),
                  status=torch.empty(1, dtype=torch.int32, device=DEV))
        if own:
            import paper_2412_03409_amd as pkv
            st.update(cache=_cache(st), ws=torch.empty(pkv.page_workspace_bytes(c["S"], c["L"]), dtype=torch.uint8, device=DEV))
        return st
    dt, D = DTYPES[c["dtype"]], c["D"]
    if k == "rope":
        L, T = c["L"], c["T"]
        q, kk, v = _projected(c, L, T, g)
        pos = torch.randint(0, c["far"] + 1, (c["axes"], T), generator=g, device=DEV, dtype=torch.int32)
        third = c["rot"] // 2 // c["axes"]
        sections = [c["rot"] // 2 - third * (c["axes"] - 1)] + [third] * (c["axes"] - 1)
        st.update(q=q, k=kk, v=v, pos=pos, sections=sections, theta=10000.0,
                  q_out=torch.empty((L, T, c["H"], D), dtype=dt, device=DEV).permute(0, 2, 1, 3))
        if c["store"]:
            pages = _pages(L * T, c["ps"]) + 3
            st["slots"] = torch.randperm(pages * c["ps"], generator=g, device=DEV)[:L * T].view(L, T).contiguous()
            st["slots"][:, T - T // 50:] = -1     # rows that pad the batch
            st.update(kp=torch.zeros((pages, c["Hkv"], c["ps"], D), dtype=dt, device=DEV), ps=c["ps"])
            st["vp"] = torch.zeros_like(st["kp"])
        else:
            st["k_out"] = torch.empty((L, T, c["Hkv"], D), dtype=dt, device=DEV).permute(0, 2, 1, 3)
        if own:
            import paper_2412_03409_amd as pkv
            st["plan"] = pkv.rope_plan(c["rot"], sections, theta=st["theta"], interleaved=c["inter"], device=DEV)
            if c["store"]:
                t = torch.zeros((1, L, 1), dtype=torch.int32, device=DEV)      # a store goes by the slots alone
                st["cache"] = pkv.PagedCache(kp=st["kp"], vp=st["vp"], table=t, lens=t[:, :, 0].contiguous(),
                                             ring=torch.zeros(pages, dtype=torch.int32, device=DEV), state=_i32([0, 0]))
        return st
    if k == "compact":
        B, L, Hkv, N = c["B"], c["L"], c["Hkv"], c["N"]
        x = torch.empty((2, B, L, Hkv, N, D), dtype=dt, device=DEV).normal_(generator=g)
        order = torch.argsort(torch.rand((B, L, N), generator=g, device=DEV), dim=-1).to(torch.int32)
        keeps = _keeps(c)
        st.update(k=x[0], v=x[1], order=order, lengths=_i32(keeps), most=max(map(max, keeps)))
        st.update(_paging(keeps, L, c["ps"], _pages(N, c["ps"]), 8, g))
        st.update(kp=torch.zeros((st["pages"], Hkv, c["ps"], D), dtype=dt, device=DEV),
                  kept_pos=torch.full((B, L, N), -1, dtype=torch.int32, device=DEV))
        st["vp"] = torch.zeros_like(st["kp"])
        if own:
            st["cache"] = _cache(st, pools=(st["kp"], st["vp"]))
        return st
    n = _rows(c)
    T, L = sum(n), c["L"]
    q, kk, v = _projected(c, L, T, g)
    scale = ((torch.rand(L, generator=g, device=DEV) * 2.5 + 0.5) / math.sqrt(D)).float()
    st.update(q=q, row_off=_row_off(n), scale=scale,
              out=torch.empty((L, T, c["H"], D), dtype=dt, device=DEV).permute(0, 2, 1, 3))
    if k == "prompt":
        kk[:, :, ::100] *= 4      # sink keys
        st.update(k=kk, v=v, longest=c["longest"], lse=torch.empty(L * c["H"] * T, dtype=torch.float32, device=DEV))
        if own:
            import paper_2412_03409_amd as pkv
            st["ws"] = torch.empty(pkv.attn_workspace_bytes(c["S"], L, c["H"], c["Hkv"], T, D, dt), dtype=torch.uint8, device=DEV)
        return st
    tot = _numbers(c)
    st.update(_paging(tot, L, c["ps"], _pages(c["ctx"] + c["new"], c["ps"]), 2, g))
    st.update(kp=torch.empty((st["pages"], c["Hkv"], c["ps"], D), dtype=dt, device=DEV).normal_(generator=g),
              vp=torch.empty((st["pages"], c["Hkv"], c["ps"], D), dtype=dt, device=DEV).normal_(generator=g), most=max(n))
    if own:
        import paper_2412_03409_amd as pkv
        st["cache"] = _cache(st, pools=(st["kp"], st["vp"]))
        st["ws"] = torch.empty(pkv.attn_workspace_bytes(c["S"], L, c["H"], c["Hkv"], T, D, dt, max_rows=st["most"]),
                               dtype=torch.uint8, device=DEV)
    return st


# ---- one pass ----------------------------------------------------------------------------------------
def run(st):
    return (_OWN if own else _PLAIN)[st["case"]["kind"]](st)


def _own_append(st):
    import paper_2412_03409_amd as pkv
    pkv.prefixkv_page_append(st["cache"], st["row_off"], st["T"], slots=st["slots"], status=st["status"],
                             lens_out=st["lens_out"], state_out=st["state_out"], ws=st["ws"])
    return st["table"], st["slots"], st["lens_out"], st["state_out"], st["status"]


def _own_resize(st):
    import paper_2412_03409_amd as pkv
    pkv.prefixkv_page_resize(st["cache"], st["target"], status=st["status"], lens_out=st["lens_out"],
                             state_out=st["state_out"], ws=st["ws"])
    return st["table"], st["ring"], st["lens_out"], st["state_out"], st["status"]


def _own_rope(st):
    import paper_2412_03409_amd as pkv
    if st["case"]["store"]:
        pkv.prefixkv_rope_store(st["cache"], st["q"], st["k"], st["v"], st["pos"], st["plan"], st["slots"], q_out=st["q_out"])
        return st["q_out"], st["kp"], st["vp"]
    return pkv.prefixkv_rope(st["q"], st["k"], st["pos"], st["plan"], q_out=st["q_out"], k_out=st["k_out"])


def _own_compact(st):
    import paper_2412_03409_amd as pkv
    pkv.prefixkv_compact_paged(st["cache"], st["k"], st["v"], st["order"], st["lengths"], kept_pos=st["kept_pos"])
    return st["kp"], st["vp"], st["kept_pos"]


def _own_prompt(st):
    import paper_2412_03409_amd as pkv
    return pkv.prefixkv_prefill_attn_packed(st["q"], st["k"], st["v"], st["row_off"], st["scale"], out=st["out"],
                                            lse=st["lse"], ws=st["ws"])


def _own_chunk(st):
    import paper_2412_03409_amd as pkv
    return pkv.prefixkv_chunk_attn(st["cache"], st["q"], st["row_off"], st["scale"], st["most"], out=st["out"], ws=st["ws"])


def _resized(st, target):
    """Tables, lengths, ring and its ends after the segments get the lengths `target`: all or nothing."""
    ps, lens, table, ring, P = st["ps"], st["lens"], st["table"], st["ring"], st["pages"]
    head, count = st["state"][0], st["state"][1]
    width = table.shape[-1]
    held, want = (lens + (ps - 1)) // ps, (target + (ps - 1)) // ps
    more, less = (want - held).clamp(min=0), (held - want).clamp(min=0)
    first_more = (more.flatten().cumsum(0) - more.flatten()).view_as(more)
    first_less = (less.flatten().cumsum(0) - less.flatten()).view_as(less)
    short, wide = more.sum() > count, (want > width).any() | (target < 0).any()
    ok = ~(short | wide)
    at = torch.arange(width, device=table.device)
    grow = (at >= held[..., None]) & (at < want[..., None]) & ok
    from_ring = ring[(head + first_more[..., None] + (at - held[..., None])) % P]
    drop = (at >= want[..., None]) & (at < held[..., None]) & ok
    to = torch.where(drop, (head + count + first_less[..., None] + (at - want[..., None])) % P, P)
    pushed = torch.cat([ring, ring[:1]])
    pushed.scatter_(0, to.flatten().long(), table.flatten())
    new_state = torch.stack([torch.where(ok, (head + more.sum()) % P, head), torch.where(ok, count - more.sum() + less.sum(), count)])
    status = (short.int() + 2 * wide.int()).view(1)
    return torch.where(grow, from_ring, table), pushed[:P], torch.where(ok, target, lens), new_state.int(), status, ok


def _plain_append(st):
    off = st["row_off"]
    n = off[1:] - off[:-1]
    table, _, lens, state, status, ok = _resized(st, st["lens"] + n[:, None])
    t = torch.arange(st["T"], device=off.device, dtype=torch.int32)
    s = torch.searchsorted(off, t, right=True) - 1
    p = st["lens"][s] + (t - off[s])[:, None]                                        # [T, L]
    page = torch.gather(table[s], 2, (p // st["ps"]).long()[..., None])[..., 0].long()
    slots = torch.where(ok, page * st["ps"] + p % st["ps"], -1).t().contiguous()
    return table, slots, lens, state, status


def _plain_resize(st):
    table, ring, lens, state, status, _ = _resized(st, st["target"])
    return table, ring, lens, state, status


def _angles(st):
    half = st["case"]["rot"] // 2
    i = torch.arange(half, device=DEV, dtype=torch.float64)
    freq = torch.pow(torch.tensor(st["theta"], dtype=torch.float64, device=DEV), -i / half)
    axis = torch.repeat_interleave(torch.arange(len(st["sections"]), device=DEV), torch.tensor(st["sections"], device=DEV),
                                   output_size=half)
    a = st["pos"][axis].double() * freq[:, None]                                    # [rot/2, T]
    return torch.cos(a).float().t(), torch.sin(a).float().t()


def _rotated(x, cos, sin, rot, inter):
    y = x.float()
    head, rest = y[..., :rot], y[..., rot:]
    if inter:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1).to(x.dtype)


def _plain_rope(st):
    c = st["case"]
    cos, sin = _angles(st)
    q, k = _rotated(st["q"], cos, sin, c["rot"], c["inter"]), _rotated(st["k"], cos, sin, c["rot"], c["inter"])
    if not c["store"]:
        return q, k
    slots, ps, got = st["slots"].flatten(), st["ps"], []
    for pool, x in ((st["kp"], k), (st["vp"], st["v"])):
        P, Hkv, _, D = pool.shape
        rows = torch.cat([pool.permute(0, 2, 1, 3).reshape(P * ps, Hkv, D), pool.new_zeros((1, Hkv, D))])
        rows[torch.where(slots < 0, P * ps, slots)] = x.permute(0, 2, 1, 3).reshape(-1, Hkv, D)
        got.append(rows[:P * ps].view(P, ps, Hkv, D).permute(0, 2, 1, 3).contiguous())
    return q, got[0], got[1]


def _plain_compact(st):
    k, v, order, lengths, ps = st["k"], st["v"], st["order"], st["lengths"], st["ps"]
    B, L, Hkv, N, D = k.shape
    at, most, P = torch.arange(N, device=k.device), st["most"], st["kp"].shape[0]
    pos = torch.sort(torch.where(at < lengths[..., None], order, N), dim=-1).values  # ascending, N behind them
    near, j = pos[..., :most], at[:most]
    page = torch.gather(st["table"], 2, (j // ps).expand(B, L, most)).long()
    slot = torch.where(near < N, page * ps + j % ps, P * ps).flatten()
    take = near.clamp(max=N - 1).long()[:, :, None, :, None].expand(B, L, Hkv, most, D)
    got = []
    for pool, x in ((st["kp"], k), (st["vp"], v)):
        rows = torch.cat([pool.permute(0, 2, 1, 3).reshape(P * ps, Hkv, D), pool.new_zeros((1, Hkv, D))])
        rows[slot] = torch.gather(x, 3, take).permute(0, 1, 3, 2, 4).reshape(-1, Hkv, D)
        got.append(rows[:P * ps].view(P, ps, Hkv, D).permute(0, 2, 1, 3).contiguous())
    return got[0], got[1], torch.where(pos < N, pos, st["kept_pos"])


def _padded_rows(x, off, most):
    """[L,heads,T,D] packed -> [S,L,heads,most,D] in 32 bits, and which rows are real."""
    at = off[:-1, None] + torch.arange(most, device=off.device)
    real = at < off[1:, None]
    rows = x[:, :, at.clamp(max=x.shape[2] - 1).long()]                              # [L,heads,S,most,D]
    return rows.permute(2, 0, 1, 3, 4).float(), real


def _softmax(s, see):
    """Probabilities over the keys that are seen, and the logarithm of their sum; rows that see nothing get zeros."""
    s = torch.where(see, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    return e / torch.where(z > 0, z, torch.ones_like(z)), (torch.log(z) + m)[..., 0]


def _places(off, T):
    """Sequence of every packed row, and the row's place in it."""
    t = torch.arange(T, device=off.device, dtype=torch.int32)
    s = torch.searchsorted(off, t, right=True) - 1
    return s, (t - off[s]).long()


def _plain_prompt(st):
    q, off, dt = st["q"], st["row_off"], st["q"].dtype
    L, H, T, D = q.shape
    Hkv, S, most = st["k"].shape[1], off.shape[0] - 1, st["longest"]
    qf, _ = _padded_rows(q, off, most)
    kf, _ = _padded_rows(st["k"], off, most)
    vf, _ = _padded_rows(st["v"], off, most)
    qf = (qf * st["scale"][None, :, None, None, None]).reshape(S * L * Hkv, H // Hkv * most, D)
    kt = kf.reshape(S * L * Hkv, most, D).transpose(1, 2).contiguous()
    s = torch.bmm(qf, kt).view(S, L, H, most, most)
    i = torch.arange(most, device=q.device)
    n = off[1:] - off[:-1]
    see = (i[None, :] <= i[:, None]) & (i < n[:, None])[:, None, None, None, :]
    p, lse = _softmax(s, see)
    o = torch.bmm(p.view(S * L * Hkv, H // Hkv * most, most), vf.reshape(S * L * Hkv, most, D).contiguous())
    o = o.view(S, L, H, most, D)
    sq, at = _places(off, T)
    out = o[sq, :, :, at].permute(1, 2, 0, 3).to(dt)
    # the logarithms of a sequence lie together: [L][H][n] behind those of the sequences before it
    where = (off[sq] * (L * H)).long()[:, None] + torch.arange(L * H, device=off.device) * n[sq].long()[:, None] + at[:, None]
    packed = torch.empty(L * H * T, dtype=torch.float32, device=q.device)
    packed[where.flatten()] = lse[sq, :, :, at].reshape(-1)
    return out, packed


def _plain_chunk(st):
    q, off, ps, dt = st["q"], st["row_off"], st["ps"], st["q"].dtype
    L, H, T, D = q.shape
    Hkv, S, most = st["kp"].shape[1], off.shape[0] - 1, st["most"]
    G = H // Hkv
    qf, _ = _padded_rows(q, off, most)                                               # [S,L,H,most,D]
    qf = (qf * st["scale"][None, :, None, None, None]).reshape(S * L * Hkv, G * most, D)
    table = st["table"].clamp(min=0).long()
    width = table.shape[2] * ps
    k = st["kp"][table].float().permute(0, 1, 3, 5, 2, 4).reshape(S * L * Hkv, D, width)
    v = st["vp"][table].float().permute(0, 1, 3, 2, 4, 5).reshape(S * L * Hkv, width, D)
    s = torch.bmm(qf, k).view(S, L, H, most, width)
    n, key = off[1:] - off[:-1], torch.arange(width, device=q.device)
    last = st["lens"][:, :, None] - n[:, None, None] + torch.arange(most, device=q.device)      # [S,L,most]
    p, _ = _softmax(s, (key <= last[..., None])[:, :, None])
    o = torch.bmm(p.view(S * L * Hkv, G * most, width), v).view(S, L, H, most, D)
    sq, at = _places(off, T)
    return o[sq, :, :, at].permute(1, 2, 0, 3).to(dt)


_PLAIN = dict(append=_plain_append, resize=_plain_resize, rope=_plain_rope, compact=_plain_compact, prompt=_plain_prompt,
              chunk=_plain_chunk)
_OWN = dict(append=_own_append, resize=_own_resize, rope=_own_rope, compact=_own_compact, prompt=_own_prompt,
            chunk=_own_chunk)


# ---- the definitions in 64 bits ------------------------------------------------------------------------
def exact(c, seed):
    """Sequence by sequence and head by head from the formulas; the page operators make whole numbers."""
    k = c["kind"]
    if k in ("append", "resize"):
        return None
    st = prepare(c, seed)
    if k == "compact":
        return _exact_compact(c, st)
    if k == "rope":
        return _exact_rope(c, st)
    off = st["row_off"].tolist()
    q = st["q"]
    L, H, T, D = q.shape
    out = torch.zeros((L, H, T, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros(L * H * T, dtype=torch.float64, device=DEV)
    for s in range(len(off) - 1):
        a, b = off[s], off[s + 1]
        for l in range(L):
            if k == "prompt":
                keys, values = st["k"][l, :, a:b].double(), st["v"][l, :, a:b].double()
            else:
                size = int(st["lens"][s, l])
                ids = st["table"][s, l, :_pages(size, c["ps"])].long()
                keys, values = (x[ids].double().transpose(0, 1).reshape(c["Hkv"], -1, D)[:, :size] for x in (st["kp"], st["vp"]))
            size = keys.shape[1]
            limit = size - (b - a) + torch.arange(b - a, device=DEV)[:, None]
            hidden = torch.arange(size, device=DEV)[None, :] > limit
            for h in range(H):
                g = h // (H // c["Hkv"])
                score = (q[l, h, a:b].double() @ keys[g].t()) * st["scale"][l].double()
                score.masked_fill_(hidden, -math.inf)
                z = torch.logsumexp(score, dim=1)
                out[l, h, a:b] = torch.exp(score - z[:, None]) @ values[g]
                at = a * L * H + (l * H + h) * (b - a)
                lse[at:at + b - a] = z
    return (out, lse) if k == "prompt" else out


def _exact_compact(c, st):
    kp, vp = st["kp"].double().clone(), st["vp"].double().clone()
    for b in range(c["B"]):
        for l in range(c["L"]):
            n = int(st["lengths"][b, l])
            pos = torch.sort(st["order"][b, l, :n].long()).values
            j = torch.arange(n, device=DEV)
            page = st["table"][b, l, j // c["ps"]].long()
            kp[page, :, j % c["ps"]] = st["k"][b, l][:, pos].double().transpose(0, 1)
            vp[page, :, j % c["ps"]] = st["v"][b, l][:, pos].double().transpose(0, 1)
    return kp, vp, None


def _exact_rope(c, st):
    half, T, L = c["rot"] // 2, c["T"], c["L"]
    axis = [a for a, n in enumerate(st["sections"]) for _ in range(n)]
    turn = torch.empty((T, half), dtype=torch.complex128, device=DEV)
    for i in range(half):
        angle = st["pos"][axis[i]].double() * st["theta"] ** (-2.0 * i / c["rot"])
        turn[:, i] = torch.polar(torch.ones_like(angle), angle)
    at = torch.arange(c["rot"], device=DEV)
    first, second = (at[0::2], at[1::2]) if c["inter"] else (at[:half], at[half:])

    def spin(x):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    q, k = spin(st["q"].double().clone()), spin(st["k"].double().clone())
    if not c["store"]:
        return q, k
    kp, vp = st["kp"].double().clone(), st["vp"].double().clone()
    for l in range(L):
        keep = (st["slots"][l] >= 0).nonzero()[:, 0]
        slot = st["slots"][l][keep]
        kp[slot // c["ps"], :, slot % c["ps"]] = k[l][:, keep].transpose(0, 1)
        vp[slot // c["ps"], :, slot % c["ps"]] = st["v"][l][:, keep].double().transpose(0, 1)
    return q, kp, vp

"""Drivers of the hot path.  Only buffer management and call sequencing; every step runs in the HIP
library.

HotPath    one rectangular batch on pre-allocated buffers: importance -> select -> compact -> T
           decode steps.  Used by the benchmark, the smoke check and the end-to-end tests.
PagedPath  sequences of different lengths that come, ask again and go: packed prompts -> rotation ->
           attention -> importance and search per sequence -> pages -> further rows over the pages.
"""
from __future__ import annotations

from operator import index
from typing import Optional

import torch

from . import binding as B_


class HotPath:
    def __init__(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: torch.Tensor,
                 budget_tokens: int, decode_steps: int, tol_tokens: int = 0, max_iters: int = 64,
                 fixup: bool = True, evict_distance: Optional[int] = None):
        self.q, self.k, self.v, self.scale = q, k, v, scale
        self.B, self.L, self.H, self.N, self.D = q.shape
        self.Hkv = k.shape[2]
        self.budget_tokens, self.T = int(budget_tokens), int(decode_steps)
        self.tol_tokens, self.max_iters, self.fixup = tol_tokens, max_iters, fixup
        # append-only decode needs one slot per step; pruning at a fixed distance needs the ring plus
        # room for the survivors (never more than one per step)
        self.evict_distance = evict_distance
        self.decode_capacity = self.T if evict_distance is None else evict_distance + 1 + self.T
        dev, dt = q.device, q.dtype
        Bn, L, H, N, D, Hkv = self.B, self.L, self.H, self.N, self.D, self.Hkv
        code = B_.PKV_F32 if dt == torch.float32 else B_.PKV_BF16
        self.importance = torch.empty((Bn, L, N), dtype=torch.float32, device=dev)
        self.imp_ws = torch.empty(B_.prefixkv_workspace_bytes(B_.OP_IMPORTANCE, Bn, L, H, Hkv, N, D, code),
                                  dtype=torch.uint8, device=dev)
        self.sel = B_.SelectResult(
            order=torch.empty((Bn, L, N), dtype=torch.int32, device=dev),
            cum=torch.empty((Bn, L, N), dtype=torch.int64, device=dev),
            prefix=torch.empty((Bn, L, N), dtype=torch.float32, device=dev),
            lengths=torch.empty((Bn, L), dtype=torch.int32, device=dev),
            p=torch.empty(Bn, dtype=torch.float64, device=dev),
            iters=torch.empty(Bn, dtype=torch.int32, device=dev),
            raw_total=torch.empty(Bn, dtype=torch.int64, device=dev),
            status=torch.empty(Bn, dtype=torch.int32, device=dev))
        self.sel_ws = torch.empty(max(256, B_.select_workspace_bytes(Bn, L, N)), dtype=torch.uint8, device=dev)
        budget_cap = min(self.budget_tokens, L * N)
        self.cache_tokens = B_.prefixkv_cache_tokens_upper_bound(Bn, budget_cap, L, self.decode_capacity)
        self.cache = B_.CompactResult(
            kc=torch.empty(self.cache_tokens * Hkv * D, dtype=dt, device=dev),
            vc=torch.empty(self.cache_tokens * Hkv * D, dtype=dt, device=dev),
            kept_pos=torch.empty(self.cache_tokens, dtype=torch.int32, device=dev),
            seg_off=torch.empty((Bn, L), dtype=torch.int64, device=dev),
            caps=torch.empty((Bn, L), dtype=torch.int32, device=dev),
            lens=torch.empty((Bn, L), dtype=torch.int32, device=dev),
            cache_tokens=self.cache_tokens, Hkv=Hkv, D=D)
        self.out = torch.empty((max(self.T, 1), Bn, L, H, D), dtype=dt, device=dev)
        self.dec_ws = torch.empty(max(256, B_.prefixkv_workspace_bytes(B_.OP_DECODE, Bn, L, H, Hkv, N, D, code)),
                                  dtype=torch.uint8, device=dev)
        self._graph: Optional[torch.cuda.CUDAGraph] = None

    # ---- the four C-ABI calls, on pre-allocated buffers ------------------------------------------
    def run_importance(self, lse: Optional[torch.Tensor] = None):
        return B_.prefixkv_importance(self.q, self.k, self.scale, lse=lse, out=self.importance, ws=self.imp_ws)

    def run_select(self):
        return B_.prefixkv_select(self.importance, self.budget_tokens, self.tol_tokens, self.max_iters,
                                  self.fixup, out=self.sel, ws=self.sel_ws)

    def run_compact(self):
        return B_.prefixkv_compact(self.k, self.v, self.sel.order, self.sel.lengths, self.decode_capacity,
                                   self.cache_tokens, out=self.cache)

    def run_decode_step(self, t: int, dq, dk, dv):
        return self._decode(t, dq[t], dk[t], dv[t], self.out[t])

    def _decode(self, t: int, q, k, v, out):
        if self.evict_distance is not None:
            return B_.prefixkv_decode_attn_evict(self.cache, self.sel.lengths, q, k, v, self.scale, self.N, t + 1,
                                                 self.evict_distance, out=out, ws=self.dec_ws)
        return B_.prefixkv_decode_attn(self.cache, q, k, v, self.scale, self.N, out=out, ws=self.dec_ws)

    def run_decode_loop(self, dq, dk, dv):
        step_own = getattr(self.run_decode_step, "__func__", None) is not HotPath.run_decode_step
        if step_own or not all(isinstance(x, torch.Tensor) for x in (dq, dk, dv)):
            # steps that are made when they are asked for, or a step of the caller's own
            for t in range(self.T):
                self.run_decode_step(t, dq, dk, dv)
            return
        if self._plain() and B_.decode_attn_steps(self.cache, dq, dk, dv, self.scale, self.N, self.T, self.out, self.dec_ws):
            return
        # the steps' tensors as views made once: indexing four tensors per step costs as much as the call
        steps = [x[:self.T].unbind(0) for x in (dq, dk, dv, self.out)]
        if min(len(x) for x in steps) < self.T:
            raise IndexError(f"{self.T} decode steps need as many tensors")
        for t, (q, k, v, out) in enumerate(zip(*steps)):
            self._decode(t, q, k, v, out)

    def _plain(self) -> bool:
        """Whether a step is the binding's call without pruning, with nothing of the caller's in between."""
        return self.evict_distance is None and getattr(self._decode, "__func__", None) is HotPath._decode

    # ---- the decode loop as one HIP graph (T launches, no host work between them) -----------
    def capture_decode_loop(self, dq, dk, dv):
        self.run_compact()            # a valid cache state for the capture-time launches
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.run_decode_loop(dq, dk, dv)
        self._graph = g
        return g

    def replay_decode_loop(self):
        self._graph.replay()


_LONGEST = 8192      # positions of a prompt that the importance and the search take


class PagedPath:
    """S places for sequences over one pool of pages.  All layers of the model are called at once, as the queries, keys and
    values [L,heads,T,D] of the packed rows of all layers are given (bf16).  Nothing is read back: `status` [1] tells whether
    the last call that needed pages got them, `search` [S] what the search said (its status bits, 0 if nothing) of the last
    prompt of every place: a prompt that it could not rank, with NaN in a query for instance, keeps no entries."""

    def __init__(self, S: int, L: int, H: int, Hkv: int, D: int, scale: torch.Tensor, plan: B_.RopePlan, num_pages: int,
                 max_pages: int, page_size: int = 64, device="cuda"):
        if scale.dtype != torch.float32 or scale.shape != (L,) or not scale.is_contiguous():
            raise ValueError("scale must be contiguous f32 [L]")
        self.S, self.L, self.H, self.Hkv, self.D = S, L, H, Hkv, D
        self.scale, self.plan, self.device = scale, plan, torch.device(device)
        self.cache = B_.paged_cache(S, L, Hkv, D, page_size, num_pages, max_pages, torch.bfloat16, device)
        self.target = torch.zeros((S, L), dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.search = torch.zeros(S, dtype=torch.int32, device=device)
        self.page_ws = torch.empty(B_.page_workspace_bytes(S, L), dtype=torch.uint8, device=device)

    def _offsets(self, lengths) -> torch.Tensor:
        off = [0]
        for n in lengths:
            off.append(off[-1] + n)
        return torch.tensor(off, dtype=torch.int32).to(self.device, non_blocking=True)

    def _look_at(self, q, k, v, positions):
        """What a later step would refuse is refused before the first: no prompt is left rotated, no length counts rows that were
        not stored."""
        T = q.shape[2] if q.dim() == 4 else 0
        for x, heads in ((q, self.H), (k, self.Hkv), (v, self.Hkv)):
            if (x.shape != (self.L, heads, T, self.D) or x.dtype != torch.bfloat16 or x.stride(3) != 1 or x.data_ptr() % 16
                    or any(st % 8 for st, n in zip(x.stride()[:3], x.shape) if n > 1) or (T > 1 and x.stride(2) == 0)):
                raise ValueError("queries, keys and values must be bf16 [L,heads,T,D], with rows that begin at multiples of 16 bytes")
        if any(x.get_device() != y.get_device() for x, y in ((q, self.cache.kp), (k, q), (v, q), (positions, q), (self.scale, q))):
            raise ValueError("all tensors must be on the cache's GPU")
        if positions.dtype != torch.int32 or positions.shape != (self.plan.axes, T) or not positions.is_contiguous():
            raise ValueError("positions must be contiguous i32 [axes,T]")

    def prefill(self, places, lengths, q, k, v, positions, budgets, kept_pos=None):
        """Prompts of these lengths, packed, for sequences that begin at `places`; budgets[i] of the L * lengths[i] entries are
        kept.  q, k are rotated in place.  A place that still has a sequence is given to the new one.  -> attention output
        [L,H,T,D] (whatever `status`).  kept_pos: a list that receives the kept positions, ascending, -1 behind them."""
        places, lengths = [index(s) for s in places], [index(n) for n in lengths]
        if len(set(places)) != len(places) or any(not 0 <= s < self.S for s in places):
            raise ValueError(f"places must be different numbers in 0 ... {self.S - 1}")
        if not 0 < len(places) == len(lengths) == len(budgets) or any(n < 1 for n in lengths) or sum(lengths) > q.shape[2]:
            raise ValueError("a length and a budget per place, rows for all of them")
        budgets = [int(b) for b in budgets]
        if any(n > _LONGEST for n in lengths) or any(not 1 <= b < 1 << 63 for b in budgets):
            raise ValueError(f"prompts of at most {_LONGEST} positions, budgets of at least 1")
        self._look_at(q, k, v, positions)
        off = self._offsets(lengths)
        B_.prefixkv_rope(q, k, positions, self.plan, q_out=q, k_out=k)
        out, lse = B_.prefixkv_prefill_attn_packed(q, k, v, off, self.scale)
        rank, a = [], 0
        self.target.copy_(self.cache.lens)
        for place, n, budget in zip(places, lengths, budgets):
            rows = slice(a, a + n)
            imp = B_.prefixkv_importance(q[None, :, :, rows], k[None, :, :, rows], self.scale,
                                         lse=lse[self.L * self.H * a:self.L * self.H * (a + n)].view(1, self.L, self.H, n))
            sel = B_.prefixkv_select(imp, budget, want_prefix=False)
            self.target[place].copy_(sel.lengths[0])
            self.search[place:place + 1].copy_(sel.status)
            rank.append((place, rows, sel))
            a += n
        B_.prefixkv_page_resize(self.cache, self.target, status=self.status, ws=self.page_ws)
        for place, rows, sel in rank:
            lengths_now = sel.lengths * (self.status == 0)      # nothing is stored after a refused call
            pos = None if kept_pos is None else torch.full_like(sel.order, -1)
            B_.prefixkv_compact_paged(self._at(place), k[None, :, :, rows], v[None, :, :, rows], sel.order, lengths_now, kept_pos=pos)
            if kept_pos is not None:
                kept_pos.append(pos[0])
        return out

    def _at(self, place: int) -> B_.PagedCache:
        c = self.cache
        return B_.PagedCache(kp=c.kp, vp=c.vp, table=c.table[place:place + 1], lens=c.lens[place:place + 1], ring=c.ring,
                             state=c.state)

    def extend(self, lengths, q, k, v, positions):
        """Further rows of every sequence (lengths[s] of place s, 0 for one that waits): they are stored, and attend to what the
        cache holds and to each other.  One row each is a decode step.  -> attention output [L,H,T,D]; zeros if `status` says that
        the rows got no pages, and then nothing is stored and every length stays."""
        lengths = [int(n) for n in lengths]
        if len(lengths) != self.S or any(n < 0 for n in lengths) or sum(lengths) > q.shape[2]:
            raise ValueError("a length per place, rows for all of them")
        self._look_at(q, k, v, positions)
        off, T = self._offsets(lengths), q.shape[2]
        slots, _ = B_.prefixkv_page_append(self.cache, off, T, status=self.status, ws=self.page_ws)
        turned = B_.prefixkv_rope_store(self.cache, q, k, v, positions, self.plan, slots)
        out = B_.prefixkv_chunk_attn(self.cache, turned, off, self.scale, max(1, max(lengths)))
        # (after a refused call the lengths do not count the rows: they would see the last entries of the cache as their own)
        return out.masked_fill_(self.status != 0, 0)

    def end(self, places):
        """The sequences at these places are over: their pages are free again."""
        places = [index(s) for s in places]
        if any(not 0 <= s < self.S for s in places):
            raise ValueError(f"places must be in 0 ... {self.S - 1}")
        self.target.copy_(self.cache.lens)
        self.target[places] = 0
        B_.prefixkv_page_resize(self.cache, self.target, status=self.status, ws=self.page_ws)

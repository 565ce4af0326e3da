"""One attention layer of a serving program on the paged cache: prompts, decoding, and eviction back to a budget.

    python -m paper_2605_05219_amd.paged_session --requests 4 --prompt 3000 --steps 200 --budget 2000

`PagedLayer` owns the pools and hands out pages; `step` runs one call of new tokens for all requests (rotary append, attention, and the
weight that every row has gathered), `evict` brings requests that hold more than `budget` rows back to `keep` of them.
Everything is computed inside the library.  The command draws random projections, reports tokens per second and what
was evicted."""
from __future__ import annotations

import argparse
import time

import numpy as np

from . import attention, paged


class PagedLayer:
    def __init__(self, H_q, H_kv, d, n_req, n_pages, page_rows=64, rot=None, decay=0.95, **scaling):
        import torch
        self.shape = attention.make_attn_shape(H_q, H_kv, d, "bf16")
        self.H_q, self.H_kv, self.d, self.P, self.n_req, self.decay = H_q, H_kv, d, page_rows, n_req, decay
        freqs, amplitude = paged.attn_rope_freqs(d if rot is None else rot, **scaling)
        self.rope = paged.make_attn_rope(freqs, "half", amplitude)
        self.k_pool = torch.empty(n_pages, H_kv, page_rows, d, dtype=torch.bfloat16, device="cuda")
        self.v_pool = torch.empty(n_pages, H_kv, page_rows, d, dtype=torch.float16, device="cuda")
        self.w_pool = torch.empty(n_pages, H_kv, page_rows, device="cuda")
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = [[] for _ in range(n_req)]
        self.rows = np.zeros(n_req, np.int32)           # rows held
        self.pos = np.zeros(n_req, np.int32)            # position of the next token; the rows are fewer after an eviction
        self.workspace = None

    def _take(self, count):
        if count > len(self.free):
            raise RuntimeError(f"out of pages: {count} wanted, {len(self.free)} free")
        return [self.free.pop() for _ in range(count)]

    def _table(self):
        cu = np.concatenate([[0], np.cumsum([len(p) for p in self.pages])]).astype(np.int32)
        return cu, np.asarray([i for p in self.pages for i in p], np.int32)

    def _room(self, tokens, n_ids):
        import torch
        need = paged.attn_paged_workspace_bytes(self.shape, self.n_req, tokens, n_ids)
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = torch.empty(need + need // 4, dtype=torch.uint8, device="cuda")
        return self.workspace

    def step(self, q, k, v, lens):
        """New tokens of every request (lens[r] of them, packed): their attention output [T][H_q][d] in bf16.  q, k, v are bf16
        tensors [T][heads][d]."""
        import torch
        lens = np.asarray(lens, np.int32)
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        T = int(cu[-1])
        for r in range(self.n_req):
            self.pages[r] += self._take(-(-int(self.rows[r] + lens[r]) // self.P) - len(self.pages[r]))
        tcu, ids = self._table()
        ws = self._room(T, ids.size)
        turned = torch.empty(T, self.H_q, self.d, dtype=torch.bfloat16, device="cuda")
        o, lse = torch.empty_like(turned), torch.empty(T, self.H_q, device="cuda")
        paged.attn_rope_append(self.shape, self.rope, q, k, v, cu, self.pos, self.rows, self.k_pool, self.v_pool, tcu, ids, turned, ws)
        paged.attn_paged_prefill(self.shape, turned, None, cu, self.rows, self.k_pool, self.v_pool, tcu, ids, o, lse, ws)
        paged.attn_key_weights(self.shape, turned, lse, cu, self.rows, self.k_pool, tcu, ids, self.decay, self.w_pool, self.w_pool, ws)
        self.rows += lens
        self.pos += lens
        return o

    def evict(self, budget, keep, first=4, recent=64):
        """Requests of more than `budget` rows go back to `keep` (those that hold no more than `keep` stay as they are), among them the
        first `first` and the last `recent` as far as `keep` has room for them, the first before the last; returns the rows dropped (per head)."""
        import torch
        first = min(first, keep)
        recent = min(recent, keep - first)
        over = [r for r in range(self.n_req) if self.rows[r] > max(budget, keep)]
        if not over:
            return 0
        n, per = len(over), -(-keep // self.P)
        cu = np.concatenate([[0], np.cumsum([len(self.pages[r]) for r in over])]).astype(np.int32)
        ids = np.asarray([i for r in over for i in self.pages[r]], np.int32)
        new_cu = np.arange(n + 1, dtype=np.int32) * per
        new = self._take(n * per)
        try:
            new_ids = np.asarray(new, np.int32)
            index = torch.empty(n * keep * self.H_kv, dtype=torch.int32, device="cuda")
            paged.attn_evict(self.shape, self.rows[over], np.full(n, keep), np.full(n, first), np.full(n, recent), self.k_pool, self.v_pool, self.w_pool,
                             cu, ids, new_cu, new_ids, index, self._room(0, ids.size + new_ids.size))
        except Exception:
            self.free += reversed(new)
            raise
        dropped = int((self.rows[over] - keep).sum())
        for i, r in enumerate(over):         # later calls of this stream see the copies; the old pages may be written by them
            self.free += self.pages[r]
            self.pages[r] = new[i * per:(i + 1) * per]
        self.rows[over] = keep
        return dropped


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=3000)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--budget", type=int, default=2000)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--d", type=int, default=128)
    ap.add_argument("--page-rows", type=int, default=64)
    a = ap.parse_args(argv)
    keep = a.budget * 3 // 4
    per = -(-(a.prompt + a.steps) // a.page_rows) + -(-keep // a.page_rows)
    layer = PagedLayer(a.heads, a.kv_heads, a.d, a.requests, a.requests * per, a.page_rows)
    gen = torch.Generator(device="cuda").manual_seed(0)

    def tokens(n):
        return [torch.randn(n, h, a.d, generator=gen, device="cuda").bfloat16() for h in (a.heads, a.kv_heads, a.kv_heads)]

    t0 = time.perf_counter()
    layer.step(*tokens(a.requests * a.prompt), [a.prompt] * a.requests)
    dropped = layer.evict(a.budget, keep)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    for _ in range(a.steps):
        layer.step(*tokens(a.requests), [1] * a.requests)
        dropped += layer.evict(a.budget, keep)
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    print(f"{a.requests} prompts of {a.prompt} tokens: {(t1 - t0) * 1e3:.1f} ms; {a.steps} steps: {(t2 - t1) / max(a.steps, 1) * 1e6:.0f} us each; "
          f"{dropped} rows evicted, {[int(x) for x in layer.rows]} held at positions {[int(x) for x in layer.pos]}")


if __name__ == "__main__":
    main()

"""A rank's SPD block served in 8 bits over a paged KV cache: prompts in chunks and decode steps of several sequences mixed in one call.

The operators of include/spd_q8.h put together the way a serving program would: 8-bit projections, keys and values quantised into
pages as they are written, attention over the pages (with a sliding window and sinks if asked for), the SPD fold X + Y_r in the second norm, the
partial MLP output added onto Y_r, and the one sync point that an SPD block keeps as a sum over the ranks' slots.

    python examples/paged_q8_block.py            # LLaMA2-70B rank of 8: two prompts in chunks of 256, four sequences decoding beside them
"""
from __future__ import annotations

import os
import sys
import time
from typing import Dict, Sequence

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2502_20727_amd import binding as B  # noqa: E402
from paper_2502_20727_amd import inputs  # noqa: E402
from paper_2502_20727_amd.workloads import BF16, Workload  # noqa: E402


class PagedPool:
    """Pages handed out as sequences grow: which page holds what is this class's to say, the library only follows the table."""

    def __init__(self, n_pages: int, page_size: int):
        self.free, self.page_size, self.table = list(range(n_pages))[::-1], page_size, {}

    def grow(self, seq: int, end: int) -> None:
        row = self.table.setdefault(seq, [])
        while len(row) * self.page_size < end:
            row.append(self.free.pop())

    def release(self, seq: int) -> None:
        self.free += self.table.pop(seq)


class Q8Block:
    """One rank's share of one SPD block: weights in 8 bits, buffers for at most `max_tokens` tokens a call."""

    def __init__(self, w: Workload, shard: Dict[str, np.ndarray], rank: int, max_tokens: int, n_pages: int, page_size: int = 64, max_ctx: int = 4096,
                 cache: int = B.SPD_E4M3, device="cuda"):
        self.w, self.rank = w, rank
        self.ctx = None
        self.ctx = B.spd_create(B.make_config(w, max_batch=1, max_ctx=32, max_tokens=max_tokens))      # for the sum over the ranks
        q, kv, d, h, f = w.q_per_rank, w.kv_per_rank, w.head_dim, w.hidden, w.ffn_per_rank
        self.pages = B.DevicePages(B.spd_pages_config(q, kv, d, page_size, n_pages, B.SPD_BF16, cache, max_ctx, w.rope_base), device)
        self.widths = {"qkv": (h, (q + 2 * kv) * d), "o": (q * d, h), "gu": (h, 2 * f), "down": (f, h)}
        dense = {"qkv": np.concatenate([shard["wq"], shard["wk"], shard["wv"]], 1), "o": shard["wo"],
                 "gu": np.concatenate([shard["wg"], shard["wu"]], 1), "down": shard["wd"]}
        self.weights = {n: torch.from_numpy(B.spd_q8_pack(np.ascontiguousarray(m))).to(device) for n, m in dense.items()}
        self.gains = [torch.from_numpy(shard[n]).to(device) for n in ("g1", "g2")]
        scratch = max(B.spd_q8_matmul_workspace(max_tokens, *s) for s in self.widths.values())
        self.scratch = torch.zeros(max(scratch, 1), dtype=torch.uint8, device=device)

        def rows(n, t):
            return torch.empty(max_tokens, n, dtype=t, device=device)
        wide = max(h, q * d, (f + 15) // 16 * 16)
        self.codes, self.scales = rows(wide, torch.int8), torch.empty(max_tokens, device=device)
        self.qkv, self.q, self.att = rows((q + 2 * kv) * d, torch.bfloat16), rows(q * d, torch.bfloat16), rows(q * d, torch.bfloat16)
        self.y, self.gu = rows(h, torch.float32), rows(2 * f, torch.bfloat16)

    def _product(self, name: str, out, add=None) -> None:
        k, n = self.widths[name]
        B.spd_q8_matmul(self.codes[:len(out), :k], self.scales[:len(out)], self.weights[name], n, add, out, self.scratch)

    def forward(self, plan: B.PagePlan, x, slots, x_out) -> None:
        """x, x_out [tokens, hidden], slots [tp, tokens, hidden], fp32; the peers' slots are given, slot `rank` is written."""
        n, w = plan.tokens, self.w
        qkv, q, att, y, gu = (t[:n] for t in (self.qkv, self.q, self.att, self.y, self.gu))
        codes, scales = self.codes[:n], self.scales[:n]
        B.spd_q8_norm(x, None, self.gains[0], w.rms_eps, None, codes[:, :w.hidden], scales)
        self._product("qkv", qkv)
        B.spd_pages_write(self.pages.ctx, plan, qkv, self.pages.rope, self.pages.pool, q)
        B.spd_pages_attention(self.pages.ctx, plan, q, self.pages.pool, att, plan.workspace)
        B.spd_q8_rows(att, codes[:, :att.shape[1]], scales)
        self._product("o", y)                                                    # Y_r
        B.spd_q8_norm(x, y, self.gains[1], w.rms_eps, None, codes[:, :w.hidden], scales)      # of X + Y_r
        self._product("gu", gu)
        B.spd_q8_swiglu(gu, codes[:, :w.ffn_per_rank], scales)
        self._product("down", slots[self.rank], y)                               # Y_r + Z_r
        # X + sum over the ranks
        B.spd_rank_sum(self.ctx, x, slots, w.tp, n * w.hidden, x_out)

    def close(self) -> None:
        if self.ctx:
            B.spd_destroy(self.ctx)
            self.ctx = None
        self.pages.close()


def main() -> None:
    w = Workload(name="70b-rank", hidden=8192, n_q_heads=64, n_kv_heads=8, head_dim=128, ffn=28672, n_layers=1, tp=8, dtype=BF16, seed=3,
                 batch=6, q_len=1, ctx=2048, mask=(1,))
    rank, chunk, prompt = 0, 256, 1024
    block = Q8Block(w, inputs.layer_shard(w, 0, rank), rank, max_tokens=2 * chunk + 4, n_pages=256, max_ctx=4096)
    pool = PagedPool(256, 64)
    g = torch.Generator(device="cuda").manual_seed(0)
    done: Dict[int, int] = {s: 0 for s in range(6)}

    def step(lens: Sequence[int]) -> None:
        for s, n in enumerate(lens):
            pool.grow(s, done[s] + n)
        plan = B.PagePlan(block.pages, [done[s] for s in range(6)], lens, [pool.table.get(s, []) for s in range(6)], window=2048, sinks=4)
        x = torch.randn(plan.tokens, w.hidden, generator=g, device="cuda")
        slots = 0.05 * torch.randn(w.tp, plan.tokens, w.hidden, generator=g, device="cuda")
        out = torch.empty_like(x)
        torch.cuda.synchronize()
        t = time.perf_counter()
        block.forward(plan, x, slots, out)
        torch.cuda.synchronize()
        print(f"{plan.tokens:4d} tokens ({' + '.join(map(str, lens))}) at {list(done.values())}: {(time.perf_counter() - t) * 1e6:8.1f} us, "
              f"output rms {float(out.square().mean().sqrt()):.3f}", flush=True)
        for s, n in enumerate(lens):
            done[s] += n

    step([64] * 4 + [0, 0])                                  # four short prompts
    for _ in range(prompt // chunk):                         # two long ones in chunks, the four decoding beside them
        step([1] * 4 + [chunk] * 2)
    for _ in range(4):
        step([1] * 6)
    block.close()


if __name__ == "__main__":
    main()

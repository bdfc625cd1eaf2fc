"""From prompts to compacted caches: a prefill in chunks over a paged cache, then the layer-wise eviction.

A ragged batch of prompts goes through the layers chunk by chunk, as a serving program does it:

1. ``PagePool.tables`` gives the chunk's tokens pages, slots and positions (on the GPU, from lengths);
2. per layer, ``PagedCache.write`` puts the chunk's K/V rows into their slots and ``PagedCache.attention``
   attends over the pages, returning the output and every row's log-sum-exp;
3. at the end of the prompts, ``PagedCache.gather`` hands each evicting layer's cache to
   ``Plan.evict_prefill``, with the window rows' log-sum-exp from step 2 (one pass over K instead of two);
   the FULL layers stay in their pages;
4. generation: the evicting layers' caches go on in the decode arena, the FULL layers in their pages
   (write, and attention of single tokens).

The model is a stand-in: random projections of random hidden states.  Run: python examples/paged_prefill.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_15157_gb300 import kvev, paged  # noqa: E402

FULL, SNAPKV, H2O, STREAMING = kvev.FULL, kvev.SNAPKV, kvev.H2O, kvev.STREAMING


def run(prompts=(2900, 1337, 700), chunk=512, steps=4, H_q=8, H_kv=2, d=128, page=16, W=32, budget=256, seed=0):
    """Returns (plan, eviction buffers, the FULL layer's last attention output, arena, per-layer Q/K/V)."""
    dev, bf16 = "cuda", torch.bfloat16
    route, route_decode = [SNAPKV, FULL, H2O, STREAMING], [FULL, FULL, H2O, STREAMING]
    L, B = len(route), len(prompts)
    g = torch.Generator(device=dev).manual_seed(seed)
    S_cap = (max(prompts) + 127) // 128 * 128
    plan = kvev.Plan(L, H_q, H_kv, d, route, [budget] * L, W, pool_kernel=7, sink=4, route_decode=route_decode)

    # the pool: one block table for all layers, pages of each layer in one tensor
    width = -(-(max(prompts) + steps) // page)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    pages = B * width
    pool = paged.PagePool(pages, page, table)
    caches = [paged.PagedCache.empty(pages, page, H_kv, d, table) for _ in range(L)]
    lens = torch.zeros(B, dtype=torch.int32, device=dev)

    # the stand-in model's rows, request by request: the fused projection [tokens][H_q + 2 H_kv][d] of a layer
    qkv = [[torch.randn((n + steps, H_q + 2 * H_kv, d), generator=g, device=dev).to(bf16) for n in prompts] for _ in range(L)]

    def forward(new, done):
        """One pass of `new` tokens per request behind `done`; (outputs, log-sum-exp, cu) per layer."""
        T = sum(new)
        _, cu, slots, _, granted = pool.tables(lens, torch.tensor(new, dtype=torch.int32, device=dev), T, kv_lens=lens)
        outs, lses = [], []
        for l in range(L):
            rows = torch.cat([qkv[l][s][done[s]:done[s] + new[s]] for s in range(B)])
            q, k, v = rows[:, :H_q], rows[:, H_q:H_q + H_kv], rows[:, H_q + H_kv:]
            caches[l].write(k, v, slots)
            lse = torch.empty((T, H_q), dtype=torch.float32, device=dev)
            outs.append(caches[l].attention(q, cu, lens, lse=lse))
            lses.append(lse)
        return outs, lses, granted

    # ---- prefill, chunk by chunk; the last W rows' log-sum-exp of every prompt are kept ----
    done = [0] * B
    window_lse = [torch.zeros((B, H_q, W), dtype=torch.float32, device=dev) for _ in range(L)]
    while any(a < n for a, n in zip(done, prompts)):
        new = [min(chunk, n - a) for a, n in zip(done, prompts)]
        _, lses, granted = forward(new, done)
        assert bool(granted.all()), "the pool is out of pages"
        row = 0
        for s, (a, q) in enumerate(zip(done, new)):
            first = max(a, prompts[s] - W)  # positions of this chunk inside the window
            if first < a + q:
                for l in range(L):
                    window_lse[l][s, :, first - prompts[s] + W:a + q - prompts[s] + W] = lses[l][row + first - a:row + q].T
            row += q
        done = [a + q for a, q in zip(done, new)]

    # ---- eviction: the evicting layers' caches leave their pages ----
    K, V, Q = [None] * L, [None] * L, [None] * L
    for l in range(L):
        if route[l] == FULL:
            continue
        K[l] = torch.zeros((B, H_kv, S_cap, d), dtype=bf16, device=dev)
        V[l] = torch.zeros_like(K[l])
        caches[l].gather(lens, K[l], V[l])
        if route[l] in (SNAPKV, H2O):
            Q[l] = torch.stack([qkv[l][s][n - W:n, :H_q].transpose(0, 1) for s, n in enumerate(prompts)]).contiguous()
    bufs = plan.buffers(B, S_cap)
    plan.evict_prefill(K, V, Q, lens, B, S_cap, bufs, lse=[window_lse[l] if Q[l] is not None else None for l in range(L)])
    arena = kvev.DecodeArena(plan, B, growth=steps)
    arena.init_from_prefill(bufs, lens)

    # ---- generation ----
    out = None
    for _ in range(steps):
        new = [1] * B
        outs, _, granted = forward(new, done)  # (a serving program passes the FULL layers only)
        out = outs[route.index(FULL)]
        k_new, v_new, q_new = [None] * L, [None] * L, [None] * L
        for l in range(L):
            if route[l] != FULL:
                rows = torch.stack([qkv[l][s][done[s]] for s in range(B)])
                q_new[l], k_new[l], v_new[l] = (x.contiguous() for x in rows.split([H_q, H_kv, H_kv], dim=1))
        arena.step(k_new, v_new, q_new)
        done = [a + 1 for a in done]

    status = [c.status() for c in caches] + [int(pool.device_status), plan.status()]
    assert not any(status), status
    return {"plan": plan, "bufs": bufs, "out": out, "arena": arena, "qkv": qkv, "K": K, "V": V, "Q": Q, "pool": pool,
            "lens": lens, "prompts": prompts, "S_cap": S_cap, "window_lse": window_lse, "route": route, "W": W, "H_kv": H_kv}


if __name__ == "__main__":
    r = run()
    used = r["pool"].num_pages - int(r["pool"].free_count)
    kept = r["bufs"]["out_count"].sum(dim=(1, 2)).tolist()
    print(f"prompts {r['prompts']}: {used} pages held, rows kept per layer {kept}")
    r["pool"].release(r["lens"], torch.ones_like(r["lens"]))
    print(f"released: {int(r['pool'].free_count)} of {r['pool'].num_pages} pages free")

"""The paged cache in front of the eviction, as cases that can be timed and compared.

A serving program holds its prompts' K/V in pages while they are prefilled in chunks, and the caches of
its FULL layers for good.  The passes here are the ones it makes of the paged operators:

* ``step``    one scheduler step: the pages of finished requests go back to the pool (release), then
              block tables, slots and positions of the new tokens are built from the request lengths
              (tables);
* ``write``   the new tokens' K/V rows go to their slots, one layer;
* ``attend``  attention of the new tokens (a prompt's chunk, or single tokens) over the pages, one
              layer: the output rows and their log-sum-exp;
* ``gather``  the pages of whole prompts as the contiguous caches that the prefill eviction reads, one
              layer.

A case is a dict of plain values.  ``prepare`` makes what the program has in hand before the call,
``run`` makes one pass, ``exact`` gives the attention's numbers from its definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

SINK = 4          # leading positions with raised logits (attention sinks)
SINK_LOGIT = 5.0

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
# Llama-3.1-8B's geometry, the one of the paper's experiments and of the benchmark
LLAMA = {"H_q": 32, "H_kv": 8, "d": 128}


def _case(name, kind, B, new_lo, new_hi, ctx_lo, ctx_hi, chunks, page, H_q=32, H_kv=8, d=128, dtype="bf16", heads_first=False,
          window=0, done=0, scarce=False):
    """B requests with ctx_lo..ctx_hi tokens in the cache; `chunks` of them bring new_lo..new_hi new
    tokens, the others one (``attend``, ``write``, ``step``) or none (``gather``).  heads_first: pages
    are [H_kv][page][d], else [page][H_kv][d].  window: sliding window, 0 = none.  done: requests that
    finish in this step.  scarce: the pool lacks pages for the last of them."""
    return {"name": name, "kind": kind, "B": B, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "chunks": chunks, "page": page, "H_q": H_q, "H_kv": H_kv, "d": d, "dtype": dtype, "heads_first": heads_first,
            "window": window, "done": done, "scarce": scarce}


def listed():
    return [
        # The smallest scheduler step: sixteen generations, one token each, one of them finished.
        _case("step_b16", "step", 16, 1, 1, 1000, 16384, 0, 16, done=1),
        # A busy server's step: 256 requests, 32 of them prefill chunks of 512 tokens or so, 20 finished.
        _case("step_b256", "step", 256, 300, 700, 0, 32768, 32, 16, done=20),
        # One generated token of sixteen requests: latency.
        _case("write_b16", "write", 16, 1, 1, 1000, 16384, 0, 16, **LLAMA),
        # Four prompts' chunks of up to 4,096 tokens.
        _case("write_16k", "write", 4, 4000, 4096, 0, 8192, 4, 16, **LLAMA),
        # One generation at a 4K context: the smallest attention call, where latency counts.
        _case("decode_b1_4k", "attend", 1, 1, 1, 4095, 4095, 0, 16, **LLAMA),
        # The benchmark's decode batch before its caches are compacted: 16 requests at 16K.
        _case("decode_b16_16k", "attend", 16, 1, 1, 16384, 16384, 0, 64, heads_first=True, **LLAMA),
        # Many ragged generations in half precision, 64-wide heads.
        _case("decode_b64_ragged", "attend", 64, 1, 1, 200, 8192, 0, 16, d=64, dtype="fp16"),
        # A mixed step: four prefill chunks between 28 generations, on a layer with a sliding window.
        _case("mixed_b32_window", "attend", 32, 500, 2048, 100, 16384, 4, 16, window=4096, **LLAMA),
        # A whole 8K prompt in one call (nothing in the cache before).
        _case("prompt_8k", "attend", 1, 8192, 8192, 0, 0, 1, 64, **LLAMA),
        # The last chunk of a 32K prompt.
        _case("chunk_4k_of_32k", "attend", 1, 4096, 4096, 28672, 28672, 1, 128, heads_first=True, **LLAMA),
        # One 8K prompt handed to the eviction.
        _case("gather_8k", "gather", 1, 0, 0, 8191, 8191, 0, 64, heads_first=True, **LLAMA),
        # The benchmark's headline batch handed over: eight ragged prompts of 16K to 32K.
        _case("gather_b8_long", "gather", 8, 0, 0, 16384, 32768, 0, 16, **LLAMA),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: batches of 1 to 256, contexts to 32K, chunks to 4K, pages of
    16 to 128, groups of 1 to 16 heads, both head sizes, types and page layouts, windows."""
    kind = rng.choice(["attend", "attend", "attend", "attend", "step", "write", "gather"])
    H_q, H_kv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 8), (64, 8), (4, 2), (8, 2), (32, 2), (12, 4), (14, 2)])
    geo = {"H_q": H_q, "H_kv": H_kv, "d": rng.choice([128, 128, 64]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
           "page": rng.choice([16, 16, 32, 64, 128]), "heads_first": rng.random() < 0.4}
    ctx_hi = _log_int(rng, 1, 32768)
    ctx_lo = rng.choice([0, ctx_hi // 4, ctx_hi // 2, ctx_hi])
    if kind == "step":
        B = _log_int(rng, 1, 256)
        chunks = rng.choice([0, B // 8, B])
        hi = max(1, min(_log_int(rng, 1, 4096), 16384 // max(chunks, 1)))
        c = _case("", kind, B, max(1, hi // 3), hi, ctx_lo, ctx_hi, chunks, done=rng.choice([0, B // 10]),
                  scarce=rng.random() < 0.25, **geo)
    elif kind == "write":
        B = _log_int(rng, 1, 64)
        hi = max(1, min(_log_int(rng, 1, 4096), 16384 // B))
        c = _case("", kind, B, max(1, hi // 3), hi, 0, min(ctx_hi, 131072 // B), B, **geo)
    elif kind == "gather":
        B = rng.choice([1, 1, 2, 3, 5, 8])
        c = _case("", kind, B, 0, 0, ctx_lo, ctx_hi, 0, **geo)
    elif rng.random() < 0.5:  # generations
        B = _log_int(rng, 1, 64)
        ctx_hi = max(1, min(ctx_hi, 262144 // B))
        c = _case("", kind, B, 1, 1, min(ctx_lo, ctx_hi), ctx_hi, 0, window=rng.choice([0, 0, 1024, 4096]), **geo)
    else:                     # chunks, some beside generations
        chunks = rng.choice([1, 1, 2, 3, 4])
        B = chunks + rng.choice([0, 0, 3, 12])
        hi = max(2, _log_int(rng, 2, 4096) // chunks)
        ctx_hi = min(ctx_hi, 28672 // chunks)
        c = _case("", kind, B, max(1, hi // 2), hi, min(ctx_lo, ctx_hi), ctx_hi, chunks, window=rng.choice([0, 0, 0, 1000, 4096]), **geo)
    return {k: v for k, v in c.items() if k != "name"}


# ---- shapes that follow from a case alone ---------------------------------------------------------

def _lengths(c):
    """(tokens in the cache before, new tokens, finished) of each request."""
    r = random.Random("%(B)d/%(new_lo)d/%(new_hi)d/%(ctx_lo)d/%(ctx_hi)d/%(chunks)d/%(done)d" % c)
    ctx = [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["B"])]
    new = [0 if c["kind"] == "gather" else 1] * c["B"]
    for s in r.sample(range(c["B"]), c["chunks"]):
        new[s] = r.randint(c["new_lo"], c["new_hi"])
    done = [0] * c["B"]
    for s in r.sample(range(c["B"]), c["done"]):
        done[s], new[s] = 1, 0
    return ctx, new, done


def _pages(n, page):
    return -(-n // page)


def _seen(c):
    """(key positions a request's rows see together, (query, key) pairs) summed over the requests."""
    keys = pairs = 0
    for n, q, _ in zip(*_lengths(c)):
        w = c["window"] or n + q
        first = max(0, n + 1 - w)
        keys += n + q - first
        # row at position t sees min(t + 1, w) keys
        a, b = min(max(w - 1 - n, 0), q), q
        pairs += sum((n + 1, n + a)) * a // 2 + (b - a) * w
    return keys, pairs


def work(case):
    """Bytes and operations that a pass cannot do without."""
    c = case
    ctx, new, done = _lengths(c)
    B, T, e = c["B"], sum(new), 2
    row = c["H_kv"] * c["d"] * e
    if c["kind"] == "step":
        freed = sum(_pages(n, c["page"]) for n, f in zip(ctx, done) if f)
        taken = sum(_pages(n + q, c["page"]) - _pages(n, c["page"]) for n, q in zip(ctx, new))
        # lengths, flags and counts in and out; pages moved twice (read, written); a slot and a position per token
        return {"bytes": 4 * (3 * B + 3 * B + 1) + 8 * (freed + taken) + 8 * T, "flops": 0}
    if c["kind"] == "write":
        return {"bytes": 2 * 2 * T * row + 4 * T, "flops": 0}
    if c["kind"] == "gather":
        return {"bytes": 2 * 2 * sum(ctx) * row + 4 * sum(_pages(n, c["page"]) for n in ctx), "flops": 0}
    keys, pairs = _seen(c)
    qo = 2 * T * c["H_q"] * c["d"] * e + 4 * T * c["H_q"]
    return {"bytes": 2 * keys * row + qo + 4 * _pages(keys, c["page"]), "flops": 4 * c["d"] * c["H_q"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 131 + what)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _held(c, seed, held, spare):
    """A block table whose requests hold `held` pages each, scattered over the pool, and the free pages."""
    total = sum(held) + spare
    perm = torch.randperm(total, generator=_gen(seed, 1), device="cuda").to(torch.int32)
    width = max(1, _pages(max(a + b for a, b, _ in zip(*_lengths(c))), c["page"]))
    col = torch.arange(width, device="cuda")
    n = _ints(held).long()
    at = (n.cumsum(0) - n)[:, None] + col
    table = torch.where(col < n[:, None], perm[at.clamp(max=total - 1)], -1).to(torch.int32)
    free = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    free[:spare] = perm[sum(held):]
    return table, free, total


def _pool(c, seed, pages, what):
    """A layer's pages, seen as [pages][page][H_kv][d] whatever their order in memory."""
    H, p, d = c["H_kv"], c["page"], c["d"]
    shape = (pages, H, p, d) if c["heads_first"] else (pages, p, H, d)
    x = torch.randn(shape, generator=_gen(seed, what), device="cuda", dtype=DTYPES[c["dtype"]])
    return x.transpose(1, 2) if c["heads_first"] else x


def prepare(case, seed):
    c = case
    ctx, new, done = _lengths(c)
    B, T, dt = c["B"], sum(new), DTYPES[c["dtype"]]
    st = {"case": c, "ctx": ctx, "new": new, "T": T, "lens": _ints(ctx), "new_lens": _ints(new)}
    before = [_pages(n, c["page"]) for n in ctx]
    after = [_pages(n + q, c["page"]) for n, q in zip(ctx, new)]
    if c["kind"] == "step":
        spare = (sum(after) - sum(before)) * 2 // 3 if c["scarce"] else sum(after) - sum(before) + 64
        st["table"], st["free"], st["pages"] = _held(c, seed, before, spare)
        st["done"] = _ints(done)
        st["free_count"] = _ints([spare])
        st["out"] = {k: torch.empty(n, dtype=torch.int32, device="cuda")
                     for k, n in (("lens_mid", B), ("count_mid", 1), ("kv_lens", B), ("cu", B + 1), ("slots", T), ("positions", T),
                                  ("granted", B), ("count", 1))}
    else:
        st["table"], _, pages = _held(c, seed, after, 3)
        st["K"], st["V"] = _pool(c, seed, pages, 2), _pool(c, seed, pages, 3)
        st["kv_lens"] = _ints([n + q for n, q in zip(ctx, new)])
        cu = [0]
        for q in new:
            cu.append(cu[-1] + q)
        st["cu"], st["cu_host"] = _ints(cu), cu
        t = torch.arange(T, device="cuda")
        s = torch.searchsorted(st["cu"][1:], t, right=True)
        pos = t - st["cu"][s] + st["lens"][s]
        st["slots"] = (st["table"][s, pos // c["page"]] * c["page"] + pos % c["page"]).to(torch.int32)
    if c["kind"] == "write":
        st["k"] = torch.randn((T, c["H_kv"], c["d"]), generator=_gen(seed, 4), device="cuda", dtype=dt)
        st["v"] = torch.randn((T, c["H_kv"], c["d"]), generator=_gen(seed, 5), device="cuda", dtype=dt)
    if c["kind"] == "gather":
        cap = max(1, -(-max(ctx) // 256) * 256)
        st["out_K"] = torch.zeros((B, c["H_kv"], cap, c["d"]), dtype=dt, device="cuda")
        st["out_V"] = torch.zeros_like(st["out_K"])
    if c["kind"] == "attend":
        # the queries of a KV head share a direction, and the first positions' keys lie along it
        G, H, d = c["H_q"] // c["H_kv"], c["H_kv"], c["d"]
        u = torch.randn((H, d), generator=_gen(seed, 6), device="cuda")
        u = u / u.norm(dim=1, keepdim=True)
        q = 1.5 * torch.randn((T, H, G, d), generator=_gen(seed, 7), device="cuda") + math.sqrt(d) * u[None, :, None, :]
        st["q"] = q.to(dt).view(T, c["H_q"], d)
        t = torch.arange(SINK, device="cuda")
        s = torch.arange(B, device="cuda")[:, None].expand(B, SINK)
        page = st["table"][s, (t // c["page"]).expand(B, SINK)].long().clamp(min=0)
        st["K"][page, t.expand(B, SINK) % c["page"]] += (SINK_LOGIT * u).to(dt)
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((T, c["H_q"]), dtype=torch.float32, device="cuda")
    if own:  # the handle a serving program keeps: the pool, its tables and a workspace
        from paper_2606_15157_gb300 import paged
        if c["kind"] == "step":
            st["pool"] = paged.PagePool(st["pages"], c["page"], st["table"], st["free"])
        else:
            st["cache"] = paged.PagedCache(st["K"], st["V"], st["table"])
    return st


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"step": _own_step, "write": _own_write, "attend": _own_attend, "gather": _own_gather}[kind](state)
    return {"step": _plain_step, "write": _plain_write, "attend": _plain_attend, "gather": _plain_gather}[kind](state)


def _own_step(st):
    o = st["out"]
    st["pool"].release(st["lens"], st["done"], free_count=st["free_count"], lens_out=o["lens_mid"], free_count_out=o["count_mid"])
    st["pool"].tables(o["lens_mid"], st["new_lens"], st["T"], free_count=o["count_mid"], kv_lens=o["kv_lens"], cu=o["cu"],
                      slots=o["slots"], positions=o["positions"], granted=o["granted"], free_count_out=o["count"])
    return {"table": st["table"], "free": st["free"], "kv_lens": o["kv_lens"], "cu": o["cu"], "slots": o["slots"],
            "positions": o["positions"], "granted": o["granted"], "count": o["count"]}


def _own_write(st):
    st["cache"].write(st["k"], st["v"], st["slots"])
    return st["K"], st["V"]


def _own_attend(st):
    st["cache"].attention(st["q"], st["cu"], st["kv_lens"], window=st["case"]["window"], out=st["o"], lse=st["lse"])
    return st["o"], st["lse"]


def _own_gather(st):
    st["cache"].gather(st["kv_lens"], st["out_K"], st["out_V"])
    return st["out_K"], st["out_V"]


def _plain_step(st):
    page, table, free = st["case"]["page"], st["table"], st["free"]
    width = table.shape[1]
    col = torch.arange(width, device="cuda")
    # the finished requests' pages on top of the free ones, in request order
    lens = st["lens"].long()
    freed = torch.where(st["done"] != 0, (lens + page - 1) // page, 0)
    first = st["free_count"] + freed.cumsum(0) - freed
    at = torch.where(col < freed[:, None], first[:, None] + col, free.numel())
    free = torch.cat((free, free[:1])).scatter_(0, at.view(-1), table.view(-1))[:-1]
    count = st["free_count"] + freed.sum()
    lens = torch.where(st["done"] != 0, 0, lens)
    # new pages from the top of the free ones, in request order while they last
    new = st["new_lens"].long()
    held = (lens + page - 1) // page
    need = (lens + new + page - 1) // page - held
    upto = need.cumsum(0)
    granted = (need == 0) | (upto <= count)
    k = col - held[:, None]
    fresh = (k >= 0) & (k < need[:, None]) & granted[:, None]
    table = torch.where(fresh, free[(count - 1 - (upto - need)[:, None] - k).clamp(0, free.numel() - 1)], table)
    kv_lens = lens + torch.where(granted, new, 0)
    cu = torch.cat((new[:1] * 0, new.cumsum(0)))
    t = torch.arange(st["T"], device="cuda")
    s = torch.searchsorted(cu[1:], t, right=True)
    pos = lens[s] + t - cu[s]
    slots = table[s, pos // page] * page + pos % page
    i32 = lambda x: x.to(torch.int32)
    return {"table": table, "free": free, "kv_lens": i32(kv_lens), "cu": i32(cu), "slots": i32(torch.where(granted[s], slots, -1)),
            "positions": i32(torch.where(granted[s], pos, -1)), "granted": i32(granted),
            "count": i32(count - torch.where(granted, need, 0).sum())}


def _plain_write(st):
    page = st["case"]["page"]
    slots = st["slots"].long()
    st["K"][slots // page, slots % page] = st["k"]
    st["V"][slots // page, slots % page] = st["v"]
    return st["K"], st["V"]


def _plain_rows(st, pool, requests, n):
    """The first n rows of the requests' pages in 32 bits, [request][H_kv][n][d]; rows past a request's end are 0."""
    c = st["case"]
    pages = st["table"][requests, :_pages(n, c["page"])].long().clamp(min=0)
    x = pool[pages].flatten(1, 2)[:, :n].transpose(1, 2).float()
    there = torch.arange(n, device="cuda") < st["kv_lens"][requests, None]
    return torch.where(there[:, None, :, None], x, 0.0)


def _plain_rows_of(st, requests, q, first, n):
    """Attention of q [request][row][H_kv][G][d] (32 bits), rows at positions first + i, over n keys."""
    c = st["case"]
    K, V = _plain_rows(st, st["K"], requests, n), _plain_rows(st, st["V"], requests, n)
    R, H, G, d = q.shape[1:]
    S = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(-1, H, G * R, d), K.transpose(2, 3)) / math.sqrt(d)
    S = S.view(-1, H, G, R, n)
    t = first[:, None] + torch.arange(R, device="cuda")
    k = torch.arange(n, device="cuda")
    sees = k <= t[..., None]
    if c["window"]:
        sees &= k > t[..., None] - c["window"]
    S.masked_fill_(~sees[:, None, None], float("-inf"))
    m = S.amax(-1, keepdim=True).clamp(min=-3e38)
    S.sub_(m).exp_()
    z = S.sum(-1, keepdim=True)
    o = torch.matmul(S.view(-1, H, G * R, n), V).view(-1, H, G, R, d) / z
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3), (m + z.log()).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)


def _plain_attend(st):
    c, new, cu = st["case"], st["new"], st["cu_host"]
    G, H, d = c["H_q"] // c["H_kv"], c["H_kv"], c["d"]
    o, lse = torch.empty_like(st["q"]), torch.empty_like(st["lse"])
    # all single tokens at once, each longer chunk by itself
    single = [s for s in range(c["B"]) if new[s] == 1]
    groups = ([single] if single else []) + [[s] for s in range(c["B"]) if new[s] > 1]
    for g in groups:
        R = new[g[0]]
        n = max(st["ctx"][s] + R for s in g)
        every = len(g) == c["B"]
        requests = slice(None) if every else _ints(g).long()
        rows = slice(0, st["T"]) if every else slice(cu[g[0]], cu[g[0]] + R) if len(g) == 1 else _ints([cu[s] for s in g]).long()
        q = st["q"][rows].float().view(len(g), R, H, G, d)
        a, b = _plain_rows_of(st, requests, q, st["lens"][requests], n)
        o[rows], lse[rows] = a.reshape(-1, c["H_q"], d).to(o.dtype), b.reshape(-1, c["H_q"])
    return o, lse


def _plain_gather(st):
    page = st["case"]["page"]
    n = st["out_K"].shape[2]
    col = torch.arange(n, device="cuda")
    pages = st["table"].long().clamp(min=0)
    at = (col // page).clamp(max=pages.shape[1] - 1)
    there = (col < st["kv_lens"][:, None])[:, None, :, None]
    K = st["K"][pages[:, at], col % page].transpose(1, 2)
    V = st["V"][pages[:, at], col % page].transpose(1, 2)
    return torch.where(there, K, st["out_K"]), torch.where(there, V, st["out_V"])


# ---- the attention from its definition, in 64 bits ---------------------------------------------------

def exact(case, seed):
    """o = sum_k p_k V[k], p_k = exp(q . K[k] / sqrt(d) - lse), lse = ln sum_k exp(q . K[k] / sqrt(d)), the
    sums over the keys max(0, t - window + 1) .. t of a row at position t; request by request, KV head by
    KV head, some rows at a time.  The other passes compute no numbers: they place and copy."""
    c = case
    if c["kind"] != "attend" or work(c)["flops"] > 6e12:
        return None
    ctx, new, _ = _lengths(c)
    st = prepare(c, seed)
    G, d = c["H_q"] // c["H_kv"], c["d"]
    o = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for s in range(c["B"]):
        total = ctx[s] + new[s]
        pages = st["table"][s, :_pages(total, c["page"])].long()
        for h in range(c["H_kv"]):
            K = st["K"][pages, :, h].reshape(-1, d)[:total].double()
            V = st["V"][pages, :, h].reshape(-1, d)[:total].double()
            for i in range(0, new[s], 1024):
                r = min(1024, new[s] - i)
                hi = ctx[s] + i + r
                lo = max(0, ctx[s] + i + 1 - c["window"]) if c["window"] else 0
                q = st["q"][row + i:row + i + r, h * G:(h + 1) * G].double()
                x = torch.matmul(q, K[lo:hi].T) / math.sqrt(d)
                t = ctx[s] + i + torch.arange(r, device="cuda")[:, None]
                k = torch.arange(lo, hi, device="cuda")[None]
                hide = (k > t) | ((k + c["window"] <= t) if c["window"] else torch.zeros_like(k, dtype=torch.bool))
                x.masked_fill_(hide[:, None], float("-inf"))
                z = torch.logsumexp(x, dim=-1)
                o[row + i:row + i + r, h * G:(h + 1) * G] = torch.matmul(torch.exp(x - z[..., None]), V[lo:hi])
                lse[row + i:row + i + r, h * G:(h + 1) * G] = z
        row += new[s]
    return o, lse

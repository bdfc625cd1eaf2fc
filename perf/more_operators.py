"""Paged caches held in eight bits, and attention of batches that share a prefix, as cases that can be timed and compared.

A serving program that keeps its FULL layers' caches, or its prompts before the eviction, in half the memory
holds them as e4m3 codes with a power of two per row: ``kvev_paged_q8_*``.  One whose requests begin with the
same tokens holds those tokens' pages once and attends to them once for all: ``kvev_paged_attention_shared``.
The passes here are the ones it makes of them, one layer each:

* ``q_write``   the new tokens' K/V rows are quantised into their slots;
* ``q_gather``  the pages of whole prompts are read back as the contiguous caches that the eviction reads;
* ``q_attend``  attention of the new tokens over quantised pages: output rows and their log-sum-exp;
* ``shared``    attention of the new tokens of groups of requests, each group's first tokens in common pages.

A row x (one token's d elements of one KV head) is held as codes c and a byte b standing for 2^(b - 127):
with a the largest magnitude, e the smallest whole number with a <= 448 2^e (within the type's limits),
b = e + 127 and c = e4m3(x 2^-e), rounded to nearest, ties to even.

A case is a dict of plain values.  ``prepare`` makes what the program has in hand before the call, ``run``
makes one pass, ``exact`` gives the numbers from their definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

SINK = 4          # leading positions with raised logits (attention sinks)
SINK_LOGIT = 5.0

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
# the least and the largest exponent of a row, and the largest code at the latter (the next one is past the type)
EXPONENTS = {"bf16": (-120, 120), "fp16": (-15, 8)}
TOP_CODE, LAST_CODE = 448.0, 240.0
E4M3 = torch.float8_e4m3fn


def _case(name, kind, B, new_lo, new_hi, ctx_lo, ctx_hi, chunks, page, H_q=32, H_kv=8, d=128, dtype="bf16", heads_first=False,
          window=0, shared=0, groups=1):
    """B requests with ctx_lo..ctx_hi tokens of their own in the cache; `chunks` of them bring new_lo..new_hi
    new tokens, the others one (``q_gather``: none).  heads_first: pages are [H_kv][page][d], else
    [page][H_kv][d].  window: sliding window, 0 = none.  shared: about so many tokens before each request's own
    are those of its group, one of `groups`."""
    return {"name": name, "kind": kind, "B": B, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo, "ctx_hi": ctx_hi,
            "chunks": chunks, "page": page, "H_q": H_q, "H_kv": H_kv, "d": d, "dtype": dtype, "heads_first": heads_first,
            "window": window, "shared": shared, "groups": groups}


def listed():
    return [
        # One generated token of sixteen requests: latency.
        _case("q_write_b16", "q_write", 16, 1, 1, 1000, 16384, 0, 16),
        # Four prompts' chunks of up to 4,096 tokens.
        _case("q_write_16k", "q_write", 4, 4000, 4096, 0, 8192, 4, 16),
        # One 8K prompt handed to the eviction, half precision, pages with heads first.
        _case("q_gather_8k", "q_gather", 1, 0, 0, 8191, 8191, 0, 64, dtype="fp16", heads_first=True),
        # Eight ragged prompts of 16K to 32K handed over, the benchmark's headline batch.
        _case("q_gather_b8_long", "q_gather", 8, 0, 0, 16384, 32768, 0, 16),
        # One generation at a 4K context: the smallest attention call, where latency counts.
        _case("q_decode_b1_4k", "q_attend", 1, 1, 1, 4095, 4095, 0, 16),
        # The benchmark's decode batch before its caches are compacted: 16 requests at 16K.
        _case("q_decode_b16_16k", "q_attend", 16, 1, 1, 16384, 16384, 0, 64, heads_first=True),
        # Many ragged generations in half precision, 64-wide heads.
        _case("q_decode_b64_ragged", "q_attend", 64, 1, 1, 200, 8192, 0, 16, d=64, dtype="fp16"),
        # The last chunk of a 32K prompt.
        _case("q_chunk_4k_of_32k", "q_attend", 1, 4096, 4096, 28672, 28672, 1, 128, heads_first=True),
        # A few answers sampled for one question of 2,000 tokens or so: the smallest group.
        _case("shared_b4_2k", "shared", 4, 1, 1, 10, 200, 0, 16, shared=2000),
        # A server whose requests all begin with the same 8K of instructions and tools.
        _case("shared_b64_8k", "shared", 64, 1, 1, 16, 1500, 0, 16, shared=8192),
        # Two tenants' instructions, half precision, 64-wide heads, ragged generations behind them.
        _case("shared_b96_2_groups", "shared", 96, 1, 1, 0, 700, 0, 32, d=64, dtype="fp16", heads_first=True, shared=5000, groups=2),
        # New prompts prefilled behind a 16K document, beside generations about it.
        _case("shared_chunks_16k", "shared", 12, 300, 700, 0, 900, 6, 64, shared=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: batches of 1 to 128, contexts and prefixes to 32K, chunks to 4K, pages
    of 16 to 128, groups of 1 to 16 heads, both head sizes, types and page layouts, windows."""
    kind = rng.choice(["q_attend", "q_attend", "q_attend", "shared", "shared", "shared", "q_write", "q_gather"])
    H_q, H_kv = rng.choice([(32, 8), (32, 8), (8, 8), (16, 8), (64, 8), (4, 2), (8, 2), (32, 2), (12, 4), (14, 2)])
    geo = {"H_q": H_q, "H_kv": H_kv, "d": rng.choice([128, 128, 64]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
           "page": rng.choice([16, 16, 32, 64, 128]), "heads_first": rng.random() < 0.4}
    ctx_hi = _log_int(rng, 1, 32768)
    ctx_lo = rng.choice([0, ctx_hi // 4, ctx_hi // 2, ctx_hi])
    if kind == "q_write":
        B = _log_int(rng, 1, 64)
        hi = max(1, min(_log_int(rng, 1, 4096), 16384 // B))
        c = _case("", kind, B, max(1, hi // 3), hi, 0, min(ctx_hi, 131072 // B), B, **geo)
    elif kind == "q_gather":
        c = _case("", kind, rng.choice([1, 1, 2, 3, 5, 8]), 0, 0, ctx_lo, ctx_hi, 0, **geo)
    elif kind == "shared":
        groups = rng.choice([1, 1, 1, 2, 3, 5])
        B = groups - 1 + _log_int(rng, 1, 124)
        shared = _log_int(rng, 64, 32768)
        own_hi = min(_log_int(rng, 1, 2048), max(1, 524288 // B - shared // 2))
        shared = max(16, min(shared, 1048576 // B))
        if rng.random() < 0.7:  # generations
            c = _case("", kind, B, 1, 1, rng.choice([0, own_hi // 2]), own_hi, 0, shared=shared, groups=groups, **geo)
        else:                   # chunks behind the prefix, some beside generations
            chunks = min(B, rng.choice([1, 2, 4]))
            B = min(B, chunks + rng.choice([0, 4, 12]))
            hi = max(2, _log_int(rng, 2, 2048) // chunks)
            c = _case("", kind, max(B, groups), max(1, hi // 2), hi, 0, min(own_hi, 4096), chunks, shared=min(shared, 24576), groups=groups, **geo)
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

def _pages(n, page):
    return -(-n // page)


def _lengths(c):
    """(tokens in the cache before, new tokens) of each request, (first request, shared tokens) of each group:
    whole pages of them, counted in the requests' tokens."""
    r = random.Random("%(B)d/%(new_lo)d/%(new_hi)d/%(ctx_lo)d/%(ctx_hi)d/%(chunks)d/%(shared)d/%(groups)d" % c)
    ctx = [r.randint(c["ctx_lo"], c["ctx_hi"]) for _ in range(c["B"])]
    new = [0 if c["kind"] == "q_gather" else 1] * c["B"]
    for s in r.sample(range(c["B"]), c["chunks"]):
        new[s] = r.randint(c["new_lo"], c["new_hi"])
    groups = []
    if c["kind"] == "shared":
        first = [0] + sorted(r.sample(range(1, c["B"]), c["groups"] - 1))
        for g, a in enumerate(first):
            b = first[g + 1] if g + 1 < len(first) else c["B"]
            n = r.randint(3 * c["shared"] // 4, c["shared"]) // c["page"] * c["page"] if g else c["shared"] // c["page"] * c["page"]
            groups.append((a, n))
            for s in range(a, b):
                ctx[s] += n
    return ctx, new, groups


def _shared_of(c):
    """Each request's shared tokens."""
    groups = _lengths(c)[2]
    out = [0] * c["B"]
    for g, (a, n) in enumerate(groups):
        for s in range(a, groups[g + 1][0] if g + 1 < len(groups) else c["B"]):
            out[s] = n
    return out


def _seen(c):
    """(key positions that the rows see, a group's shared ones counted once; (query, key) pairs) over the requests."""
    ctx, new, groups = _lengths(c)
    keys, pairs = sum(n for _, n in groups), 0
    for n, q, m in zip(ctx, new, _shared_of(c)):
        w = c["window"] or n + q
        keys += n + q - max(m, n + 1 - w, 0)
        # row at position t sees min(t + 1, w) keys
        a, b = min(max(w - 1 - n, 0), q), q
        pairs += sum((n + 1, n + a)) * a // 2 + (b - a) * w
    return keys, pairs


def work(case):
    """Bytes and operations that a pass cannot do without."""
    c = case
    ctx, new, _ = _lengths(c)
    T = sum(new)
    row, coded = c["H_kv"] * c["d"] * 2, c["H_kv"] * (c["d"] + 1)
    if c["kind"] == "q_write":
        return {"bytes": 2 * T * (row + coded) + 4 * T, "flops": 0}
    if c["kind"] == "q_gather":
        return {"bytes": 2 * sum(ctx) * (row + coded) + 4 * sum(_pages(n, c["page"]) for n in ctx), "flops": 0}
    keys, pairs = _seen(c)
    qo = 2 * T * c["H_q"] * c["d"] * 2 + 4 * T * c["H_q"]
    return {"bytes": 2 * keys * (row if c["kind"] == "shared" else coded) + qo + 4 * _pages(keys, c["page"]),
            "flops": 4 * c["d"] * c["H_q"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 131 + what)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(c, seed):
    """A block table whose requests hold their pages scattered over the pool, a group's shared ones in common."""
    ctx, new, groups = _lengths(c)
    after = [_pages(n + q, c["page"]) for n, q in zip(ctx, new)]
    common = [n // c["page"] for n in _shared_of(c)]
    total = sum(a - m for a, m in zip(after, common)) + sum(n // c["page"] for _, n in groups) + 3
    perm = torch.randperm(total, generator=_gen(seed, 1), device="cuda").to(torch.int32)
    width = max(1, max(after))
    col = torch.arange(width, device="cuda")
    own_n, m = _ints([a - b for a, b in zip(after, common)]).long(), _ints(common).long()
    at = (own_n.cumsum(0) - own_n)[:, None] + col - m[:, None]
    if groups:
        of = torch.searchsorted(_ints([a for a, _ in groups]), torch.arange(c["B"], device="cuda"), right=True) - 1
        n = _ints([n // c["page"] for _, n in groups]).long()
        first = int(own_n.sum()) + n.cumsum(0) - n
        at = torch.where(col < m[:, None], first[of][:, None] + col, at)
    table = torch.where(col < (own_n + m)[:, None], perm[at.clamp(0, total - 1)], -1).to(torch.int32)
    return table, total


def _rows_of_pool(c, seed, pages, what):
    """A layer's pages of 16-bit rows, seen as [pages][page][H_kv][d] whatever their order in memory."""
    H, p, d = c["H_kv"], c["page"], c["d"]
    shape = (pages, H, p, d) if c["heads_first"] else (pages, p, H, d)
    x = torch.randn(shape, generator=_gen(seed, what), device="cuda", dtype=DTYPES[c["dtype"]])
    return x.transpose(1, 2) if c["heads_first"] else x


def _quantised(x, dtype):
    """(e4m3 codes, bytes of the rows' exponents) of rows x [...][d] in 32 bits."""
    lo, hi = EXPONENTS[dtype]
    m, k = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(m == 0, lo, k - 9 + (m > 0.875).to(k.dtype)).clamp(lo, hi)
    top = torch.where(e == hi, LAST_CODE, TOP_CODE)
    y = torch.ldexp(x, -e)
    return torch.minimum(torch.maximum(y, -top), top).to(E4M3), (e + 127).squeeze(-1).to(torch.uint8)


def _quantised_pool(c, x):
    """The pool's rows as codes in the same order of memory, and the exponents' bytes [pages][H_kv][page]."""
    codes = torch.empty_like(x, dtype=torch.uint8)  # (keeps the strides)
    scale = torch.empty((x.shape[0], c["H_kv"], c["page"]), dtype=torch.uint8, device="cuda")
    for i in range(0, x.shape[0], 8192):
        y, b = _quantised(x[i:i + 8192].float(), c["dtype"])
        codes[i:i + 8192], scale[i:i + 8192] = y.view(torch.uint8), b.transpose(1, 2)
    return codes.view(E4M3), scale


def prepare(case, seed):
    c = case
    ctx, new, groups = _lengths(c)
    B, T, dt = c["B"], sum(new), DTYPES[c["dtype"]]
    st = {"case": c, "ctx": ctx, "new": new, "T": T, "lens": _ints(ctx)}
    st["table"], pages = _table(c, seed)
    K, V = _rows_of_pool(c, seed, pages, 2), _rows_of_pool(c, seed, pages, 3)
    st["kv_lens"] = _ints([n + q for n, q in zip(ctx, new)])
    cu = [0]
    for q in new:
        cu.append(cu[-1] + q)
    st["cu"], st["cu_host"] = _ints(cu), cu
    if c["kind"] == "q_write":
        t = torch.arange(T, device="cuda")
        s = torch.searchsorted(st["cu"][1:], t, right=True)
        pos = t - st["cu"][s] + st["lens"][s]
        st["slots"] = (st["table"][s, pos // c["page"]] * c["page"] + pos % c["page"]).to(torch.int32)
        # rows of a projection: magnitudes differ from head to head and from token to token
        for name, what in (("k", 4), ("v", 5)):
            x = torch.randn((T, c["H_kv"], c["d"]), generator=_gen(seed, what), device="cuda")
            st[name] = (x * torch.exp(torch.randn((T, c["H_kv"], 1), generator=_gen(seed, what + 8), device="cuda"))).to(dt)
    if c["kind"] == "q_gather":
        cap = max(1, -(-max(ctx) // 256) * 256)
        st["out_K"] = torch.zeros((B, c["H_kv"], cap, c["d"]), dtype=dt, device="cuda")
        st["out_V"] = torch.zeros_like(st["out_K"])
    if c["kind"] in ("q_attend", "shared"):
        # the queries of a KV head share a direction, and the first positions' keys lie along it
        G, H, d = c["H_q"] // c["H_kv"], c["H_kv"], c["d"]
        u = torch.randn((H, d), generator=_gen(seed, 6), device="cuda")
        u = u / u.norm(dim=1, keepdim=True)
        q = 1.5 * torch.randn((T, H, G, d), generator=_gen(seed, 7), device="cuda") + math.sqrt(d) * u[None, :, None, :]
        st["q"] = q.to(dt).view(T, c["H_q"], d)
        heads = [a for a, n in groups if n] + [s for s, m in enumerate(_shared_of(c)) if not m]  # a request of each set of pages
        t = torch.arange(SINK, device="cuda").expand(len(heads), SINK)
        page = st["table"][_ints(heads).long()[:, None], t // c["page"]].long().clamp(min=0)
        K[page, t % c["page"]] += (SINK_LOGIT * u).to(dt)
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((T, c["H_q"]), dtype=torch.float32, device="cuda")
    if c["kind"] == "shared":
        st["K"], st["V"] = K, V
        st["groups"], st["shared"] = _ints([a for a, _ in groups] + [B]), _ints([n for _, n in groups])
    else:
        st["K"], st["K_scale"] = _quantised_pool(c, K)
        st["V"], st["V_scale"] = _quantised_pool(c, V)
    if own:  # the handle a serving program keeps
        from paper_2606_15157_gb300 import paged
        if c["kind"] == "shared":
            st["cache"] = paged.PagedCache(st["K"], st["V"], st["table"])
        else:
            st["cache"] = paged.QuantizedCache(st["K"], st["V"], st["K_scale"], st["V_scale"], st["table"], dtype=dt)
    return st


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"q_write": _own_write, "q_gather": _own_gather, "q_attend": _own_attend, "shared": _own_shared}[kind](state)
    return {"q_write": _plain_write, "q_gather": _plain_gather, "q_attend": _plain_attend, "shared": _plain_attend}[kind](state)


def _own_write(st):
    st["cache"].write(st["k"], st["v"], st["slots"])
    return st["K"], st["V"], st["K_scale"], st["V_scale"]


def _own_gather(st):
    st["cache"].gather(st["kv_lens"], st["out_K"], st["out_V"])
    return st["out_K"], st["out_V"]


def _own_attend(st):
    st["cache"].attention(st["q"], st["cu"], st["kv_lens"], window=st["case"]["window"], out=st["o"], lse=st["lse"])
    return st["o"], st["lse"]


def _own_shared(st):
    st["cache"].attention_shared(st["q"], st["cu"], st["kv_lens"], st["groups"], st["shared"], out=st["o"], lse=st["lse"])
    return st["o"], st["lse"]


def _plain_write(st):
    page, slots = st["case"]["page"], st["slots"].long()
    for x, pool, scale in ((st["k"], st["K"], st["K_scale"]), (st["v"], st["V"], st["V_scale"])):
        codes, b = _quantised(x.float(), st["case"]["dtype"])
        pool.view(torch.uint8)[slots // page, slots % page] = codes.view(torch.uint8)
        scale.transpose(1, 2)[slots // page, slots % page] = b
    return st["K"], st["V"], st["K_scale"], st["V_scale"]


def _plain_values(st, name, pages):
    """The values of whole pages in 32 bits, [...][page][H_kv][d]."""
    x = st[name]
    if st["case"]["kind"] == "shared":
        return x[pages].float()
    b = st[name + "_scale"].transpose(1, 2)[pages]
    return torch.ldexp(x.view(torch.uint8)[pages].view(E4M3).float(), b[..., None].to(torch.int32) - 127)


def _plain_gather(st):
    page, dt = st["case"]["page"], st["out_K"].dtype
    n = st["out_K"].shape[2]
    col = torch.arange(n, device="cuda")
    pages = st["table"].long().clamp(min=0)
    there = (col < st["kv_lens"][:, None])[:, None, :, None]
    out = []
    for name in ("K", "V"):
        x = _plain_values(st, name, pages).to(dt).flatten(1, 2)
        x = x[:, col.clamp(max=x.shape[1] - 1)].transpose(1, 2)
        out.append(torch.where(there, x, st["out_" + name]))
    return tuple(out)


def _plain_rows(st, name, requests, n):
    """The first n rows of the requests' pages in 32 bits, [request][H_kv][n][d]; rows past a request's end are 0."""
    c = st["case"]
    pages = st["table"][requests, :_pages(n, c["page"])].long().clamp(min=0)
    x = _plain_values(st, name, pages).flatten(1, 2)[:, :n].transpose(1, 2)
    there = torch.arange(n, device="cuda") < st["kv_lens"][requests, None]
    return torch.where(there[:, None, :, None], x, 0.0)


def _plain_rows_of(st, requests, q, first, n):
    """Attention of q [request][row][H_kv][G][d] (32 bits), rows at positions first + i, over n keys."""
    c = st["case"]
    K, V = _plain_rows(st, "K", requests, n), _plain_rows(st, "V", requests, n)
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


# ---- the numbers from their definition, in 64 bits ---------------------------------------------------

def _exact_values(st, name, pages, h):
    """The values of a KV head's rows in those pages, [rows][d]."""
    x = st[name]
    if st["case"]["kind"] == "shared":
        return x[pages, :, h].double().flatten(0, 1)
    codes = x.view(torch.uint8)[pages, :, h].view(E4M3).double()
    return (codes * torch.exp2(st[name + "_scale"][pages, h].double() - 127)[..., None]).flatten(0, 1)


def _exact_write(c, st):
    """Codes and exponents of the new rows, each exponent found by comparing with every 448 2^e."""
    lo, hi = EXPONENTS[c["dtype"]]
    e = torch.arange(lo, hi + 1, dtype=torch.float64, device="cuda")
    # the codes of e4m3 that are not negative, in order; a value between two goes to the nearer, in the middle to the even one
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(E4M3).double()
    page, slots = c["page"], st["slots"].long()
    out = []
    for x, pool, scale in ((st["k"], st["K"], st["K_scale"]), (st["v"], st["V"], st["V_scale"])):
        values = pool.double()
        scales = scale.double()
        for i in range(0, st["T"], 4096):
            y, s = x[i:i + 4096].double(), slots[i:i + 4096]
            n = torch.searchsorted(448 * torch.exp2(e), y.abs().amax(-1)).clamp(max=e.numel() - 1)
            y = y * torch.exp2(-e[n])[..., None]
            y = torch.minimum(y.abs(), torch.where(e[n] == hi, 240.0, 448.0)[..., None].double()) * torch.sign(y)
            j = torch.searchsorted(codes, y.abs().contiguous()).clamp(1, 126)
            below, above = y.abs() - codes[j - 1], codes[j] - y.abs()
            j = torch.where((below < above) | ((below == above) & (j % 2 == 1)), j - 1, j)
            values[s // page, s % page] = codes[j] * torch.sign(y)
            scales.transpose(1, 2)[s // page, s % page] = e[n] + 127
        out.append((values, scales))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def exact(case, seed):
    """``q_attend``, ``shared``: o = sum_k p_k V[k], p_k = exp(q . K[k] / sqrt(d) - lse), lse = ln sum_k exp(q . K[k] /
    sqrt(d)), the sums over the keys max(0, t - window + 1) .. t of a row at position t and the values that the
    pages stand for; request by request, KV head by KV head, some rows at a time.  ``q_write``: the rows' codes
    and exponents.  ``q_gather``: what the codes stand for."""
    c = case
    if c["kind"] in ("q_attend", "shared") and work(c)["flops"] > 6e12:
        return None
    ctx, new, _ = _lengths(c)
    st = prepare(c, seed)
    if c["kind"] == "q_write":
        return _exact_write(c, st)
    if c["kind"] == "q_gather":
        out = []
        for name in ("K", "V"):
            x = torch.zeros(st["out_K"].shape, dtype=torch.float64, device="cuda")
            for s in range(c["B"]):
                pages = st["table"][s, :_pages(ctx[s], c["page"])].long()
                for h in range(c["H_kv"]):
                    x[s, h, :ctx[s]] = _exact_values(st, name, pages, h)[:ctx[s]]
            out.append(x)
        return tuple(out)
    G, d = c["H_q"] // c["H_kv"], c["d"]
    o = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for s in range(c["B"]):
        total = ctx[s] + new[s]
        pages = st["table"][s, :_pages(total, c["page"])].long()
        for h in range(c["H_kv"]):
            K, V = _exact_values(st, "K", pages, h)[:total], _exact_values(st, "V", pages, h)[:total]
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

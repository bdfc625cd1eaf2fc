"""The paged cache on the GPU: tables, release, write, gather and attention against their plain forms."""
import math
import random

import pytest
import torch

from paper_2606_15157_gb300 import kvev
from tests import paged_ref as ref

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def paged():
    from paper_2606_15157_gb300 import build, paged
    build.build()
    return paged


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def host(t):
    return t.cpu().tolist()


# ---- tables and release -----------------------------------------------------------------------------

def pool_state(rng, lens, page, num_pages, max_pages, rows):
    """Requests holding their pages, scattered; (table, free stack, count) as host lists."""
    perm = list(range(num_pages))
    rng.shuffle(perm)
    table, at = [[-1] * max_pages for _ in range(rows)], 0
    for s, n in enumerate(lens):
        k = ref.pages_of(n, page)
        table[s][:k] = perm[at:at + k]
        at += k
    free = perm[at:] + [-1] * at
    return table, free, num_pages - at


@pytest.mark.parametrize("B,page,ctx,new,share", [
    (1, 16, 0, 1, 1.0), (1, 8, 40, 1, 1.0), (3, 16, 100, 40, 1.0), (17, 32, 500, 3, 1.0), (64, 16, 1000, 1, 1.0),
    (64, 16, 1000, 200, 0.5), (256, 256, 5000, 300, 0.7), (1023, 16, 90, 3, 1.0), (1025, 16, 90, 3, 0.6), (5000, 8, 20, 2, 0.9),
    (2, 128, 9000, 9000, 1.0), (40, 64, 0, 64, 0.0)])
def test_tables_match_plain(paged, B, page, ctx, new, share):
    rng = random.Random(f"{B}/{page}/{ctx}/{new}")
    lens = [rng.choice([0, rng.randint(0, ctx), page * (ctx // page)]) for _ in range(B)]
    q = [rng.choice([0, 1, rng.randint(0, new)]) for _ in range(B)]
    need = sum(ref.pages_of(n + k, page) - ref.pages_of(n, page) for n, k in zip(lens, q))
    held = sum(ref.pages_of(n, page) for n in lens)
    num_pages = max(1, held + int(need * share) + (3 if share >= 1 else 0))
    max_pages = ref.pages_of(ctx + new, page) + 1
    table, free, count = pool_state(rng, lens, page, num_pages, max_pages, B)
    T = sum(q) + rng.choice([0, 5])
    dtab = ints(table)
    pool = paged.PagePool(num_pages, page, dtab, ints(free), ints([count]))
    dlens = ints(lens)
    kv, cu, slots, pos, granted = pool.tables(dlens, ints(q), T, kv_lens=dlens)  # lengths and count in place
    want = ref.tables(lens, q, page, num_pages, free, count, table, max_pages, T)
    assert host(dlens) == want[0] and host(cu) == want[1] and host(granted) == want[4]
    assert host(slots) == want[2] and host(pos) == want[3]
    assert host(dtab) == table and host(pool.free_count) == [want[5]]
    assert int(pool.device_status) == 0
    # the same call with outputs of its own changes none of the inputs
    pool2 = paged.PagePool(num_pages, page, dtab, ints(free), ints([count]))
    out = torch.empty(1, dtype=torch.int32, device="cuda")
    l0 = ints(lens)
    pool2.tables(l0, ints(q), T, free_count_out=out)
    assert host(l0) == lens and host(pool2.free_count) == [count] and host(out) == [want[5]] and host(dtab) == table


@pytest.mark.parametrize("B,page,ctx", [(1, 16, 33), (16, 16, 3000), (300, 8, 200), (1500, 32, 100)])
def test_release_matches_plain(paged, B, page, ctx):
    rng = random.Random(B)
    lens = [rng.choice([0, rng.randint(0, ctx)]) for _ in range(B)]
    done = [rng.choice([0, 0, 1, -3]) for _ in range(B)]
    num_pages, max_pages = sum(ref.pages_of(n, page) for n in lens) + 7, ref.pages_of(ctx, page) + 1
    table, free, count = pool_state(rng, lens, page, num_pages, max_pages, B)
    pool = paged.PagePool(num_pages, page, ints(table), ints(free), ints([count]))
    dlens = ints(lens)
    pool.release(dlens, ints(done))
    want, c = ref.release(lens, done, page, num_pages, free, count, table)
    assert host(dlens) == want and host(pool.free_count) == [c] and host(pool.free)[:c] == free[:c]
    assert int(pool.device_status) == 0
    # and what is released is given out again
    q = [rng.randint(0, 2 * page) for _ in range(B)]
    T = sum(q)
    pool.tables(dlens, ints(q), T, kv_lens=dlens)
    w2 = ref.tables(want, q, page, num_pages, free, c, table, max_pages, T)
    assert host(dlens) == w2[0] and host(pool.block_table) == table


def test_tables_flag_what_is_out_of_range(paged):
    table = ints([[0, -1], [5, 99]])
    pool = paged.PagePool(8, 16, table, ints([1, 2, 3, 4, 6, 7, -1, -1]), ints([6]))
    # a negative length and a request past the table's width
    kv, cu, slots, pos, granted = pool.tables(ints([-4, 16]), ints([2, 40]), 42)
    assert host(kv) == [2, 16] and host(cu) == [0, 2, 42] and host(granted) == [1, 0]
    assert host(slots)[:2] == [7 * 16, 7 * 16 + 1] and host(slots)[2:] == [-1] * 40
    assert int(pool.device_status) == 2
    pool.device_status.zero_()
    # a held page outside the pool
    kv, cu, slots, pos, granted = pool.tables(ints([0, 20]), ints([0, 2]), 2)
    assert host(slots) == [-1, -1] and int(pool.device_status) == 2
    pool.device_status.zero_()
    # more tokens than rows
    _, cu, slots, _, _ = pool.tables(ints([0, 0]), ints([3, 4]), 5)
    assert host(cu) == [0, 3, 7] and min(host(slots)) >= 0 and int(pool.device_status) == 2
    pool.device_status.zero_()
    # a stack that would overflow
    pool.release(ints([16, 20]), ints([1, 1]))
    assert int(pool.device_status) == 2 and host(pool.free_count)[0] <= 8


# ---- write and gather ---------------------------------------------------------------------------------

def make_cache(paged, pages, page, H, d, table, dtype, heads_first, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = paged.PagedCache.empty(pages, page, H, d, table, dtype, heads_first)
    for x in (c.K, c.V):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float32))
    return c


@pytest.mark.parametrize("T,H,d,page,dtype,heads_first", [
    (1, 8, 128, 16, BF16, False), (1, 1, 64, 8, FP16, True), (17, 3, 128, 32, BF16, True), (300, 2, 64, 128, BF16, False),
    (5000, 8, 128, 16, FP16, True), (4097, 5, 128, 256, BF16, False)])
def test_write_matches_plain(paged, T, H, d, page, dtype, heads_first):
    g = torch.Generator(device="cuda").manual_seed(T)
    pages = ref.pages_of(T, page) + 3
    table = ints([[0]])
    c = make_cache(paged, pages, page, H, d, table, dtype, heads_first)
    # k and v as slices of a fused projection
    qkv = torch.randn((T, 3, H, d), generator=g, device="cuda").to(dtype)
    k, v = qkv[:, 1], qkv[:, 2]
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T].to(torch.int32)
    if T > 2:
        slots[1] = -1
    K, V = c.K.clone(), c.V.clone()
    keep = (slots >= 0).nonzero().flatten()
    at = slots[keep].long()
    K[at // page, at % page], V[at // page, at % page] = k[keep], v[keep]
    c.write(k, v, slots)
    assert torch.equal(c.K, K) and torch.equal(c.V, V) and c.status() == 0


def test_write_skips_slots_past_the_pool(paged):
    c = make_cache(paged, 2, 16, 2, 64, ints([[0]]), BF16, False)
    K = c.K.clone()
    k = torch.ones((3, 2, 64), dtype=BF16, device="cuda")
    c.write(k, k, ints([32, -7, 2 ** 31 - 1]))
    assert torch.equal(c.K, K) and c.status() == 2 and c.status() == 0


@pytest.mark.parametrize("lens,H,d,page,dtype,heads_first,S_cap", [
    ([1], 8, 128, 16, BF16, False, 1), ([0, 5, 64], 2, 64, 32, FP16, True, 70), ([1000, 0, 313, 1024], 3, 128, 8, BF16, False, 1024),
    ([2000, 1999], 8, 128, 256, BF16, True, 2048), ([500, 31, 32, 33], 1, 64, 64, FP16, False, 512)])
def test_gather_matches_plain(paged, lens, H, d, page, dtype, heads_first, S_cap):
    rng = random.Random(page)
    num_pages = sum(ref.pages_of(n, page) for n in lens) + 2
    table, _, _ = pool_state(rng, lens, page, num_pages, ref.pages_of(S_cap, page), len(lens))
    c = make_cache(paged, num_pages, page, H, d, ints(table), dtype, heads_first)
    oK = torch.full((len(lens), H, S_cap, d), 7.0, dtype=dtype, device="cuda")
    oV = oK.clone()
    wK, wV = oK.clone(), oV.clone()
    for s, n in enumerate(lens):
        p = torch.tensor(table[s][:ref.pages_of(n, page)], dtype=torch.long, device="cuda")
        wK[s, :, :n] = c.K[p].flatten(0, 1)[:n].transpose(0, 1)
        wV[s, :, :n] = c.V[p].flatten(0, 1)[:n].transpose(0, 1)
    c.gather(ints(lens), oK, oV)
    assert torch.equal(oK, wK) and torch.equal(oV, wV) and c.status() == 0


def test_gather_flags_what_is_out_of_range(paged):
    c = make_cache(paged, 4, 16, 1, 64, ints([[0, 9], [1, 2], [3, -1]]), BF16, False)
    o = torch.zeros((3, 1, 24, 64), dtype=BF16, device="cuda")
    oV = torch.zeros_like(o)
    c.gather(ints([20, 40, -3]), o, oV)
    assert c.status() == 2
    assert torch.equal(o[0, 0, :16], c.K[0, :, 0]) and not o[0, 0, 16:].any()  # page 9 is left out
    assert torch.equal(o[1, 0, :16], c.K[1, :, 0]) and torch.equal(o[1, 0, 16:], c.K[2, :8, 0]) and not o[2].any()


# ---- attention --------------------------------------------------------------------------------------

def attend_case(paged, reqs, H_q, H, d, page, dtype, heads_first, window=0, scale=0.0, junk=None, seed=0, q_gain=1.5):
    """reqs: [(kv length, new rows)].  Returns (cache, q, cu, kv, table)."""
    rng = random.Random(f"{reqs[:8]}/{page}/{seed}")
    kv, q_len = [r[0] for r in reqs], [r[1] for r in reqs]
    num_pages = sum(ref.pages_of(n, page) for n in kv) + 3
    table, _, _ = pool_state(rng, kv, page, num_pages, max(1, max(ref.pages_of(n, page) for n in kv)) + 1, len(reqs))
    c = make_cache(paged, num_pages, page, H, d, ints(table), dtype, heads_first, seed)
    cu = [0]
    for n in q_len:
        cu.append(cu[-1] + n)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (q_gain * torch.randn((max(cu[-1], 1), H_q, d), generator=g, device="cuda")).to(dtype)[:cu[-1]]
    if junk is not None:  # everything that no row may see
        dead = torch.ones(c.K.shape[:2], dtype=torch.bool, device="cuda")
        for s, (n, m) in enumerate(reqs):
            lo = max(0, n - m + 1 - window) if window else 0
            for k in range(lo if m else n, n):
                dead[table[s][k // page], k % page] = False
        c.K[dead], c.V[dead] = junk, junk
    return c, q, cu, kv, table


def run_attention(c, q, cu, kv, **kw):
    lse = torch.full((q.shape[0], q.shape[1]), 77.0, device="cuda")
    o = c.attention(q, ints(cu), ints(kv), lse=lse, **kw)
    return o, lse


def check(paged, reqs, H_q, H, d, page, dtype=BF16, heads_first=False, window=0, scale=0.0, **kw):
    c, q, cu, kv, table = attend_case(paged, reqs, H_q, H, d, page, dtype, heads_first, window, scale, **kw)
    o, lse = run_attention(c, q, cu, kv, window=window, scale=scale)
    assert c.status() == 0
    ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv, scale, window), dtype)
    o2, lse2 = run_attention(c, q, cu, kv, window=window, scale=scale)  # the same bits again
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


SINGLE = [(n, 1) for n in (1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 5000)]


@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (32, 8, 128, 64, FP16, True), (8, 8, 64, 8, BF16, False), (16, 2, 64, 128, FP16, True),
    (7, 1, 128, 256, BF16, True), (10, 2, 128, 32, BF16, False), (128, 1, 128, 16, FP16, False), (96, 1, 64, 16, BF16, True),
    (1, 1, 128, 16, BF16, False)])
def test_attention_single_tokens(paged, H_q, H, d, page, dtype, heads_first):
    check(paged, SINGLE, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("reqs", [
    [(1, 1)], [(4095, 1)], [(20011, 1)], [(300, 2), (2, 2), (33, 33)], [(128, 128)], [(129, 129)], [(700, 1), (700, 700), (3000, 13)],
    [(1000, 31), (1000, 32), (1000, 33), (64, 64), (65, 65)], [(2500, 257)], [(517, 500), (0, 0), (1, 1), (4000, 0), (260, 3)]],
    ids=lambda r: "_".join(f"{a}x{b}" for a, b in r))
@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (8, 2, 128, 16, BF16, False), (6, 2, 64, 32, FP16, True), (14, 2, 128, 64, BF16, True), (2, 2, 64, 128, BF16, False)])
def test_attention_chunks(paged, reqs, H_q, H, d, page, dtype, heads_first):
    check(paged, reqs, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000, 10 ** 9])
@pytest.mark.parametrize("H_q,H,d,page", [(8, 2, 128, 16), (5, 1, 64, 64)])
def test_attention_windows(paged, window, H_q, H, d, page):
    check(paged, [(1, 1), (900, 1), (900, 300), (2000, 140), (400, 400)], H_q, H, d, page, window=window)


@pytest.mark.parametrize("scale", [0.3, 1e-6])
def test_attention_scale(paged, scale):
    check(paged, [(500, 100), (77, 1)], 8, 4, 64, 16, scale=scale)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_attention_sharp_and_rising_rows(paged, dtype):
    # logits over a range of hundreds: the running maximum rises from tile to tile and weights underflow
    c, q, cu, kv, table = attend_case(paged, [(1500, 200), (3000, 1)], 8, 2, 128, 16, dtype, False, q_gain=8.0)
    ramp = torch.linspace(0.1, 3.0, c.K.shape[0] * c.K.shape[1], device="cuda").view(c.K.shape[0], c.K.shape[1], 1, 1)
    c.K.copy_((c.K.float() * ramp).to(dtype))
    o, lse = run_attention(c, q, cu, kv)
    ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv), dtype)


@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf, -3.3e38])
@pytest.mark.parametrize("window,heads_first", [(0, False), (50, True)])
def test_attention_ignores_what_no_row_sees(paged, junk, window, heads_first):
    check(paged, [(1, 1), (130, 3), (333, 333), (1000, 1), (45, 40), (600, 129)], 8, 2, 128, 16, BF16, heads_first,
          window=window, junk=junk)


def test_attention_masked_keys_of_a_row_may_be_the_lowest_value(paged):
    # keys that later rows see, with logits at the type's range, do not reach the rows before them
    c, q, cu, kv, table = attend_case(paged, [(64, 64)], 4, 1, 64, 16, BF16, False)
    c.K[table[0][3], 8:] = 1e36
    o, lse = run_attention(c, q, cu, kv)
    n = 48 + 8
    r = ref.attention(c.K, c.V, table, q[:n], [0, n], [n])
    ref.check_attention(o[:n], lse[:n], r, BF16)


def test_attention_empty_rows(paged):
    # more new rows than positions: rows before position 0 see no key
    c, q, cu, kv, table = attend_case(paged, [(300, 20)], 8, 2, 128, 16, BF16, False)
    reqs_kv, reqs_cu = [5, 0], [0, 12, 20]
    c2 = paged.PagedCache(c.K, c.V, c.block_table.repeat(2, 1))
    o, lse = run_attention(c2, q, reqs_cu, reqs_kv)
    assert c2.status() == 0
    ref.check_attention(o, lse, ref.attention(c.K, c.V, table * 2, q, reqs_cu, reqs_kv), BF16)
    assert not o[:7].any() and not o[12:].any() and torch.isinf(lse[:7]).all()


def test_attention_rows_past_the_last_are_left(paged):
    c, q, cu, kv, table = attend_case(paged, [(300, 20), (5, 1)], 8, 2, 128, 16, BF16, False)
    o = torch.full_like(q, 3.0)
    lse = torch.full((21, 8), 5.0, device="cuda")
    c.attention(q, ints([0, 11, 15]), ints([300, 5]), out=o, lse=lse)
    assert (o[15:] == 3).all() and (lse[15:] == 5).all() and c.status() == 0
    c.attention(q[:0], ints([0, 0, 0]), ints([300, 5]))
    assert c.status() == 0


def test_attention_strides(paged):
    # queries and outputs inside wider rows, heads of the pool inside a pool of two layers
    g = torch.Generator(device="cuda").manual_seed(5)
    page, H, d, H_q = 16, 2, 128, 6
    x = torch.randn((40, 2, page, 2, H, d + 8), generator=g, device="cuda").to(BF16)  # [page][layer][row][K, V][head]
    K, V = x[:, 1, :, 0, :, :d], x[:, 1, :, 1, :, 8:]
    table = [[7, 3, 39, 0, 12], [1, 2, 4, 5, 6]]
    wide = torch.randn((30, H_q + 2, 2, d), generator=g, device="cuda").to(BF16)
    q = wide[:, 1:-1, 1]
    out = torch.zeros((30, 2, H_q, d), dtype=BF16, device="cuda")
    c = paged.PagedCache(K, V, ints(table))
    cu, kv = [0, 29, 30], [70, 65]
    lse = torch.empty((30, H_q), device="cuda")
    o = c.attention(q, ints(cu), ints(kv), out=out[:, 1], lse=lse)
    assert o.data_ptr() == out[:, 1].data_ptr() and not out[:, 0].any() and c.status() == 0
    ref.check_attention(o, lse, ref.attention(K, V, table, q, cu, kv), BF16)


def test_attention_and_write_past_32_bit_offsets(paged):
    # pages over 4 G elements apart, rows over 2 G
    page, H, d = 16, 1, 64
    base = torch.zeros(3 * 2 ** 31 + 2 ** 16, dtype=BF16, device="cuda")
    K = torch.as_strided(base, (3, page, H, d), (2 ** 31, d, d, 1))
    V = torch.as_strided(base, (3, page, H, d), (2 ** 31, d, d, 1), 2 ** 15)
    table = [[2, 1, 0]]
    c = paged.PagedCache(K, V, ints(table))
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn((40, n, d), generator=g, device="cuda").to(BF16) for n in (1, 1, 4))
    slots = [table[0][t // page] * page + t % page for t in range(40)]
    c.write(k, v, ints(slots))
    o, lse = run_attention(c, q, [0, 40], [40])
    small = paged.PagedCache(K.clone(), V.clone(), ints(table))
    r = ref.attention(small.K, small.V, table, q, [0, 40], [40])
    ref.check_attention(o, lse, r, BF16)
    oK, oV = torch.zeros((1, 1, 48, d), dtype=BF16, device="cuda"), torch.zeros((1, 1, 48, d), dtype=BF16, device="cuda")
    c.gather(ints([40]), oK, oV)
    assert torch.equal(oK[0, 0, :40], k[:, 0]) and torch.equal(oV[0, 0, :40], v[:, 0]) and c.status() == 0


def test_attention_flags_what_is_out_of_range(paged):
    c, q, cu, kv, table = attend_case(paged, [(100, 4), (60, 4), (90, 2)], 4, 2, 64, 16, BF16, False)
    good = run_attention(c, q, cu, kv)
    for bad in ([100, -1, 90], [100, 10 ** 6, 90], [100, -2 ** 31, 90]):
        o, lse = run_attention(c, q, cu, bad)
        assert c.status() == 2
        for i in (0, 2):
            assert torch.equal(o[cu[i]:cu[i + 1]], good[0][cu[i]:cu[i + 1]])
    o, lse = run_attention(c, q, [0, 4, 2, 99], kv)
    assert c.status() == 2 and torch.equal(o[:4], good[0][:4])
    # pages outside the pool count as zero rows
    t2 = [list(r) for r in table]
    t2[0][1], t2[0][2] = -5, 10 ** 6
    c2 = paged.PagedCache(c.K, c.V, ints(t2))
    o, lse = run_attention(c2, q, cu, kv)
    assert c2.status() == 2 and torch.equal(o[4:], good[0][4:])
    Kz, Vz = c.K.clone(), c.V.clone()
    for j in (1, 2):
        Kz[table[0][j]], Vz[table[0][j]] = 0, 0
    ref.check_attention(o, lse, ref.attention(Kz, Vz, table, q, cu, kv), BF16)


def test_attention_on_another_stream_and_in_a_graph(paged):
    reqs = [(3000, 1), (100, 1), (1, 1)]
    c, q, cu, kv, table = attend_case(paged, reqs, 8, 2, 128, 16, BF16, False)
    dcu, dkv = ints(cu), ints(kv)
    lse = torch.empty((3, 8), device="cuda")
    o = torch.empty_like(q)
    s = torch.cuda.Stream()
    c.workspace(8, s)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c.attention(q, dcu, dkv, out=o, lse=lse)
    s.synchronize()
    ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv), BF16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.attention(q, dcu, dkv, out=o, lse=lse, stream=s)
    for kv2 in ([2999, 55, 1], [17, 16, 0], [3000, 100, 1]):  # replayed with other lengths
        dkv.copy_(ints(kv2))
        g.replay()
        torch.cuda.synchronize()
        ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv2), BF16)
    assert c.status() == 0


def test_attention_many_requests(paged):
    rng = random.Random(4)
    reqs = [(n, min(n, rng.choice([1, 1, 1, 2, 40]))) for n in (rng.randint(0, 400) for _ in range(700))]
    check(paged, reqs, 4, 2, 64, 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [31, 32, 33, 64, 383, 384, 385, 700])
def test_attention_batches_around_the_schedule_s_sizes(paged, B, d):
    # the schedule of a warp, of a block in one pass and in several, in both orders of units: requests
    # without rows (the first and last among them), single tokens, chunks, and contexts cut over many CTAs
    rng = random.Random(f"{B}/{d}")
    reqs = [(n, min(n, rng.choice([0, 1, 1, 1, 2, 40, 200]))) for n in (rng.randint(0, 400) for _ in range(B))]
    reqs[0], reqs[-1] = (50, 0), (0, 0)
    reqs[rng.randrange(1, B - 1)] = (9000, 1)
    reqs[rng.randrange(1, B - 1)] = (3000, 300)
    check(paged, reqs, 6, 3, d, 16)


def test_chunks_in_turn_equal_the_prompt_in_one(paged):
    """A ragged batch prefilled chunk by chunk through tables, write and attention against one causal pass."""
    H_q, H, d, page = 8, 2, 128, 16
    prompts = [700, 33, 260]
    g = torch.Generator(device="cuda").manual_seed(9)
    full = [tuple(torch.randn((n, h, d), generator=g, device="cuda").to(BF16) for h in (H_q, H, H)) for n in prompts]
    table = torch.full((3, 64), -1, dtype=torch.int32, device="cuda")
    pool = paged.PagePool(100, page, table)
    c = paged.PagedCache.empty(100, page, H, d, table)
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    got = [[], [], []]
    at = [0, 0, 0]
    while any(a < n for a, n in zip(at, prompts)):
        new = [min(130, n - a) for a, n in zip(at, prompts)]
        rows = [torch.cat([full[s][i][at[s]:at[s] + new[s]] for s in range(3)]) for i in range(3)]
        T = sum(new)
        _, cu, slots, pos, granted = pool.tables(lens, ints(new), T, kv_lens=lens)
        c.write(rows[1], rows[2], slots)
        o, lse = run_attention(c, rows[0], host(cu), host(lens))
        assert host(granted) == [1, 1, 1]
        row = 0
        for s in range(3):
            assert host(pos)[row:row + new[s]] == list(range(at[s], at[s] + new[s]))
            got[s].append((o[row:row + new[s]], lse[row:row + new[s]]))
            row += new[s]
            at[s] += new[s]
    for s, n in enumerate(prompts):
        Kp = torch.zeros((ref.pages_of(n, page), page, H, d), dtype=BF16, device="cuda")
        Vp = torch.zeros_like(Kp)
        Kp.view(-1, H, d)[:n], Vp.view(-1, H, d)[:n] = full[s][1], full[s][2]
        r = ref.attention(Kp, Vp, [list(range(len(Kp)))], full[s][0], [0, n], [n])
        ref.check_attention(torch.cat([a for a, _ in got[s]]), torch.cat([b for _, b in got[s]]), r, BF16)
    assert c.status() == 0 and int(pool.device_status) == 0
    pool.release(lens, ints([1, 1, 1]))
    assert host(pool.free_count) == [100] and sorted(host(pool.free)) == list(range(100))


# ---- what the tensor-level calls refuse ---------------------------------------------------------------

def test_refused_tensors(paged):
    table = ints([[0, 1], [2, 3]])
    pool = paged.PagePool(8, 16, table)
    c = paged.PagedCache.empty(8, 16, 2, 64, table)
    lens, i64 = ints([5, 6]), torch.zeros(2, dtype=torch.int64, device="cuda")
    k = torch.zeros((3, 2, 64), dtype=BF16, device="cuda")
    q = torch.zeros((3, 4, 64), dtype=BF16, device="cuda")
    cu, slots = ints([0, 1, 3]), ints([0, 1, 2])
    o = torch.zeros((2, 2, 32, 64), dtype=BF16, device="cuda")
    bad = [
        lambda: paged.PagedCache(c.K.cpu(), c.V.cpu(), table), lambda: paged.PagedCache(c.K, c.V[:, :8], table),
        lambda: paged.PagedCache(c.K.float(), c.V.float(), table), lambda: paged.PagedCache(c.K, c.V.half(), table),
        lambda: paged.PagedCache(c.K, c.V, table.long()), lambda: paged.PagedCache(c.K, c.V, table[:, :1]),
        lambda: paged.PagedCache(c.K.transpose(2, 3), c.V.transpose(2, 3), table),
        lambda: paged.PagePool(8, 16, table, ints([1, 2])), lambda: paged.PagePool(8, 16, table[0]),
        lambda: pool.tables(lens, i64, 3), lambda: pool.tables(lens, lens[:1], 3), lambda: pool.tables(ints([1, 2, 3]), ints([1, 1, 1]), 3),
        lambda: pool.tables(lens, lens, 3, slots=ints([0, 0])), lambda: pool.tables(lens, ints([1, 7, 2, 7])[::2], 3),
        lambda: pool.tables(lens.cpu(), lens, 3), lambda: pool.tables(lens, None, 3), lambda: pool.release(lens, i64),
        lambda: pool.release(lens, ints([1])), lambda: c.write(k, k[:2], slots), lambda: c.write(k, k, slots[:2]),
        lambda: c.write(k.half(), k.half(), slots), lambda: c.write(k[..., :32], k[..., :32], slots), lambda: c.write(q, q, slots),
        lambda: c.write(k, k.transpose(0, 1).contiguous().transpose(0, 1), slots), lambda: c.write(k.cpu(), k.cpu(), slots),
        lambda: c.write(k, k, slots.long()), lambda: c.attention(q, cu, ints([5])), lambda: c.attention(q, ints([0, 1]), lens),
        lambda: c.attention(q, cu, lens, out=q[:2]), lambda: c.attention(q, cu, lens, out=q.half()),
        lambda: c.attention(q, cu, lens, lse=torch.zeros((3, 2), device="cuda")),
        lambda: c.attention(q, cu, lens, lse=torch.zeros((3, 4), device="cuda", dtype=torch.float64)),
        lambda: c.attention(q[0], cu, lens), lambda: c.attention(q, ints([0, 1, 2, 3]), ints([1, 1, 1])),
        lambda: c.attention(q, cu, lens, window=2 ** 40),
        lambda: c.gather(lens, o[:1], o[:1]), lambda: c.gather(lens, o, o[:, :1]), lambda: c.gather(lens, o.half(), o.half()),
        lambda: c.gather(lens, o.transpose(2, 3).contiguous().transpose(2, 3), o)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(kvev.KvevError) as e:  # heads that no group divides: the library's own refusal
        c.attention(q[:, :3], cu, lens)
    assert e.value.code == kvev.EINVAL
    assert c.status() == 0 and int(pool.device_status) == 0


def test_one_token_views_with_any_stride(paged):
    # a dimension of one element may carry any stride
    c, q, cu, kv, table = attend_case(paged, [(200, 1)], 4, 2, 64, 16, BF16, False)
    odd = torch.as_strided(q, q.shape, (3, q.stride(1), 1))
    o, lse = run_attention(c, odd, cu, kv)
    ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv), BF16)
    k = torch.randn((1, 2, 64), device="cuda").to(BF16)
    c.write(torch.as_strided(k, k.shape, (5, 64, 1)), torch.as_strided(k, k.shape, (64, 64, 1)), ints([7]))
    assert torch.equal(c.K[0, 7], k[0]) and torch.equal(c.V[0, 7], k[0]) and c.status() == 0


# ---- captured graphs ------------------------------------------------------------------------------------

def test_graphs_in_any_order_and_side_by_side(paged):
    """Graphs captured on torch's own capture stream, with no call there before, each with units cut over many CTAs."""
    cases = []
    for seed, reqs in enumerate(([(9000, 1), (5, 1)], [(4000, 60), (300, 200)], [(12000, 3)])):
        c, q, cu, kv, table = attend_case(paged, reqs, 8, 2, 128, 16, BF16, False, seed=seed)
        dcu, dkv = ints(cu), ints(kv)
        want = c.attention(q, dcu, dkv)
        cases.append((c, q, dcu, dkv, want, torch.empty_like(q)))
    torch.cuda.synchronize()
    graphs = []
    for c, q, dcu, dkv, _, out in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attention(q, dcu, dkv, out=out)
            c.attention(q, dcu, dkv, out=out)
        graphs.append(g)
    for order in ((2, 1, 0), (1, 0, 2, 1)):
        for i in order:
            cases[i][5].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(cases[i][5], cases[i][4])
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):  # side by side, and beside calls that no graph holds
        for case, g, s in zip(cases, graphs, streams):
            with torch.cuda.stream(s):
                case[5].zero_()
                g.replay()
        again = [c.attention(q, dcu, dkv) for c, q, dcu, dkv, _, _ in cases]
        torch.cuda.synchronize()
        for case, o in zip(cases, again):
            assert torch.equal(case[5], case[4]) and torch.equal(o, case[4]) and case[0].status() == 0


# ---- released entries outside the pool --------------------------------------------------------------------

@pytest.mark.parametrize("B,page,ctx,room", [(3, 16, 40, 0), (40, 8, 1500, 0), (700, 8, 1500, 0), (300, 8, 900, 500)])
def test_release_leaves_out_pages_outside_the_pool(paged, B, page, ctx, room):
    rng = random.Random(B)
    lens = [ctx] + [rng.randint(0, ctx) for _ in range(B - 1)]
    done = [1] + [rng.choice([0, 1, 1]) for _ in range(B - 1)]
    held = [ref.pages_of(n, page) for n in lens]
    num_pages, max_pages = sum(held) + 9, max(held) + 1
    table, free, count = pool_state(rng, lens, page, num_pages, max_pages, B)
    if room:  # more comes back than the stack holds
        free, count = [0] * num_pages, num_pages - room
    bad = 0
    for s in range(B):
        for j in range(held[s]):
            if rng.random() < 0.05 or (s, j) in ((0, 0), (B - 1, held[s] - 1)):
                table[s][j] = rng.choice([-1, num_pages, 2 ** 31 - 1, -2 ** 31])
                bad += done[s]
    back = [table[s][j] for s in range(B) if done[s] for j in range(held[s]) if 0 <= table[s][j] < num_pages]
    want = (free[:count] + back)[:num_pages]
    pool = paged.PagePool(num_pages, page, ints(table), ints(free), ints([count]))
    dlens = ints(lens)
    pool.release(dlens, ints(done))
    assert bad and host(pool.free_count) == [len(want)] and host(pool.free)[:len(want)] == want
    assert host(dlens) == [0 if f else n for n, f in zip(lens, done)] and int(pool.device_status) == 2
    pool.device_status.zero_()
    # what is given out afterwards is in the pool, and the last ones first
    kv, cu, slots, pos, granted = pool.tables(ints([0]), ints([2 * page]), 2 * page)
    assert host(slots)[::page] == [want[-1] * page, want[-2] * page] and int(pool.device_status) == 0


# ---- streams ------------------------------------------------------------------------------------------------

def test_status_waits_for_every_stream(paged):
    c = make_cache(paged, 2, 16, 2, 64, ints([[0]]), BF16, False)
    k = torch.ones((1, 2, 64), dtype=BF16, device="cuda")
    bad, good = ints([99]), ints([3])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(1000)
        c.write(k, k, good)
    assert c.status() == 0  # (and all kernels are loaded)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)  # 0.1 s
    c.write(k, k, bad, stream=s)
    assert c.status() == 2 and c.status() == 0


def test_new_outputs_on_another_stream(paged):
    c, q, cu, kv, table = attend_case(paged, [(900, 3), (40, 40)], 8, 2, 128, 16, BF16, False)
    dcu, dkv = ints(cu), ints(kv)
    want = c.attention(q, dcu, dkv)
    pool = paged.PagePool(8, 16, ints([[0] * 4]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = c.attention(q, dcu, dkv, stream=s)
    got = pool.tables(ints([0]), ints([20]), 20, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and host(got[0]) == [20] and host(got[1]) == [0, 20] and c.status() == 0


# ---- sums past 32 bits ----------------------------------------------------------------------------------------

def test_tables_lengths_behind_refused_requests_of_any_size(paged):
    big = 2 ** 31 - 1
    pool = paged.PagePool(64, 16, ints([[60, -1], [61, -1], [62, -1], [63, -1]]), ints(list(range(64))), ints([60]))
    kv, cu, slots, pos, granted = pool.tables(ints([0, 0, 5, 15]), ints([big, big, 3, 2]), 16)
    assert host(granted) == [0, 0, 1, 1] and host(kv) == [0, 0, 8, 17]
    assert host(cu) == [0, big, big, big, big]  # cut off at the most that an int holds
    assert host(slots) == [-1] * 16 and host(pos) == [-1] * 16 and int(pool.device_status) == 2
    assert host(pool.free_count) == [59] and host(pool.block_table)[3] == [63, 59]


def test_gather_into_rows_of_the_largest_capacity(paged):
    import ctypes
    c = make_cache(paged, 4, 16, 1, 64, ints([[2, 1]]), BF16, False)
    o = torch.zeros((2, 20, 64), dtype=BF16, device="cuda")  # of one request and head: the rows past lens are not touched
    lens = ints([20])
    rc = kvev.kvev_paged_gather(ctypes.addressof(c.desc), c.block_table.data_ptr(), 2, lens.data_ptr(), 1, 2 ** 31 - 1,
                                o[0].data_ptr(), o[1].data_ptr(), c.device_status.data_ptr(),
                                torch.cuda.current_stream().cuda_stream)
    assert rc == kvev.OK and c.status() == 0
    assert torch.equal(o[0, :16], c.K[2, :, 0]) and torch.equal(o[1, 16:], c.V[1, :4, 0])

"""Paged caches of 8 bits on the GPU: rows quantised, read back and attended with, against their plain forms."""
import math
import random

import pytest
import torch

from paper_2606_15157_gb300 import kvev
from tests import paged_ref as ref
from tests import q8_ref
from tests.test_gpu_paged import BF16, FP16, host, ints, pool_state

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    from paper_2606_15157_gb300 import build, paged
    build.build()
    return paged


def bytes_of(c):
    return [x.view(torch.uint8).clone() for x in (c.K, c.V, c.K_scale, c.V_scale)]


def make_cache(paged, pages, page, H, d, table, dtype, heads_first, seed=0, spread=2.0):
    """A cache whose rows are quantised ones, of magnitudes e^(spread randn)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = paged.QuantizedCache.empty(pages, page, H, d, table, dtype, heads_first)
    for x, b in ((c.K, c.K_scale), (c.V, c.V_scale)):
        rows = torch.randn((pages, page, H, d), generator=g, device="cuda")
        rows = rows * torch.exp((spread * torch.randn((pages, page, H, 1), generator=g, device="cuda")).clamp(-4, 2 if x is c.K else 4))
        codes, e = q8_ref.quantise(rows.to(dtype))
        x.view(torch.uint8).copy_(codes)
        b.copy_(e.transpose(1, 2))
    return c


# ---- write ------------------------------------------------------------------------------------------

def rows_of_every_kind(T, H, d, dtype, seed):
    """Rows of all magnitudes of the type, zeros, single elements, the type's ends, halves of steps, NaN and infinities."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    top = 127 if dtype is BF16 else 15
    x = torch.randn((T, H, d), generator=g, device="cuda") * torch.exp2(torch.randint(-top - 3, top - 1, (T, H, 1), generator=g, device="cuda").float())
    x = x.clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype)
    special = [0.0, -0.0, torch.finfo(dtype).max, -torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal, torch.finfo(dtype).tiny / 2,
               1.75, 1.8125, 448.0, 464.0, 2.0 ** -9]
    for i, v in enumerate(special):
        x[i % T, i % H, (3 * i) % d:] = v
    flat = x.view(-1)
    flat[5::97] = torch.tensor([17.0, 18.0, 19.0, -17.0], device="cuda").to(dtype).repeat(flat[5::97].numel() // 4 + 1)[:flat[5::97].numel()]
    if T > 2:
        x[T - 1, 0, 1], x[T - 1, H - 1, 2], x[T - 2, 0, 0] = math.nan, math.inf, -math.inf
        x[T - 2, H - 1] = math.nan  # a row without a finite element
    return x


@pytest.mark.parametrize("T,H,d,page,dtype,heads_first", [
    (1, 8, 128, 16, BF16, False), (1, 1, 64, 8, FP16, True), (17, 3, 128, 32, BF16, True), (300, 2, 64, 128, BF16, False),
    (2100, 8, 128, 16, FP16, True), (2049, 5, 128, 256, BF16, False), (40, 7, 64, 16, FP16, False)])
def test_write_matches_plain(paged, T, H, d, page, dtype, heads_first):
    g = torch.Generator(device="cuda").manual_seed(T)
    pages = ref.pages_of(T, page) + 3
    c = make_cache(paged, pages, page, H, d, ints([[0]]), dtype, heads_first)
    # k and v as slices of a fused projection
    qkv = torch.stack([rows_of_every_kind(T, H, d, dtype, i) for i in range(3)], dim=1)
    k, v = qkv[:, 1], qkv[:, 2]
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T].to(torch.int32)
    if T > 2:
        slots[1] = -1
    want = bytes_of(c)
    keep = (slots >= 0).nonzero().flatten()
    at = slots[keep].long()
    for x, i in ((k, 0), (v, 1)):
        codes, e = q8_ref.quantise(x[keep])
        want[i][at // page, at % page] = codes
        want[i + 2].transpose(1, 2)[at // page, at % page] = e
    c.write(k, v, slots)
    got = bytes_of(c)
    for i in (0, 1):  # (a NaN's sign says nothing)
        nan = want[i] & 0x7f == 0x7f
        assert torch.equal(got[i] & torch.where(nan, 0x7f, 0xff).to(torch.uint8), want[i])
    assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3]) and c.status() == 0


def test_write_skips_slots_past_the_pool(paged):
    c = make_cache(paged, 2, 16, 2, 64, ints([[0]]), BF16, False)
    want = bytes_of(c)
    k = torch.ones((3, 2, 64), dtype=BF16, device="cuda")
    c.write(k, k, ints([32, -7, 2 ** 31 - 1]))
    assert all(torch.equal(a, b) for a, b in zip(bytes_of(c), want)) and c.status() == 2 and c.status() == 0
    c.write(k[:0], k[:0], ints([]))


# ---- gather -----------------------------------------------------------------------------------------

@pytest.mark.parametrize("lens,H,d,page,dtype,heads_first,S_cap", [
    ([1], 8, 128, 16, BF16, False, 1), ([0, 5, 64], 2, 64, 32, FP16, True, 70), ([1000, 0, 313, 1024], 3, 128, 8, BF16, False, 1024),
    ([2000, 1999], 8, 128, 256, BF16, True, 2048), ([500, 31, 32, 33], 1, 64, 64, FP16, False, 512), ([700, 64], 5, 128, 64, FP16, True, 705)])
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
        for x, b, w in ((c.K, c.K_scale, wK), (c.V, c.V_scale, wV)):
            v = q8_ref.values(x.view(torch.uint8)[p], b[p])
            assert torch.equal(v.to(dtype).double(), v)
            w[s, :, :n] = v.to(dtype).flatten(0, 1)[:n].transpose(0, 1)
    c.gather(ints(lens), oK, oV)
    assert torch.equal(oK, wK) and torch.equal(oV, wV) and c.status() == 0


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_gather_reads_every_code_at_every_exponent(paged, dtype):
    lo, hi = q8_ref.RANGE[dtype]
    n = (hi - lo + 1) * 2
    page = 16
    pages = ref.pages_of(n, page)
    c = paged.QuantizedCache.empty(pages, page, 1, 128, ints([list(range(pages))]), dtype)
    every = torch.arange(256, dtype=torch.uint8, device="cuda").view(2, 128).repeat(pages * page // 2, 1)
    for x, b in ((c.K, c.K_scale), (c.V, c.V_scale)):
        x.view(torch.uint8).copy_(every.view(pages, page, 1, 128))
        e = (torch.arange(pages * page, device="cuda") // 2 + lo + 127).clamp(max=hi + 126)  # (at the largest, codes over 240 stand for none)
        b.copy_(e.view(pages, 1, page).to(torch.uint8))
    o = torch.zeros((1, 1, n, 128), dtype=dtype, device="cuda")
    oV = torch.zeros_like(o)
    c.gather(ints([n]), o, oV)
    want = q8_ref.values(c.K, c.K_scale).view(-1, 128)[:n]
    got = o[0, 0].double()
    nan = torch.isnan(want)
    assert torch.equal(nan, torch.isnan(got)) and torch.equal(got[~nan], want[~nan]) and torch.equal(oV.view(torch.int16), o.view(torch.int16))


def test_gather_flags_what_is_out_of_range(paged):
    c = make_cache(paged, 4, 16, 1, 64, ints([[0, 9], [1, 2], [3, -1]]), BF16, False)
    o = torch.zeros((3, 1, 24, 64), dtype=BF16, device="cuda")
    oV = torch.zeros_like(o)
    c.gather(ints([20, 40, -3]), o, oV)
    assert c.status() == 2
    K = q8_ref.values(c.K, c.K_scale).to(BF16)
    assert torch.equal(o[0, 0, :16], K[0, :, 0]) and not o[0, 0, 16:].any()  # page 9 is left out
    assert torch.equal(o[1, 0, :16], K[1, :, 0]) and torch.equal(o[1, 0, 16:], K[2, :8, 0]) and not o[2].any()


# ---- attention --------------------------------------------------------------------------------------

def attend_case(paged, reqs, H_q, H, d, page, dtype, heads_first, window=0, junk=False, seed=0, q_gain=0.7, spread=1.0):
    """reqs: [(kv length, new rows)].  Returns (cache, q, cu, kv, table).  junk: NaN codes and any exponent where no row sees."""
    rng = random.Random(f"{reqs[:8]}/{page}/{seed}")
    kv, q_len = [r[0] for r in reqs], [r[1] for r in reqs]
    num_pages = sum(ref.pages_of(n, page) for n in kv) + 3
    table, _, _ = pool_state(rng, kv, page, num_pages, max(1, max(ref.pages_of(n, page) for n in kv)) + 1, len(reqs))
    c = make_cache(paged, num_pages, page, H, d, ints(table), dtype, heads_first, seed, spread)
    cu = [0]
    for n in q_len:
        cu.append(cu[-1] + n)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (q_gain * torch.randn((max(cu[-1], 1), H_q, d), generator=g, device="cuda")).to(dtype)[:cu[-1]]
    if junk:
        dead = torch.ones(c.K.shape[:2], dtype=torch.bool, device="cuda")
        for s, (n, m) in enumerate(reqs):
            lo = max(0, n - m + 1 - window) if window else 0
            for k in range(lo if m else n, n):
                dead[table[s][k // page], k % page] = False
        for x, b in ((c.K, c.K_scale), (c.V, c.V_scale)):
            x.view(torch.uint8)[dead] = 0x7f
            b.transpose(1, 2)[dead] = 255
    return c, q, cu, kv, table


def run_attention(c, q, cu, kv, **kw):
    lse = torch.full((q.shape[0], q.shape[1]), 77.0, device="cuda")
    o = c.attention(q, ints(cu), ints(kv), lse=lse, **kw)
    return o, lse


def plain(c, table, q, cu, kv, scale=0.0, window=0):
    return ref.attention(q8_ref.values(c.K, c.K_scale), q8_ref.values(c.V, c.V_scale), table, q, cu, kv, scale, window)


def check(paged, reqs, H_q, H, d, page, dtype=BF16, heads_first=False, window=0, scale=0.0, **kw):
    c, q, cu, kv, table = attend_case(paged, reqs, H_q, H, d, page, dtype, heads_first, window, **kw)
    o, lse = run_attention(c, q, cu, kv, window=window, scale=scale)
    assert c.status() == 0
    q8_ref.check_attention(o, lse, plain(c, table, q, cu, kv, scale, window), dtype)
    o2, lse2 = run_attention(c, q, cu, kv, window=window, scale=scale)  # the same bits again
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


SINGLE = [(n, 1) for n in (1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 5000)]


@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (32, 8, 128, 64, FP16, True), (8, 8, 64, 8, BF16, False), (16, 2, 64, 128, FP16, True),
    (7, 1, 128, 256, BF16, True), (10, 2, 128, 32, BF16, False), (128, 1, 128, 16, FP16, False), (96, 1, 64, 16, BF16, True),
    (1, 1, 128, 16, BF16, False), (12, 1, 64, 32, FP16, False)])
def test_attention_single_tokens(paged, H_q, H, d, page, dtype, heads_first):
    check(paged, SINGLE, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("reqs", [[(3, 3)], [(16, 16)], [(400, 400)], [(129, 5), (1000, 33), (0, 0), (260, 64), (1, 1)],
                                  [(2000, 300), (700, 1), (513, 65), (64, 2)], [(1500, 1025)], [(900, 4), (4000, 3), (77, 2)]])
@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (8, 8, 64, 32, FP16, True), (8, 2, 64, 8, BF16, False), (5, 1, 128, 128, FP16, False)])
def test_attention_chunks(paged, reqs, H_q, H, d, page, dtype, heads_first):
    check(paged, reqs, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (8, 8, 64, 32, FP16, True), (8, 1, 64, 8, BF16, False), (15, 1, 128, 128, FP16, False), (40, 2, 128, 16, BF16, True)])
def test_attention_chunks_among_as_many_requests_as_rows(paged, H_q, H, d, page, dtype, heads_first):
    check(paged, [(300, 40), (77, 5)] + [(50, 0)] * 45 + [(9, 1)], H_q, H, d, page, dtype, heads_first, window=70)


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 129, 1000, 10 ** 9])
@pytest.mark.parametrize("H_q,H,d,page", [(8, 2, 128, 16), (5, 1, 64, 64)])
def test_attention_windows(paged, window, H_q, H, d, page):
    check(paged, [(1, 1), (130, 3), (333, 333), (1000, 1), (45, 40), (3000, 1)], H_q, H, d, page, window=window)


@pytest.mark.parametrize("window,heads_first", [(0, False), (50, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_ignores_what_no_row_sees(paged, window, heads_first, d):
    check(paged, [(1, 1), (130, 3), (333, 333), (1000, 1), (45, 40), (600, 129)], 8, 2, d, 16, BF16, heads_first, window=window, junk=True)


@pytest.mark.parametrize("scale", [0.3, 1e-6])
def test_attention_scale(paged, scale):
    check(paged, [(300, 1), (200, 20)], 8, 2, 128, 16, scale=scale, q_gain=0.2)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 40])
def test_attention_rows_whose_values_differ_by_powers_of_two(paged, dtype, new):
    # the keys with nearly all of the weight hold small values, the others' are up to 2^20 times theirs; logits rise along the context
    c, q, cu, kv, table = attend_case(paged, [(900, new)], 4, 1, 128, 16, dtype, False, spread=0.0)
    lo, hi = q8_ref.RANGE[dtype]
    pos = torch.arange(900, device="cuda")
    p = torch.tensor(table[0], device="cuda")[pos // 16]
    q.abs_()
    codes = torch.full((128,), 0x38, dtype=torch.uint8, device="cuda")  # 1
    c.K.view(torch.uint8)[p, pos % 16, 0] = codes
    # logits: q.1 2^e / sqrt(d), e from far below to one; then V's exponents fall as they rise
    e = (-12 + pos // 75).clamp(max=0)
    c.K_scale[p, 0, pos % 16] = (127 + e.clamp(min=lo)).to(torch.uint8)
    c.V_scale[p, 0, pos % 16] = (127 + (8 if dtype is BF16 else 2) - 20 * (pos // 75) // 12).clamp(min=127 + lo).to(torch.uint8)
    o, lse = run_attention(c, q, cu, kv)
    r = plain(c, table, q, cu, kv)
    q8_ref.check_attention(o, lse, r, dtype)


def test_attention_zero_rows(paged):
    # rows of zeros have the smallest exponent; so may all rows of a request
    c, q, cu, kv, table = attend_case(paged, [(300, 1), (300, 30), (40, 1)], 8, 2, 128, 16, BF16, False)
    k = torch.zeros((16, 2, 128), dtype=BF16, device="cuda")
    for s in (0, 1):
        for j in table[s][:ref.pages_of(kv[s], 16)]:
            c.write(k, k, ints(range(16 * j, 16 * j + 16)))
    o, lse = run_attention(c, q, cu, kv)
    assert c.status() == 0 and not o[:31].any()
    q8_ref.check_attention(o, lse, plain(c, table, q, cu, kv), BF16)


def test_attention_empty_rows_and_rows_past_the_last(paged):
    c, q, cu, kv, table = attend_case(paged, [(300, 20)], 8, 2, 128, 16, BF16, False)
    reqs_kv, reqs_cu = [5, 0, 0], [0, 12, 19, 20]
    c2 = paged.QuantizedCache(c.K, c.V, c.K_scale, c.V_scale, c.block_table.repeat(3, 1))
    o, lse = run_attention(c2, q, reqs_cu, reqs_kv)
    assert c2.status() == 0
    q8_ref.check_attention(o, lse, plain(c, table * 3, q, reqs_cu, reqs_kv), BF16)
    assert not o[:7].any() and not o[12:].any() and torch.isinf(lse[:7]).all()
    out = torch.full_like(q, 3.0)
    lse = torch.full((20, 8), 5.0, device="cuda")
    c2.attention(q, ints([0, 11, 12, 12]), ints([300, 5, 0]), out=out, lse=lse)
    assert (out[12:] == 3).all() and (lse[12:] == 5).all() and c2.status() == 0


def test_strides_and_32_bit_offsets(paged):
    # pages over 2^31 bytes apart, in one tensor with their scales' pages apart too
    page, H, d = 16, 2, 64
    base = torch.zeros(3 * 2 ** 31 + 2 ** 16, dtype=torch.uint8, device="cuda")
    at = lambda off: torch.as_strided(base, (3, page, H, d), (2 ** 31, d * H * 2, d, 1), off).view(q8_ref.E4M3)  # noqa: E731
    sc = lambda off: torch.as_strided(base, (3, H, page), (2 ** 31, page, 1), off)  # noqa: E731
    table = [[2, 1, 0]]
    c = paged.QuantizedCache(at(0), at(2 ** 13), sc(2 ** 14), sc(2 ** 14 + 64), ints(table))
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn((40, 8, d), generator=g, device="cuda").to(BF16)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    slots = [table[0][t // page] * page + t % page for t in range(40)]
    c.write(k, v, ints(slots))
    wide = torch.zeros((40, 6, 2, d), dtype=BF16, device="cuda")
    out, lse = wide[:, 1:5, 1], torch.empty((40, 4), device="cuda")
    c.attention(q, ints([0, 40]), ints([40]), out=out, lse=lse)
    small = paged.QuantizedCache(*(x.view(torch.uint8).clone().view(q8_ref.E4M3) for x in (c.K, c.V)), c.K_scale.clone(), c.V_scale.clone(),
                                 ints(table))
    q8_ref.check_attention(out, lse, plain(small, table, q, [0, 40], [40]), BF16)
    assert not wide[:, :, 0].any() and not wide[:, 0].any() and not wide[:, 5].any()
    one = torch.empty_like(lse[:1])
    o1 = c.attention(q[39:], ints([0, 1]), ints([40]), lse=one)
    q8_ref.check_attention(o1, one, plain(small, table, q[39:], [0, 1], [40]), BF16)
    oK, oV = torch.zeros((1, H, 48, d), dtype=BF16, device="cuda"), torch.zeros((1, H, 48, d), dtype=BF16, device="cuda")
    c.gather(ints([40]), oK, oV)
    codes, e = q8_ref.quantise(k)
    want = (codes.view(q8_ref.E4M3).double() * torch.exp2(e.double() - 127)[..., None]).to(BF16)
    assert torch.equal(oK[0, :, :40].transpose(0, 1), want) and c.status() == 0


def test_attention_flags_what_is_out_of_range(paged):
    for new in (4, 40):
        c, q, cu, kv, table = attend_case(paged, [(100, new), (60, new), (90, 2)], 4, 2, 64, 16, BF16, False)
        good = run_attention(c, q, cu, kv)
        for bad in ([100, -1, 90], [100, 10 ** 6, 90], [100, -2 ** 31, 90]):
            o, lse = run_attention(c, q, cu, bad)
            assert c.status() == 2
            for i in (0, 2):
                assert torch.equal(o[cu[i]:cu[i + 1]], good[0][cu[i]:cu[i + 1]])
        o, lse = run_attention(c, q, [0, new, 2, 99], kv)
        assert c.status() == 2 and torch.equal(o[:new], good[0][:new])
        # pages outside the pool count as zero rows
        t2 = [list(r) for r in table]
        t2[0][1], t2[0][2] = -5, 10 ** 6
        c2 = paged.QuantizedCache(c.K, c.V, c.K_scale, c.V_scale, ints(t2))
        o, lse = run_attention(c2, q, cu, kv)
        assert c2.status() == 2 and torch.equal(o[new:], good[0][new:])
        zero = paged.QuantizedCache(*(x.view(torch.uint8).clone().view(q8_ref.E4M3) for x in (c.K, c.V)), c.K_scale, c.V_scale, ints(table))
        for j in (1, 2):
            zero.K.view(torch.uint8)[table[0][j]] = 0
            zero.V.view(torch.uint8)[table[0][j]] = 0
        q8_ref.check_attention(o, lse, plain(zero, table, q, cu, kv), BF16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B", [31, 32, 33, 385, 511, 513, 700])
def test_attention_batches_around_the_schedule_s_sizes(paged, B, d):
    rng = random.Random(B)
    reqs = [(n, min(n, rng.choice([1, 1, 1, 1, 2, 40]))) for n in (rng.randint(0, 300) for _ in range(B))]
    check(paged, reqs, 4, 2, d, 16)


def test_attention_on_another_stream_and_in_graphs(paged):
    cases = []
    for seed, reqs in enumerate(([(3000, 1), (100, 1), (1, 1)], [(9000, 1), (300, 200)], [(5000, 30)])):
        c, q, cu, kv, table = attend_case(paged, reqs, 8, 2, 128, 16, BF16, False, seed=seed)
        dcu, dkv = ints(cu), ints(kv)
        cases.append((c, q, dcu, dkv, c.attention(q, dcu, dkv), torch.empty_like(q)))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [c.attention(q, dcu, dkv, stream=s) for c, q, dcu, dkv, _, _ in cases]
    s.synchronize()
    assert all(torch.equal(a, case[4]) for a, case in zip(got, cases))
    graphs = []
    for c, q, dcu, dkv, _, out in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attention(q, dcu, dkv, out=out)
            c.attention(q, dcu, dkv, out=out)
        graphs.append(g)
    for i in (2, 0, 1, 0, 2):
        cases[i][5].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(cases[i][5], cases[i][4])
    c, q, dcu, dkv, _, out = cases[0]  # replayed with other lengths
    dkv.copy_(ints([2999, 55, 0]))
    graphs[0].replay()
    assert torch.equal(out, c.attention(q, dcu, dkv)) and all(case[0].status() == 0 for case in cases)


def test_refused_tensors(paged):
    table = ints([[0, 1], [2, 3]])
    c = paged.QuantizedCache.empty(8, 16, 2, 64, table)
    k = torch.zeros((3, 2, 64), dtype=BF16, device="cuda")
    q = torch.zeros((3, 4, 64), dtype=BF16, device="cuda")
    lens, cu, slots = ints([5, 6]), ints([0, 1, 3]), ints([0, 1, 2])
    o = torch.zeros((2, 2, 32, 64), dtype=BF16, device="cuda")
    make = lambda K=c.K, V=c.V, a=c.K_scale, b=c.V_scale, t=table, **kw: paged.QuantizedCache(K, V, a, b, t, **kw)  # noqa: E731
    bad = [
        lambda: make(c.K.cpu(), c.V.cpu()), lambda: make(V=c.V[:, :8]), lambda: make(c.K.view(torch.uint8), c.V.view(torch.uint8)),
        lambda: make(dtype=torch.float32), lambda: make(a=c.K_scale.float()), lambda: make(a=c.K_scale[:, :1]),
        lambda: make(a=c.K_scale.transpose(1, 2).contiguous().transpose(1, 2)), lambda: make(t=table.long()),
        lambda: make(a=c.K_scale.cpu(), b=c.V_scale.cpu()), lambda: make(c.K.transpose(2, 3), c.V.transpose(2, 3)),
        lambda: c.write(k, k[:2], slots), lambda: c.write(k.half(), k.half(), slots), lambda: c.write(k, k, slots[:2]),
        lambda: c.write(k, k, slots.long()), lambda: c.write(q, q, slots), lambda: c.write(k.cpu(), k.cpu(), slots),
        lambda: c.attention(q, cu, ints([5])), lambda: c.attention(q.half(), cu, lens), lambda: c.attention(q, cu, lens, out=q[:2]),
        lambda: c.attention(q, cu, lens, lse=torch.zeros((3, 2), device="cuda")), lambda: c.attention(q[0], cu, lens),
        lambda: c.attention(q, ints([0, 1, 2, 3]), ints([1, 1, 1])), lambda: c.attention(q, cu, lens, window=2 ** 40),
        lambda: c.attention(q, cu, lens, workspace=torch.zeros(8)),
        lambda: c.gather(lens, o[:1], o[:1]), lambda: c.gather(lens, o.half(), o.half()), lambda: c.gather(lens, o, o[:, :1])]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(kvev.KvevError) as e:
        c.attention(q[:, :3], cu, lens)
    assert e.value.code == kvev.EINVAL
    with pytest.raises(kvev.KvevError) as e:  # codes whose heads start between 16-byte boundaries
        x = torch.zeros((8, 16, 2, 72), dtype=torch.uint8, device="cuda").view(q8_ref.E4M3)[..., :64]
        make(x, x).write(k, k, slots)
    assert e.value.code == kvev.EINVAL and c.status() == 0


def test_a_prompt_in_chunks_then_generations(paged):
    """Tables, writes, attention and read-back together, as a serving program makes them; each layer call against the plain form
    of what its pages then stand for."""
    H_q, H, d, page, B = 8, 2, 128, 16, 3
    prompts, steps, chunk = [150, 70, 33], 3, 64
    width = ref.pages_of(max(prompts) + steps, page)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    pool = paged.PagePool(B * width, page, table)
    c = paged.QuantizedCache.empty(B * width, page, H, d, table)
    g = torch.Generator(device="cuda").manual_seed(0)
    rows = [torch.randn((n + steps, H_q + 2 * H, d), generator=g, device="cuda").to(BF16) for n in prompts]
    lens, done = torch.zeros(B, dtype=torch.int32, device="cuda"), [0] * B
    for i in range(3 + steps):
        new = [min(chunk, n - a) if a < n else 0 for a, n in zip(done, prompts)] if i < 3 else [1] * B
        T = sum(new)
        _, cu, slots, _, granted = pool.tables(lens, ints(new), T, kv_lens=lens)
        assert bool(granted.all())
        x = torch.cat([rows[s][done[s]:done[s] + new[s]] for s in range(B)])
        q, k, v = x[:, :H_q], x[:, H_q:H_q + H], x[:, H_q + H:]
        c.write(k, v, slots)
        lse = torch.empty((T, H_q), device="cuda")
        o = c.attention(q, cu, lens, lse=lse)
        done = [a + n for a, n in zip(done, new)]
        K, V = (torch.nan_to_num(q8_ref.values(x, b)) for x, b in ((c.K, c.K_scale), (c.V, c.V_scale)))
        q8_ref.check_attention(o, lse, ref.attention(K, V, host(table), q, host(cu), host(lens)), BF16)
    oK, oV = (torch.zeros((B, H, 160, d), dtype=BF16, device="cuda") for _ in range(2))
    c.gather(lens, oK, oV)
    for s in range(B):
        codes, e = q8_ref.quantise(rows[s][:done[s], H_q:H_q + H])
        want = (codes.view(q8_ref.E4M3).double() * torch.exp2(e.double() - 127)[..., None]).to(BF16)
        assert torch.equal(oK[s, :, :done[s]].transpose(0, 1), want)
    assert c.status() == 0


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("new", [1, 17])
def test_attention_many_small_weights(paged, dtype, new):
    """One key has nearly all of the weight, 8,000 others 2^-20 each: together 2^-7 of the result.  Single tokens hold a weight to 2^-30 of the
    largest, so all of them to 8,000 2^-30 |v| < 2^-17; chunks to the type's unit roundoff of each."""
    n = 8001
    c, q, cu, kv, table = attend_case(paged, [(n, new)], 4, 1, 128, 16, dtype, False, spread=0.0)
    pos = torch.arange(n, device="cuda")
    p = torch.tensor(table[0], device="cuda")[pos // 16]
    q.fill_(1.0)
    c.K.view(torch.uint8)[p, pos % 16, 0] = 0  # logits of 0, but for key 5:
    c.K.view(torch.uint8)[p[5], 5, 0] = 0x38
    c.K_scale[p[5], 0, 5] = 127
    c.V.view(torch.uint8)[p, pos % 16, 0] = 0x38  # values 1, of key 5 one half
    c.V_scale[p, 0, pos % 16] = 127
    c.V_scale[p[5], 0, 5] = 126
    scale = 20 * math.log(2) / 128  # key 5's logit is 20 ln 2 above
    o, lse = run_attention(c, q, cu, kv, scale=scale)
    q8_ref.check_attention(o, lse, plain(c, table, q, cu, kv, scale), dtype, small_weights=n * 2.0 ** -30 if new == 1 else 0.0)


@pytest.mark.parametrize("new", [1, 40])
def test_attention_of_codes_that_are_no_numbers(paged, new):
    """A NaN in a row that is seen is the answer of its head's rows that see it, and of nobody else's."""
    c, q, cu, kv, table = attend_case(paged, [(300, new), (200, 1)], 8, 2, 128, 16, BF16, False)
    good, _ = run_attention(c, q, cu, kv)
    c.V.view(torch.uint8)[table[0][3], 2, 1, 77] = 0xff
    o, lse = run_attention(c, q, cu, kv)
    assert torch.isnan(o[:new, 4:, 77]).all() and c.status() == 0
    assert torch.equal(o[:, :4], good[:, :4]) and torch.equal(o[new:], good[new:])
    c.K.view(torch.uint8)[table[0][5], 1, 0, 3] = 0x7f
    o, lse = run_attention(c, q, cu, kv)
    assert torch.isnan(o[:new, :4]).all() and torch.isnan(lse[:new, :4]).all() and torch.equal(o[new:], good[new:])


@pytest.mark.parametrize("e", [-120, -60, 60, 115])
@pytest.mark.parametrize("new", [1, 20])
def test_attention_over_values_at_the_ends_of_the_type(paged, e, new):
    c, q, cu, kv, table = attend_case(paged, [(500, new)], 4, 1, 128, 16, BF16, False, spread=0.0)
    c.V_scale.fill_(127 + e)
    o, lse = run_attention(c, q, cu, kv)
    r = list(plain(c, table, q, cu, kv))
    f = 2.0 ** -e  # (compared at 1: the tolerance has an absolute part)
    if e > -110:  # (below, the results are subnormal)
        q8_ref.check_attention(o.double() * f, lse, [r[0] * f, r[1], r[2] * f, r[3]], BF16)
    else:
        assert ((o.double() - r[0]).abs() <= 2.0 ** -126 + 2.0 ** -6 * r[2]).all()


@pytest.mark.parametrize("H_q,H", [(2, 2), (8, 2), (16, 1), (40, 2)])
def test_attention_of_few_rows_flags_what_is_out_of_range(paged, H_q, H):
    """Batches with no more rows than a request of few rows has: counts that decrease, are negative or past T, lengths past the table."""
    for T, cus in ((1, ([0, 2], [0, -1], [-1, 0], [1, 0])), (3, ([0, 99], [2, 0], [0, -2 ** 31], [-7, 1], [0, 4])), (4, ([0, 5], [0, 2 ** 31 - 1], [4, 3]))):
        c, q, cu, kv, table = attend_case(paged, [(100, T)], H_q, H, 64, 16, BF16, False)
        good = run_attention(c, q, cu, kv)
        assert c.status() == 0 and not (good[1] == 77).any()
        for bad_cu, bad_kv in [(x, kv) for x in cus] + [(cu, [-1]), (cu, [10 ** 6])]:
            out = torch.full_like(q, 3.0)
            o, lse = run_attention(c, q, bad_cu, bad_kv, out=out)
            assert c.status() == 2, (T, bad_cu, bad_kv)
            assert (o == 3).all() and (lse == 77).all()
        # beside a request in order
        c, q, cu, kv, table = attend_case(paged, [(100, T), (60, 0)], H_q, H, 64, 16, BF16, False)
        good = run_attention(c, q, cu, kv)
        o, lse = run_attention(c, q, [0, T, T + 1], kv)
        assert c.status() == 2 and torch.equal(o, good[0]) and torch.equal(lse, good[1])


@pytest.mark.parametrize("H_q,H,new,slots", [(8, 2, 30, 31), (8, 2, 5, 7), (2, 2, 17, 32), (40, 2, 3, 9)])
def test_attention_of_a_long_request_among_idle_ones(paged, H_q, H, new, slots):
    """A request of more than 16 query rows to a KV head attends as it does alone, also where there are no more rows than requests: the same bits
    (up to 32 requests a warp makes the schedule, whose shares go by the rows there are)."""
    c, q, cu, kv, table = attend_case(paged, [(1500, new)], H_q, H, 128, 16, BF16, False)
    want = run_attention(c, q, cu, kv)
    at = slots // 2
    t = torch.full((slots, len(table[0])), -1, dtype=torch.int32, device="cuda")
    t[at] = ints(table[0])
    c2 = paged.QuantizedCache(c.K, c.V, c.K_scale, c.V_scale, t)
    o, lse = run_attention(c2, q, [0] * (at + 1) + [new] * (slots - at), [0] * at + kv + [0] * (slots - 1 - at))
    assert c2.status() == 0 and torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("H_q,H,d", [(8, 2, 128), (2, 2, 64), (40, 2, 128)])
@pytest.mark.parametrize("reqs", [[(300, 46)] + [(50, 0)] * 45, [(300, 30), (77, 4)] + [(50, 0)] * 32 + [(9, 1), (700, 1)], [(130, 5), (2, 0), (1, 1), (40, 0), (5, 0), (5, 0)]],
                         ids=["one", "some", "six"])
def test_attention_of_as_many_rows_as_requests(paged, reqs, H_q, H, d):
    assert sum(n for _, n in reqs) == len(reqs)
    check(paged, reqs, H_q, H, d, 16)


@pytest.mark.parametrize("H_q,H,new", [(4, 1, 1), (4, 1, 3), (2, 2, 16), (16, 1, 1), (10, 2, 3)])
@pytest.mark.parametrize("others", [0, 30])
def test_attention_of_few_rows_is_on_the_codes_whatever_else_there_is(paged, H_q, H, new, others):
    """Keys 0 and 1 have weights 1 and 2^-(2^-10) and values 1 and -1, the others weights under 2^-39: the result is 3.4e-4, and 0 where weights are
    rounded to bf16.  32-bit logits of 20 err by 8 2^-24 20 at most, weights held in parts by 2^-16 of their own size, the result by half a step,
    2^-9 of its own: (7e-6 + 2 x 1.6e-5) / 2 + 7e-7 < 2e-5."""
    kv = new + 2
    c, q, cu, kvs, table = attend_case(paged, [(kv, new)] + [(3, 1)] * others, H_q, H, 64, 16, BF16, False)
    page = table[0][0]  # (one page: 18 keys at most)
    p2 = table[0][1] if kv > 16 else page
    q[:new] = 0
    q[:new, :, 0], q[:new, :, 1] = 1.0, 2.0 ** -10
    for p in {page, p2}:
        c.K.view(torch.uint8)[p], c.V.view(torch.uint8)[p] = 0, 0
        c.K_scale[p], c.V_scale[p] = 127, 127
        c.K.view(torch.uint8)[p, :, :, 0] = 0x80 | 0x5a  # -20
    code = lambda v: int(torch.tensor(v).to(q8_ref.E4M3).view(torch.uint8))  # noqa: E731
    assert code(-20.0) == 0xda
    c.K.view(torch.uint8)[page, :2, :, 0] = code(20.0)
    c.K.view(torch.uint8)[page, 1, :, 1] = code(-1.0)
    c.V.view(torch.uint8)[page, 0], c.V.view(torch.uint8)[page, 1] = code(1.0), code(-1.0)
    o, lse = run_attention(c, q, cu, kvs, scale=math.log(2))
    w = 2.0 ** -(2.0 ** -10)
    assert c.status() == 0 and ((o[:new].double() - (1 - w) / (1 + w)).abs() <= 2e-5).all()


@pytest.mark.parametrize("H", [3, 5, 7, 10, 16, 32])
@pytest.mark.parametrize("G,d,heads_first", [(1, 64, False), (4, 128, True), (12, 64, False)])
def test_attention_of_any_number_of_kv_heads(paged, H, G, d, heads_first):
    """Numbers of KV heads that do not divide the CTAs (456, or 304 for 16 rows) among them: shares that end inside a head."""
    check(paged, [(n, 1) for n in (1, 129, 1000, 3000, 0, 257)], G * H, H, d, 16, BF16, heads_first)
    check(paged, [(700, 2), (130, 3), (1, 1), (900, 40), (40, 0)], G * H, H, d, 32, FP16, heads_first)

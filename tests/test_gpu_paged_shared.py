"""Attention of groups of requests that share a prefix, on the GPU, against the plain form of each request by itself."""
import math
import random

import pytest
import torch

from paper_2606_15157_gb300 import kvev
from tests import paged_ref as ref
from tests import q8_ref
from tests.test_gpu_paged import BF16, FP16, ints, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def paged():
    from paper_2606_15157_gb300 import build, paged
    build.build()
    return paged


def shared_case(paged, groups, H_q, H, d, page, dtype=BF16, heads_first=False, seed=0, junk=None):
    """groups: [(shared tokens, [(tokens of the request's own in all, new rows)])].  The first whole pages of a group are the
    same physical ones; (cache, q, cu, kv, table, first requests, shared lengths)."""
    rng = random.Random(f"{str(groups)[:200]}/{page}/{seed}")
    kv, q_len, common, first, shared = [], [], [], [], []
    for n, reqs in groups:
        first.append(len(kv))
        shared.append(n)
        for own, new in reqs:
            kv.append(n + own)
            q_len.append(new)
            common.append((len(first) - 1, n // page))
    width = max(1, max(ref.pages_of(n, page) for n in kv)) + 1
    pages = [n // page for n in shared]
    num_pages = sum(pages) + sum(ref.pages_of(n, page) - m for n, (_, m) in zip(kv, common)) + 3
    ids = list(range(num_pages))
    rng.shuffle(ids)
    take = lambda n: [ids.pop() for _ in range(n)]  # noqa: E731
    held = [take(n) for n in pages]
    table = []
    for n, (g, m) in zip(kv, common):
        r = held[g] + take(ref.pages_of(n, page) - m)
        table.append(r + [-1] * (width - len(r)))
    c = make_cache(paged, num_pages, page, H, d, ints(table), dtype, heads_first, seed)
    if junk is not None:
        dead = torch.ones(c.K.shape[:2], dtype=torch.bool, device="cuda")
        for s, n in enumerate(kv):
            for k in range(n):
                dead[table[s][k // page], k % page] = False
        c.K[dead], c.V[dead] = junk, junk
    cu = [0]
    for n in q_len:
        cu.append(cu[-1] + n)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (1.5 * torch.randn((max(cu[-1], 1), H_q, d), generator=g, device="cuda")).to(dtype)[:cu[-1]]
    return c, q, cu, kv, table, first + [len(kv)], shared


def run(c, q, cu, kv, groups, shared, **kw):
    lse = torch.full((q.shape[0], q.shape[1]), 77.0, device="cuda")
    o = c.attention_shared(q, ints(cu), ints(kv), ints(groups), ints(shared), lse=lse, **kw)
    return o, lse


def check(paged, groups, H_q, H, d, page, dtype=BF16, heads_first=False, scale=0.0, **kw):
    c, q, cu, kv, table, first, shared = shared_case(paged, groups, H_q, H, d, page, dtype, heads_first, **kw)
    o, lse = run(c, q, cu, kv, first, shared, scale=scale)
    assert c.status() == 0
    K, V = (torch.nan_to_num(x.double()) for x in (c.K, c.V))
    q8_ref.check_attention(o, lse, ref.attention(K, V, table, q, cu, kv, scale), dtype, parts=2)
    o2, lse2 = run(c, q, cu, kv, first, shared, scale=scale)  # the same bits again
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def ones(n, lo=1, hi=200, seed=0):
    rng = random.Random(seed)
    return [(rng.randint(lo, hi), 1) for _ in range(n)]


@pytest.mark.parametrize("groups", [
    [(2000, ones(4))], [(16, ones(2))], [(4096, ones(64, 1, 700))], [(513, ones(70)), (128, ones(3)), (300, ones(17))],
    [(1000, ones(1)), (640, ones(2))], [(0, ones(5))], [(129, [(1, 1), (1, 1), (128, 1)])]], ids=lambda g: f"{len(g)}g{g[0][0]}x{len(g[0][1])}")
@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (8, 8, 64, 32, FP16, True), (8, 2, 64, 8, BF16, False), (5, 1, 128, 128, FP16, True), (32, 2, 128, 64, BF16, False)])
def test_generations_behind_a_prefix(paged, groups, H_q, H, d, page, dtype, heads_first):
    check(paged, groups, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("groups", [
    [(1024, [(300, 300), (40, 1), (64, 64), (500, 130)])], [(700, [(129, 129), (129, 128)]), (64, [(1000, 700)]), (256, [(3, 3), (5, 2)])],
    [(2048, [(17, 17)] * 9)], [(160, [(50, 0), (60, 3), (70, 0)])], [(96, [(10, 0)] * 3), (96, [(4, 4), (4, 4)])]],
    ids=lambda g: f"{len(g)}g{g[0][0]}x{len(g[0][1])}")
@pytest.mark.parametrize("H_q,H,d,page,dtype,heads_first", [
    (32, 8, 128, 16, BF16, False), (8, 8, 64, 32, FP16, True), (6, 2, 64, 8, BF16, False)])
def test_chunks_behind_a_prefix(paged, groups, H_q, H, d, page, dtype, heads_first):
    check(paged, groups, H_q, H, d, page, dtype, heads_first)


@pytest.mark.parametrize("B,N", [(30, 1), (31, 1), (32, 1), (31, 2), (382, 1), (383, 1), (384, 1), (700, 40), (90, 90)])
@pytest.mark.parametrize("d", [64, 128])
def test_batches_around_the_schedule_s_sizes(paged, B, N, d):
    rng = random.Random(B)
    cut = sorted(rng.sample(range(1, B), N - 1)) if N < B else list(range(1, B))
    groups = []
    for a, b in zip([0] + cut, cut + [B]):
        groups.append((rng.choice([64, 100, 320]), [(n, min(n, rng.choice([1, 1, 2, 20]))) for n in (rng.randint(0, 150) for _ in range(a, b))]))
    check(paged, groups, 4, 2, d, 16)


@pytest.mark.parametrize("junk", [math.nan, math.inf, -3.3e38])
def test_what_no_row_sees_may_hold_anything(paged, junk):
    check(paged, [(100, [(29, 3), (1, 1), (300, 40)]), (33, [(5, 1), (7, 1)])], 8, 2, 128, 16, junk=junk)


def test_scale(paged):
    check(paged, [(300, ones(6)), (64, [(100, 50), (3, 1)])], 8, 2, 128, 16, scale=0.25)


def test_what_cannot_be_shared_is_left_to_the_request(paged):
    """A request without the whole prefix before its new rows, requests of no group, and no group at all."""
    c, q, cu, kv, table, first, shared = shared_case(paged, [(512, [(100, 30), (1, 1), (40, 1), (64, 64), (9, 2)])], 8, 2, 128, 16)
    r = ref.attention(c.K, c.V, table, q, cu, kv)
    kv2 = [kv[0], 400, kv[2], 20, kv[4]]  # the second holds less than the prefix, the fourth's new rows are the prefix's
    r2 = ref.attention(c.K, c.V, table, q, cu, kv2)
    o, lse = run(c, q, cu, kv2, first, shared)
    assert c.status() == 0
    q8_ref.check_attention(o, lse, r2, BF16, parts=2)
    for groups, lens in (([1, 4], [512]), ([0, 2, 2, 5], [512, 512, 256]), ([0, 0], [512]), ([3, 4, 5], [512, 100]), ([5, 5], [16])):
        o, lse = run(c, q, cu, kv, groups, lens)
        q8_ref.check_attention(o, lse, r, BF16, parts=2)
    want = torch.empty_like(lse)
    o = c.attention(q, ints(cu), ints(kv), lse=want)
    o2, lse2 = run(c, q, cu, kv, [0], [])
    assert torch.equal(o, o2) and torch.equal(want, lse2) and c.status() == 0


@pytest.mark.parametrize("gone", [[0], [0, 1, 2], list(range(11))])
def test_requests_that_are_gone_keep_their_place_in_a_group(paged, gone):
    """Finished requests have no rows, and their rows of the table name pages that are others' by now, or none."""
    c, q, cu, kv, table, first, shared = shared_case(paged, [(256, ones(12))], 8, 2, 128, 16)
    t2, kv2, cu2 = [list(r) for r in table], list(kv), [0]
    for s in range(12):
        cu2.append(cu2[-1] + (0 if s in gone else 1))
    for s in gone:
        kv2[s] = 0
        t2[s][:16] = [-1] * 8 + table[11][17:18] * 8
    c2 = paged.PagedCache(c.K, c.V, ints(t2))
    q2 = q[[s for s in range(12) if s not in gone]]
    o, lse = run(c2, q2, cu2, kv2, first, shared)
    assert c2.status() == 0
    q8_ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q2, cu2, kv2), BF16, parts=2)


def test_groups_and_lengths_out_of_range_are_flagged(paged):
    c, q, cu, kv, table, first, shared = shared_case(paged, [(512, ones(5)), (64, [(100, 50), (3, 1)])], 8, 2, 128, 16)
    r = ref.attention(c.K, c.V, table, q, cu, kv)
    for groups, lens in (([0, 5, 3], shared), ([-1, 5, 7], shared), ([0, 5, 8], shared), (first, [-1, 64]), (first, [10 ** 9, 64]),
                         ([7, 5, 0], shared), (first, [-2 ** 31, 2 ** 31 - 1])):
        o, lse = run(c, q, cu, kv, groups, lens)
        assert c.status() == 2
        q8_ref.check_attention(o, lse, r, BF16, parts=2)
    # a request out of range is left out, the others of its group are not
    for bad in (-1, 10 ** 6):
        kv2 = list(kv)
        kv2[1] = bad
        out, lse = torch.full_like(q, 3.0), torch.full((q.shape[0], 8), 5.0, device="cuda")
        c.attention_shared(q, ints(cu), ints(kv2), ints(first), ints(shared), out=out, lse=lse)
        assert c.status() == 2 and (out[1] == 3).all() and (lse[1] == 5).all()
        keep = [t for t in range(q.shape[0]) if t != 1]
        q8_ref.check_attention(out[keep], lse[keep], [x[keep] for x in r], BF16, parts=2)
    # row counts out of range, in the middle of the group and at its end
    for bad in ([0, 1, 2, 9, 4, 5, 55, 56], [0, 1, 2, 3, 4, 500, 55, 56]):
        out = torch.full_like(q, 3.0)
        c.attention_shared(q, ints(bad), ints(kv), ints(first), ints(shared), out=out)
        assert c.status() == 2
        q8_ref.check_attention(out[:2], None, [x[:2] for x in r], BF16, parts=2)


def test_rows_past_the_last_are_left(paged):
    c, q, cu, kv, table, first, shared = shared_case(paged, [(256, ones(9))], 8, 2, 128, 16)
    wide = torch.cat((q, torch.full((7, 8, 128), math.nan, dtype=BF16, device="cuda")))
    out, lse = torch.full_like(wide, 3.0), torch.full((16, 8), 5.0, device="cuda")
    c.attention_shared(wide, ints(cu), ints(kv), ints(first), ints(shared), out=out, lse=lse)
    assert (out[9:] == 3).all() and (lse[9:] == 5).all() and c.status() == 0
    q8_ref.check_attention(out[:9], lse[:9], ref.attention(c.K, c.V, table, q, cu, kv), BF16, parts=2)
    c.attention_shared(q[:0], ints([0] * 10), ints(kv), ints(first), ints(shared))
    assert c.status() == 0


def test_strides_and_a_workspace_of_ones_own(paged):
    c, q, cu, kv, table, first, shared = shared_case(paged, [(256, [(40, 30), (3, 3), (7, 1)])], 6, 2, 128, 16)
    wide = torch.zeros((34, 8, 2, 128), dtype=BF16, device="cuda")
    wide[:, 1:7, 1] = q
    out = torch.zeros((34, 2, 6, 128), dtype=BF16, device="cuda")
    n = kvev.kvev_paged_attention_shared_workspace(6, 2, 128, 34)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    lse = torch.empty((34, 6), device="cuda")
    o = c.attention_shared(wide[:, 1:7, 1], ints(cu), ints(kv), ints(first), ints(shared), out=out[:, 1], lse=lse, workspace=ws)
    assert o.data_ptr() == out[:, 1].data_ptr() and not out[:, 0].any() and c.status() == 0
    q8_ref.check_attention(o, lse, ref.attention(c.K, c.V, table, q, cu, kv), BF16, parts=2)
    assert not ws[:kvev.PAGED_SYNC_BYTES].any()  # left as found
    with pytest.raises(kvev.KvevError) as e:
        c.attention_shared(q, ints(cu), ints(kv), ints(first), ints(shared), workspace=ws[:n - 1])
    assert e.value.code == kvev.ENOMEM


def test_streams_growing_scratch_and_graphs(paged):
    cases = []
    for seed, groups in enumerate(([(800, ones(6))], [(2000, ones(40)), (64, [(200, 200), (30, 1)])], [(3000, [(900, 900), (700, 600)])])):
        c, q, cu, kv, table, first, shared = shared_case(paged, groups, 8, 2, 128, 16, seed=seed)
        a = (q, ints(cu), ints(kv), ints(first), ints(shared))
        cases.append((c, a, c.attention_shared(*a), torch.empty_like(q)))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for c, a, _, _ in cases:  # each needs more scratch than the one before, with a plain call in flight between
        got.append((c.attention_shared(*a, stream=s), c.attention(*a[:3], stream=s), c.attention_shared(*a, stream=s)))
    s.synchronize()
    for (x, _, y), case in zip(got, cases):
        assert torch.equal(x, case[2]) and torch.equal(y, case[2])
    graphs = []
    for c, a, _, out in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attention(*a[:3], out=out)  # (takes a smaller scratch first)
            c.attention_shared(*a, out=out)
        graphs.append(g)
    for i in (2, 0, 1, 0, 2):
        cases[i][3].zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(cases[i][3], cases[i][2])
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):  # side by side
        for case, g, st in zip(cases, graphs, streams):
            with torch.cuda.stream(st):
                case[3].zero_()
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(case[3], case[2]) and case[0].status() == 0 for case in cases)
    c, a, _, out = cases[0]  # replayed with another prefix and other lengths
    a[4].copy_(ints([400]))
    a[2].copy_(a[2] - 1)
    graphs[0].replay()
    assert torch.equal(out, c.attention_shared(*a)) and c.status() == 0


def test_refused_tensors(paged):
    table = ints([[0, 1], [2, 3]])
    c = paged.PagedCache.empty(8, 16, 2, 64, table)
    q = torch.zeros((3, 4, 64), dtype=BF16, device="cuda")
    lens, cu, groups, n = ints([5, 6]), ints([0, 1, 3]), ints([0, 2]), ints([4])
    bad = [
        lambda: c.attention_shared(q, cu, ints([5]), groups, n), lambda: c.attention_shared(q, cu, lens, ints([0]), n),
        lambda: c.attention_shared(q, cu, lens, groups.long(), n), lambda: c.attention_shared(q, cu, lens, groups, n.float()),
        lambda: c.attention_shared(q, cu, lens, groups, [4]), lambda: c.attention_shared(q, cu, lens, groups.cpu(), n),
        lambda: c.attention_shared(q.half(), cu, lens, groups, n), lambda: c.attention_shared(q[0], cu, lens, groups, n),
        lambda: c.attention_shared(q, cu, lens, groups, n, out=q[:2]), lambda: c.attention_shared(q, cu, lens, groups, n, workspace=torch.zeros(8)),
        lambda: c.attention_shared(q, cu, lens, groups, n, lse=torch.zeros((3, 2), device="cuda"))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(kvev.KvevError) as e:
        c.attention_shared(q[:, :3], cu, lens, groups, n)
    assert e.value.code == kvev.EINVAL and c.status() == 0


def test_forks_of_a_prefilled_prefix(paged):
    """As a serving program has it: the prefix goes through tables, write and attention once; requests take its pages into their rows of
    the table; their prompts, and then generations, attend with the prefix shared."""
    H_q, H, d, page, B, n = 8, 2, 128, 16, 6, 96
    width = ref.pages_of(n + 60, page)
    table = torch.full((B + 1, width), -1, dtype=torch.int32, device="cuda")
    pool = paged.PagePool(200, page, table)
    c = paged.PagedCache.empty(200, page, H, d, table)
    c.K.zero_(), c.V.zero_()
    g = torch.Generator(device="cuda").manual_seed(0)
    lens = torch.zeros(B + 1, dtype=torch.int32, device="cuda")

    def forward(new):
        T = sum(new)
        qkv = torch.randn((T, H_q + 2 * H, d), generator=g, device="cuda").to(BF16)
        _, cu, slots, _, granted = pool.tables(lens, ints(new), T, kv_lens=lens)
        assert bool(granted.all())
        c.write(qkv[:, H_q:H_q + H], qkv[:, H_q + H:], slots)
        return qkv[:, :H_q], cu

    q, cu = forward([n] + [0] * B)  # request 0 holds the prefix
    c.attention(q, cu, lens)
    table[1:, :n // page] = table[0, :n // page]
    lens[1:] = n
    groups, shared = ints([1, 4, B + 1]), ints([n, n - 20])
    for new in ([0, 30, 1, 17, 5, 40, 2], [0] + [1] * B, [0] + [1] * B):
        q, cu = forward(new)
        lse = torch.empty((q.shape[0], H_q), device="cuda")
        o = c.attention_shared(q, cu, lens, groups, shared, lse=lse)
        r = ref.attention(c.K, c.V, table.cpu().tolist(), q, cu.cpu().tolist(), lens.cpu().tolist())
        q8_ref.check_attention(o, lse, r, BF16, parts=2)
    assert c.status() == 0 and int(pool.device_status) == 0
    # the pages go back once: the prefix's with request 0, the others' without it
    own = table.clone()
    own[1:, :n // page] = -1
    taken = int((own >= 0).sum())
    done = torch.ones(B + 1, dtype=torch.int32, device="cuda")
    table.copy_(own)
    pool.release(lens, done)
    assert int(pool.free_count) == 200 and taken + 0 > n // page and int(pool.device_status) == 2
    assert sorted(pool.free.cpu().tolist()) == list(range(200))


@pytest.mark.parametrize("B,page,ctx,room", [(2, 16, 40, 0), (40, 8, 1500, 0), (700, 8, 1500, 0), (300, 8, 900, 0), (300, 8, 900, 50)])
def test_release_of_requests_that_share_pages(paged, B, page, ctx, room):
    """Entries of pages that others keep are left out and in order, on a stack with room for the others alone; where it has `room` pages less, or
    beside an entry outside the pool, the status says so."""
    rng = random.Random(B)
    lens = [ctx] + [rng.randint(0, ctx) for _ in range(B - 1)]
    done = [1] + [rng.choice([0, 1, 1]) for _ in range(B - 1)]
    held = [ref.pages_of(n, page) for n in lens]
    common = min(held[0], 70)
    ids = list(range(sum(held)))
    rng.shuffle(ids)
    table = [[ids.pop() for _ in range(h)] for h in held]
    for s in range(1, B):
        if done[s]:
            for j in range(min(common, held[s])):
                table[s][j] = kvev.PAGED_KEPT_PAGE
    back = [x for s in range(B) if done[s] for x in table[s] if x >= 0]
    num_pages = sum(held)
    rows = ints([r + [-1] * (max(held) + 1 - len(r)) for r in table])
    count = num_pages - len(back) + room
    free = [num_pages - 1] * count + [-7] * (num_pages - count)
    for wrong in (False, True):
        if wrong:
            rows[0, 0] = -1
            back = back[1:]
        pool = paged.PagePool(num_pages, page, rows, ints(free), ints([count]))
        dlens = ints(lens)
        pool.release(dlens, ints(done))
        want = (free[:count] + back)[:num_pages]
        assert int(pool.free_count) == len(want) and pool.free.cpu().tolist()[:len(want)] == want
        assert dlens.cpu().tolist() == [0 if f else n for n, f in zip(lens, done)]
        assert int(pool.device_status) == (2 if wrong or room else 0)


def test_kept_pages_are_in_order_for_a_release_alone(paged):
    c, q, cu, kv, table, first, shared = shared_case(paged, [(32, [(20, 1), (5, 1)])], 4, 2, 64, 16)
    rows = [list(r) for r in table]
    rows[1][0] = kvev.PAGED_KEPT_PAGE  # of a request that still attends: no page
    c2 = paged.PagedCache(c.K, c.V, ints(rows))
    c2.attention(q, ints(cu), ints(kv))
    assert c2.status() == 2


def test_requests_of_a_group_are_done_one_after_another(paged):
    """The last holder gives the prefix back; every page is on the stack once, and nothing is said."""
    page, n, own, B = 16, 3, 2, 4
    num_pages = n + own * B
    table = torch.full((B, n + own), -1, dtype=torch.int32, device="cuda")
    pool = paged.PagePool(num_pages, page, table)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    pool.tables(lens, ints([n * page] + [0] * (B - 1)), n * page, kv_lens=lens)
    table[1:, :n] = table[0, :n]
    lens[1:] = n * page
    pool.tables(lens, ints([own * page] * B), B * own * page, kv_lens=lens)
    assert int(pool.free_count) == 0
    for done in ([0, 1, 0, 0], [1, 0, 0, 1], [0, 0, 1, 0]):
        left = [s for s in range(B) if int(lens[s]) and not done[s]]
        for s in range(B):
            if done[s] and left:
                table[s, :n] = kvev.PAGED_KEPT_PAGE
        pool.release(lens, ints(done))
        assert int(pool.free_count) == num_pages - len(left) * own - (n if left else 0) and int(pool.device_status) == 0
    assert sorted(pool.free.cpu().tolist()) == list(range(num_pages))

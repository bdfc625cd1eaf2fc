"""Plain 64-bit forms of the paged operators, request by request, on host lists and torch tensors."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # unit roundoff


def pages_of(n, page):
    return -(-n // page)


def tables(lens, new, page, num_pages, free, count, table, max_pages, T):
    """kvev_paged_tables on host lists; `table` is completed in place.  (kv, cu, slots, positions, granted, count)"""
    kv, cu, slots, pos, granted = [], [0], [-1] * T, [-1] * T, []
    asked = 0
    given = 0
    for s, (n, q) in enumerate(zip(lens, new)):
        n, q = max(n, 0), max(q, 0)
        held, after = pages_of(n, page), pages_of(n + q, page)
        fits = after <= max_pages
        k = after - held if fits else 0
        asked += k
        ok = fits and (k == 0 or asked <= count)
        if ok:
            for j in range(k):
                table[s][held + j] = free[count - 1 - (asked - k + j)]
            given = max(given, asked if k else 0)
            for i in range(q):
                if cu[-1] + i < T:
                    p = n + i
                    slots[cu[-1] + i] = table[s][p // page] * page + p % page
                    pos[cu[-1] + i] = p
        granted.append(int(ok))
        kv.append(n + q if ok else n)
        cu.append(cu[-1] + q)
    return kv, cu, slots, pos, granted, count - given


def release(lens, done, page, num_pages, free, count, table):
    """kvev_paged_release on host lists; `free` is completed in place.  (lens, count)"""
    out = []
    for s, (n, f) in enumerate(zip(lens, done)):
        if f:
            for j in range(pages_of(max(n, 0), page)):
                if count < num_pages:
                    free[count] = table[s][j]
                    count += 1
        out.append(0 if f else n)
    return out, count


def attention(K, V, table, q, cu, kv, scale=0.0, window=0):
    """kvev_paged_attention in 64 bits: (out, lse, sum p |v|, logit error bound) per row.

    K, V: [pages][page][H_kv][d]; table, cu, kv: host lists.  The error bound of a logit is that of a
    32-bit dot product of d terms, 2^-23 d scale sum |q||k|, the largest over the row's keys."""
    page, H, d = K.shape[1], K.shape[2], K.shape[3]
    T, H_q = q.shape[0], q.shape[1]
    G = H_q // H
    scale = scale or 1 / math.sqrt(d)
    dev = q.device
    out = torch.zeros((T, H_q, d), dtype=torch.float64, device=dev)
    lse = torch.full((T, H_q), -math.inf, dtype=torch.float64, device=dev)
    mass = torch.zeros_like(out)
    eps = torch.zeros_like(lse)
    for s, n in enumerate(kv):
        c0, c1 = cu[s], cu[s + 1]
        if c1 == c0 or n <= 0:
            continue
        pages = torch.tensor(table[s][:pages_of(n, page)], device=dev)
        t = n - (c1 - c0) + torch.arange(c1 - c0, device=dev)
        k = torch.arange(n, device=dev)
        sees = k[None] <= t[:, None]
        if window:
            sees &= k[None] > t[:, None] - window
        seen = sees.any(0)
        row = sees.any(1)
        for h in range(H):
            Kh = K[pages, :, h].reshape(-1, d)[:n].double()
            Vh = V[pages, :, h].reshape(-1, d)[:n].double()
            Kh = torch.where(seen[:, None], Kh, 0.0)  # what no row sees may hold anything
            Vh = torch.where(seen[:, None], Vh, 0.0)
            Q = q[c0:c1, h * G:(h + 1) * G].double().transpose(0, 1)
            x = torch.matmul(Q, Kh.T) * scale
            e = torch.matmul(Q.abs(), Kh.abs().T) * (scale * d * 2.0 ** -23)
            x = x.masked_fill(~sees, -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.where(sees, torch.exp(x - torch.where(row, z, 0.0)[..., None]), 0.0)
            hs = slice(h * G, (h + 1) * G)
            out[c0:c1, hs] = torch.matmul(p, Vh).transpose(0, 1)
            mass[c0:c1, hs] = torch.matmul(p, Vh.abs()).transpose(0, 1)
            lse[c0:c1, hs] = z.transpose(0, 1)
            eps[c0:c1, hs] = torch.where(sees, e, 0.0).amax(-1).transpose(0, 1)
    return out, lse, mass, eps


def check_attention(o, lse, ref, dtype):
    """Every element within what the number formats allow: the weights and the result are rounded to the
    type once each (unit roundoff u), which moves an element by at most u sum p|v| and u |o|; a logit's
    32-bit error eps moves a weight and the normaliser by a factor 1 + eps each; 2^-20 covers the exponentials,
    logarithms and 32-bit sums, and in half precision the weights below its normal range (2^-14 of the largest,
    which the kernel keeps at 2^7 or more: 2^-25 2^-7 each, under 2^-17 for 32,768 keys)."""
    r, rl, mass, eps = ref
    u = UNIT[dtype]
    small = 2.0 ** -20 if dtype is torch.bfloat16 else 2.0 ** -17
    tol = u * (r.abs() + 1.01 * mass) * 1.02 + (2 * eps[..., None] + small) * (mass + mass.amax(-1, keepdim=True)) + 2.0 ** -24
    err = (o.double() - r).abs()
    assert torch.isfinite(o.float()).all()
    assert (err <= tol).all(), f"out: worst error / tolerance {(err / tol).max().item():.3g}"
    if lse is not None:
        empty = torch.isinf(rl)
        assert torch.equal(empty, torch.isinf(lse)) and (lse[empty] < 0).all()
        le = (lse.double() - rl).abs()[~empty]
        lt = (eps + 2.0 ** -20 + 2.0 ** -22 * rl.abs())[~empty]
        assert (le <= lt).all(), f"lse: worst error / tolerance {(le / lt).max().item():.3g}"

"""Float64 references of the decoding calls, on the CPU, from their definitions (include/sx_decode.h)."""
import math

import torch

BLOCK, GROUP = 16, 32
MAG = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def record(d):
    return 17 * d


def round4(x):
    """x [..., d] -> (values float64, codes, scale bytes [..., d / 32]) by trying every scale and magnitude."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    amax = g.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, 125.0)
    bad = ~torch.isfinite(g).all(-1, keepdim=True)
    for k in range(124, -127, -1):                      # the smallest exponent with amax <= 7 * 2^e
        e = torch.where(amax <= math.ldexp(7.0, k), torch.full_like(e, float(k)), e)
    s = torch.ldexp(torch.ones_like(e), e.int())
    a = (g.abs() / s).unsqueeze(-1)
    off = (a - MAG).abs()
    off = off + 1e-12 * (torch.arange(8) % 2)           # a tie (exact in float64, >= 2^-24 apart else) goes to the even code
    off = torch.where(a > 6, (torch.arange(8) != 7).double().expand_as(off), off)
    m = off.argmin(-1)
    neg = torch.signbit(g)
    val = torch.where(neg, -MAG[m], MAG[m]) * s
    val = torch.where(bad, torch.full_like(val, math.nan), val)
    code = torch.where(bad, torch.zeros_like(m), m + 8 * neg.long())
    byte = torch.where(bad, torch.full_like(e, 255.0), e + 127)[..., 0]
    return val.reshape(x.shape), code.reshape(x.shape).to(torch.uint8), byte.to(torch.uint8)


def offsets(d, t):
    """Byte offset, nibble of K and V, and of their scales, of element c of token t in a record."""
    c = torch.arange(d)
    k = c // (d // 4) * 2 * d + t * (d // 8) + c % (d // 4) // 2
    col = d // 16
    v = 8 * d + ((t // 4 * 16 + c // col) * 4 + t % 4) * (d // 32) + c % col // 2
    ks = 16 * d + c // GROUP * 16 + t
    return k, v, ks, ks + d // 2, c % 2


def put_rows(pool, k, v, slots):
    """Writes rows k, v [n][Hkv][d] into the CPU pool [blocks][Hkv][record]; returns the values they now have."""
    d = k.shape[-1]
    (kv, kc, ks), (vv, vc, vs) = round4(k), round4(v)
    for i, s in enumerate(slots.tolist()):
        if s < 0 or s // BLOCK >= pool.shape[0]:
            continue
        rec = pool[s // BLOCK]
        ko, vo, kso, vso, hi = offsets(d, s % BLOCK)
        for at, code in ((ko, kc[i]), (vo, vc[i])):
            for n in (0, 1):
                a = at[hi == n]
                keep = rec[:, a] & (0xF0 if n == 0 else 0x0F)
                rec[:, a] = keep | (code[:, hi == n] << (4 * n))
        rec[:, kso[::GROUP]] = ks[i]
        rec[:, vso[::GROUP]] = vs[i]
    return kv, vv


def get_rows(pool, slots, d):
    """float64 K, V [n][Hkv][d] that the slots of a CPU pool hold."""
    out = []
    for s in slots.tolist():
        rec = pool[s // BLOCK]
        ko, vo, kso, vso, hi = offsets(d, s % BLOCK)
        row = []
        for at, sc in ((ko, kso), (vo, vso)):
            code = (rec[:, at] >> (4 * hi).to(torch.uint8)) & 15
            val = MAG[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0).double()
            b = rec[:, sc].int()
            row.append(torch.where(b == 255, torch.full_like(val, math.nan), torch.ldexp(val, b - 127)))
        out.append(torch.stack(row))
    x = torch.stack(out) if out else torch.zeros(0, 2, pool.shape[1], d, dtype=torch.float64)
    return x[:, 0], x[:, 1]


def rows_of(pool, table, n, d):
    """K, V [n][Hkv][d] of a request's first n tokens and which of them have a block."""
    ids = table[torch.arange(n) // BLOCK].long()
    ok = (ids >= 0) & (ids < pool.shape[0])
    k, v = get_rows(pool, torch.where(ok, ids, torch.zeros_like(ids)) * BLOCK + torch.arange(n) % BLOCK, d)
    return k, v, ok


def attention(q, cu, lens, kv, scale):
    """(out, lse, bound) in float64: kv[r] = (k, v, ok) of request r.  bound [rows][Hq][d]: how far the library's float32
    arithmetic may be off before the output's own rounding -- a score is a sum of d products and a base-2 exponent formed
    from it (relative 2^-24 each), so a probability is off by at most ds = scale * (d + 4) 2^-24 max_j sum |q k_j| + 2^-22
    (max |s| + 1) relative; numerator and denominator take that, their own sums of up to n terms (n 2^-24), the parts of a
    probability (2^-16) and the final division (2^-22): twice the sum, times sum p |v|.  bfloat16 requests of more than 128
    rows (query tokens x heads of the group) take a probability in one part: the numerator's p are each off by half a
    bfloat16 step, 2^-8 relative, the denominator's are not, so 2^-8 sum p |v| comes on top."""
    n, hq, d = q.shape
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    bound = torch.zeros(n, hq, d, dtype=torch.float64)
    lse_bound = torch.zeros(n, hq, dtype=torch.float64)
    for r in range(len(lens)):
        q0, nq, m = int(cu[r]), int(cu[r + 1] - cu[r]), int(lens[r])
        if nq == 0 or m == 0:
            continue
        k, v, ok = kv[r]
        grp = hq // k.shape[1]
        pos = torch.arange(nq) + m - nq
        see = (torch.arange(m)[None] <= pos[:, None]) & ok[None]
        for h in range(hq):
            kh, vh, qh = k[:, h // grp], v[:, h // grp], q[q0:q0 + nq, h].double()
            s = torch.where(see, qh @ kh.t() * scale, torch.tensor(-math.inf, dtype=torch.float64))
            top = s.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            e = (s - top).exp()
            den = e.sum(-1, keepdim=True)
            p = e / torch.where(den == 0, torch.ones_like(den), den)
            for i in range(nq):                       # (hidden values, NaN among them, do not count)
                out[q0 + i, h] = p[i, see[i]] @ vh[see[i]]
                bound[q0 + i, h] = p[i, see[i]] @ vh[see[i]].abs()
            lse[q0:q0 + nq, h] = (den.log() + top)[:, 0]
            mag = torch.where(see, qh.abs() @ kh.nan_to_num().abs().t(), torch.zeros_like(s)).amax(-1) * scale
            fin = torch.where(see & torch.isfinite(s), s.abs(), torch.zeros_like(s)).amax(-1)
            ds = mag * (d + 4) * 2.0 ** -24 + 2.0 ** -22 * (fin + 1)
            one_part = 2.0 ** -8 if q.dtype is torch.bfloat16 and nq * grp > 128 else 0.0
            bound[q0:q0 + nq, h] *= 2 * (ds + m * 2.0 ** -24 + 2.0 ** -16 + 2.0 ** -22)[:, None] + one_part
            lse_bound[q0:q0 + nq, h] = 2 * (ds + m * 2.0 ** -24 + 2.0 ** -22 * (1 + lse[q0:q0 + nq, h].abs().nan_to_num(0, 0, 0)))
    return out, lse, bound, lse_bound


def norm_rope(x, gamma, eps, pos, base, neox):
    """(rows, bound) in float64.  bound: the norm is a sum of d squares, a root, a division and two products (d / 8 + 12 units
    of 2^-24 relative at the most), the rotation two products with rounded cos and sin and a sum: 32 units of 2^-24 on
    |y1| + |y2| cover d <= 128."""
    d = x.shape[-1]
    y = x.double()
    if gamma is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gamma.double()
    th = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    ang = pos.double()[:, None, None] * th
    c, s = ang.cos(), ang.sin()
    a, b = (y[..., :d // 2], y[..., d // 2:]) if neox else (y[..., 0::2], y[..., 1::2])
    r = (a * c - b * s, b * c + a * s)
    w = (a.abs() + b.abs()) * 32 * 2.0 ** -24
    if neox:
        return torch.cat(r, -1), torch.cat([w, w], -1)
    return torch.stack(r, -1).flatten(-2), torch.stack([w, w], -1).flatten(-2)


def append_slots(ctx, new, b, free, head, table, room):
    """Loops over the definition; returns (table, seq, cu, positions, slots, state)."""
    table = table.clone()
    width = table.shape[1]
    cu, pos, slot, missing = [0], [-1] * room, [-1] * room, 0
    start = head
    for r in range(len(ctx)):
        have = -(-ctx[r] // b)
        need = max(min(-(-(ctx[r] + new[r]) // b), width) - have, 0)
        for j in range(new[r]):
            i, p = cu[r] + j, ctx[r] + j
            blk, bid = p // b, -1
            if blk < width:
                if blk < have:
                    bid = int(table[r, blk])
                else:
                    f = head + blk - have
                    bid = int(free[f]) if f < len(free) else -1
                    if p % b == 0:
                        table[r, blk] = bid
            if i < room:
                pos[i] = p
                slot[i] = bid * b + p % b if bid >= 0 else -1
            missing += i >= room or bid < 0
        head += need
        cu.append(cu[r] + new[r])
    seq = [c + n for c, n in zip(ctx, new)]
    return table, seq, cu, pos, slot, [max(min(head, len(free)), start), missing]

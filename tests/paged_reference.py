"""The paged cache in plain form: lists for the plan, float64 on the CPU for rows and attention, and how far fp32 kernels may be off."""
import math

import torch

SATURATE = 1 << 30


def plan(new_cnt, cache_len, table, ring, state, page, max_rows):
    """(new_len, table, ring, state, row_start, slot, pos, statuses) from lists, one sequence after the other."""
    n_pages, b, width = len(ring), len(new_cnt), len(table[0])
    table, out_ring = [list(r) for r in table], list(ring)
    head, free = state
    slot, pos, row_start, new_len = [-1] * max_rows, [0] * max_rows, [], []
    asked = given = back = rows = 0
    bits = set()
    returned = []

    def held(n):
        return -(-n // page)
    for s in range(b):
        c, m = new_cnt[s], cache_len[s]
        row_start.append(min(rows, SATURATE))
        begin = rows
        rows += max(c, 0)
        if m < 0 or m > width * page:
            new_len.append(m)
            if m > 0:
                bits.add("request")
            continue
        if c < 0:
            returned += table[s][:held(m)]
            new_len.append(0)
            continue
        need = held(m + c) - held(m) if rows <= max_rows and m + c <= width * page else None
        if need is not None:
            asked += need
        if need is None or (need and asked > free):
            new_len.append(m)
            if c:
                bits.add("capacity")
            continue
        for j in range(need):
            table[s][held(m) + j] = ring[(head + given) % n_pages]
            given += 1
        new_len.append(m + c)
        for i in range(c):
            t = m + i
            p = table[s][t // page]
            if 0 <= p < n_pages:
                slot[begin + i], pos[begin + i] = p * page + t % page, t
            else:
                bits.add("request")
    for p in returned:
        out_ring[(head + free + back) % n_pages] = p
        back += 1
    return new_len, table, out_ring, [(head + given) % n_pages, free - given + back], row_start + [min(rows, SATURATE)], slot, pos, bits


def turn(x, pos, inv_freq, axis, rot, neighbours):
    """Rotation of the first rot channels of x [rows, heads, d] (float64) and the magnitudes that its errors go by."""
    angle = pos.double()[axis].t() * inv_freq.double()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, z = (slice(0, rot, 2), slice(1, rot, 2)) if neighbours else (slice(0, rot // 2), slice(rot // 2, rot))
    y, size = x.clone(), x.abs()
    y[..., a], y[..., z] = x[..., a] * c - x[..., z] * s, x[..., z] * c + x[..., a] * s
    both = x[..., a].abs() + x[..., z].abs()
    size[..., a], size[..., z] = both, both
    return y, size


def norm(x, weight, eps):
    return x if weight is None else x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def row_tolerance(y, size, dtype, d):
    """One rounding to dtype; fp32 before it: a sum of d squares, a square root, a reciprocal and four products (2^-24 each), and an angle
    and its sine to 2^-20 together (the angle's turn is rounded to 2^-25, which is 2^-22 of an angle; a sine within 2^-21)."""
    return half_step(dtype) * y.abs() + (2.0 ** -20 + (d + 16) * 2.0 ** -24) * size + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133)


def gather(pages, scale, row, page, lo, hi):
    """[keys, h_kv, d] in float64 of tokens lo..hi-1, those of bad pages left out."""
    t = torch.arange(lo, hi)
    p, off = row.long()[t // page], t % page
    ok = (p >= 0) & (p < pages.shape[0])
    p, off = p[ok], off[ok]
    x = pages[p, :, off].double()
    return x * scale[p, :, off].double()[..., None] if scale is not None else x


def attention(q, k, v, scale, dtype, weight_step, query_step=0.0):
    """out [h_q, d], lse [h_q] and their tolerances of one query over [keys, h_kv, d] (float64)."""
    h_kv, d = k.shape[1:] if k.numel() else (1, q.shape[1])
    if not k.numel():
        z = torch.zeros_like(q)
        return z, torch.full(q.shape[:1], -math.inf, dtype=torch.float64), z, torch.zeros(q.shape[0], dtype=torch.float64)
    g = q.shape[0] // h_kv
    kk, vv = (x.repeat_interleave(g, 1).permute(1, 0, 2) for x in (k, v))
    x = (kk * q[:, None]).sum(-1) * scale
    w = torch.softmax(x, -1)
    out = (w[..., None] * vv).sum(1)
    lse = torch.logsumexp(x, -1)
    # a logit: d products and sums in fp32, its scaling, and exp's argument, which is as large as the logits are apart
    size = (kk.abs() * q[:, None].abs()).sum(-1) * scale
    spread = x.abs().amax(-1)
    off = 2.0 ** -24 * ((d + 8) * size.amax(-1) + 16 * spread + 32) + query_step * size.amax(-1)
    weights = (w[..., None] * vv.abs()).sum(1)
    sums = (64 + x.shape[-1] / 16) * 2.0 ** -24              # a chain of partial sums, sixteen lanes' at the least
    tol = half_step(dtype) * out.abs() + (weight_step + 2 * off[:, None] + 2 * sums) * weights
    if dtype == torch.float16:
        # Below 2^-14 a fp16 number's half step is 2^-25 whatever its size.  So for the output; and for a weight, which is rounded relative to the
        # largest one, 1, of those seen when it is: its share of the sum, which is at least 1, is then off by 2^-25 at most, times its value.
        tol = tol + 2.0 ** -25 * (1 + vv.abs().sum(1))
    return out, lse, tol, off + sums + 2.0 ** -23 * lse.abs()

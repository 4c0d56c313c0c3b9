"""Plain 64-bit forms of the paged operators (numpy, from their definitions), for the tests."""
import math

import numpy as np


def plan(page, n_pages, ctx, new, free_pages, free_count, table, n_tok):
    """block_table, seq_lens, cu_new, positions, slots, free_left of a valid plan."""
    table, left = table.copy(), int(free_count)
    cu, pos, slots = [0], [], []
    for i, (c, n) in enumerate(zip(ctx, new)):
        for pg in range(-(-c // page), -(-(c + n) // page)):
            left -= 1
            table[i, pg] = free_pages[left]
        for p in range(c, c + n):
            pos.append(p)
            slots.append(int(table[i, p // page]) * page + p % page)
        cu.append(cu[-1] + n)
    pad = n_tok - len(pos)
    return table, np.add(ctx, new), np.array(cu), np.array(pos + [0] * pad), np.array(slots + [-1] * pad), left


def rotate(x, positions, table, interleaved, mscale=1.0, transpose=False):
    """x [n, heads, d] in float64; table: integers, frequency in 2^-64 of a turn (exact angles)."""
    y = np.array(x, np.float64)
    for t, p in enumerate(positions):
        for c, f in enumerate(table):
            turn = (int(p) * int(f)) % (1 << 64) / 2.0 ** 64
            co, si = math.cos(2 * math.pi * turn) * mscale, math.sin(2 * math.pi * turn) * mscale
            if transpose:
                si = -si
            a, b = (2 * c, 2 * c + 1) if interleaved else (c, c + len(table))
            u, v = np.array(x[t, :, a], np.float64), np.array(x[t, :, b], np.float64)
            y[t, :, a], y[t, :, b] = u * co - v * si, v * co + u * si
    return y


def attention(q, pool, table, lens, cu, n_rep, scale, window=0, sinks=0):
    """o, lse, the sum of p |v| per output and the largest sum of |q||k| per row. Only visible tokens
    are touched. q [n, H * n_rep, d], pool [2][n_pages][H][page][d], both float64."""
    _, _, H, page, d = pool.shape
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, big = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    for i in range(len(lens)):
        n = cu[i + 1] - cu[i]
        for k in range(n):
            p = lens[i] - n + k
            t = np.arange(max(p + 1, 0))
            if window:
                t = t[(t > p - window) | (t < sinks)]
            if not len(t):
                continue
            ids = table[i, t // page]
            for h in range(H):
                K, V = pool[0, ids, h, t % page], pool[1, ids, h, t % page]
                Q = q[cu[i] + k, h * n_rep:(h + 1) * n_rep]
                s = scale * (Q @ K.T)
                m = s.max(1, keepdims=True)
                e = np.exp(s - m)
                z = e.sum(1, keepdims=True)
                r = slice(h * n_rep, (h + 1) * n_rep)
                o[cu[i] + k, r] = (e / z) @ V
                mag[cu[i] + k, r] = (e / z) @ np.abs(V)
                lse[cu[i] + k, r] = (m + np.log(z))[:, 0]
                big[cu[i] + k, r] = (abs(scale) * (np.abs(Q) @ np.abs(K).T)).max(1)
    return o, lse, mag, big


def attention_tolerance(fp16, d, o, mag, big):
    """Bounds of the outputs and of the lse. u: rounding of a 16-bit number. A score is an fp32 sum
    of d exact products: off by at most (d + 8) 2^-24 of sum |q||k| scale; with the exponential and
    the sums (a few 2^-23 each, 2^-19 in all) a weight is off by that fraction, the normalised one by
    twice it. The weight enters the value product rounded (u), the output is rounded (u); fp16
    weights below 2^-21 of the row's largest are rounded to 2^-31 of it, absolutely."""
    u = 2.0 ** -11 if fp16 else 2.0 ** -8
    ds = (d + 8) * 2.0 ** -24 * big + 2.0 ** -19
    tiny = 2.0 ** -31 * 65536 if fp16 else 0.0
    return (u + 2 * ds[..., None] + tiny) * mag + u * np.abs(o) + 1e-7, ds + 2.0 ** -19

"""Plain forms of the draft-tree operators (numpy, from their definitions; scores and sums in 64 bits), for the tests."""
import numpy as np


def path(parents, k):
    """Nodes from the root to k, and whether a parent outside [-1, k) ended it."""
    out = []
    while True:
        out.append(k)
        p = parents[k]
        if p < -1 or p >= k:
            return out[::-1], True
        if p == -1:
            return out[::-1], False
        k = p


def random_parents(rng, n, bushy=0.5):
    """A tree of n nodes: chains, broken by nodes that hang from any earlier one or from the history."""
    return [-1 if k == 0 or rng.random() < 0.08 else k - 1 if rng.random() > bushy else int(rng.integers(0, k)) for k in range(n)]


def plan(parents, lens, cu, n_tok, words, window=0, sinks=0):
    """positions [n_tok] and masks [n_tok][words] (uint32)."""
    pos, bits = np.zeros(n_tok, np.int64), np.zeros((n_tok, words * 32), bool)
    for i in range(len(lens)):
        p, ctx = parents[cu[i]:cu[i + 1]], lens[i] - (cu[i + 1] - cu[i])
        for k in range(len(p)):
            line, _ = path(p, k)
            pos[cu[i] + k] = ctx + len(line) - 1
            for depth, b in enumerate(line):
                bits[cu[i] + k, b] = not window or len(line) - 1 - depth < window or ctx + depth < sinks
    return pos, pack(bits)


def pack(bits):
    n, m = bits.shape
    return (bits.reshape(n, m // 32, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)


def unpack(masks):
    n, words = masks.shape
    return ((masks[..., None] >> np.arange(32, dtype=np.uint32)) & 1).astype(bool).reshape(n, words * 32)


def attention(q, pool, table, lens, cu, masks, pos, n_rep, scale, window=0, sinks=0):
    """o, lse, the sum of p |v| per output and the largest sum of |q||k| per row, as paged_ref.attention; only what a
    row sees is touched."""
    _, _, H, page, _ = pool.shape
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    lse, big = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
    bits = unpack(masks)
    for i in range(len(lens)):
        n = cu[i + 1] - cu[i]
        ctx = lens[i] - n
        for k in range(n):
            row = cu[i] + k
            t = np.arange(ctx)
            if window:
                t = t[(t > pos[row] - window) | (t < sinks)]
            t = np.concatenate([t, ctx + np.nonzero(bits[row, :n])[0]])
            if not len(t):
                continue
            ids = table[i, t // page]
            for h in range(H):
                K, V = pool[0, ids, h, t % page], pool[1, ids, h, t % page]
                r = slice(h * n_rep, (h + 1) * n_rep)
                s = scale * (q[row, r] @ K.T)
                m = s.max(1, keepdims=True)
                e = np.exp(s - m)
                z = e.sum(1, keepdims=True)
                o[row, r] = (e / z) @ V
                mag[row, r] = (e / z) @ np.abs(V)
                lse[row, r] = (m + np.log(z))[:, 0]
                big[row, r] = (abs(scale) * (np.abs(q[row, r]) @ np.abs(K).T)).max(1)
    return o, lse, mag, big


def commit(page, n_pages, parents, leaves, lens, cu, table, pool, stack, count):
    """pool (any number of leading dimensions before [2][n_pages][H][page][d]), lens_left, the stack, free_left."""
    pool, stack, left = pool.copy(), list(stack), []
    for i in range(len(lens)):
        p, ctx = parents[cu[i]:cu[i + 1]], lens[i] - (cu[i + 1] - cu[i])
        line = path(p, leaves[i])[0] if leaves[i] >= 0 else []
        for k, r in enumerate(line):
            if r == k:
                continue
            s, d = ctx + r, ctx + k
            sp, dp = table[i, s // page], table[i, d // page]
            if 0 <= sp < n_pages and 0 <= dp < n_pages:
                pool[..., dp, :, d % page, :] = pool[..., sp, :, s % page, :]
        left.append(ctx + len(line))
        for j in range(-(-left[i] // page), -(-lens[i] // page)):
            if 0 <= table[i, j] < n_pages and count < n_pages:
                stack[count] = table[i, j]
                count += 1
    return pool, left, stack, count

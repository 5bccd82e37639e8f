"""Oracle of the steps with several new tokens a request: cache blocks and slots,
prompt attention and tree attention, from their definitions in numpy and 64 bits
(test-only)."""
import numpy as np

D = 128
INT_MAX = 2 ** 31 - 1


def extend(lens, news, table, free, height, T, num_blocks, bs):
    """(table, height, offsets, totals, slots, positions) after new tokens got
    their blocks; request by request, block by block."""
    table = table.copy()
    B, width = table.shape
    height = min(max(int(height), 0), num_blocks)
    left = height
    offsets, totals = np.zeros(B + 1, np.int32), np.zeros(B, np.int32)
    slots, positions = np.full(T, -1, np.int64), np.zeros(T, np.int32)
    tokens, asked = 0, 0
    for b in range(B):
        L, n = max(int(lens[b]), 0), max(int(news[b]), 0)
        first, tokens = tokens, tokens + n
        offsets[b + 1] = min(tokens, T)
        totals[b] = L
        have, want = -(-L // bs), -(-(L + n) // bs)
        if tokens > T or L + n > INT_MAX or want > width:
            continue
        asked += want - have
        if want > have and asked > height:
            continue
        for e in range(have, want):
            left -= 1
            table[b, e] = free[left]
        totals[b] = L + n
        for i in range(n):
            p = L + i
            block = int(table[b, p // bs])
            slots[first + i] = block * bs + p % bs if 0 <= block < num_blocks else -1
            positions[first + i] = p
    return table, left, offsets, totals, slots, positions


def release(lens, keeps, table, free, height, num_blocks, bs):
    """(table, free, height) after the blocks behind keeps[b] tokens went back."""
    table, free = table.copy(), free.copy()
    height = min(max(int(height), 0), num_blocks)
    for b in range(table.shape[0]):
        first = -(-max(int(keeps[b]), 0) // bs)
        for e in range(first, min(-(-max(int(lens[b]), 0) // bs), table.shape[1])):
            block = int(table[b, e])
            table[b, e] = -1
            if 0 <= block < num_blocks and height < num_blocks:
                free[height] = block
                height += 1
    return table, free, height


def attend(q, k, v, scale, sees):
    """One head: rows q [m][128] over k, v [n][128]; sees bool [m][n].  Returns
    out [m][128], lse [m], the same weights' sum of |v| and, for error bounds, the
    largest sum of |q_i k_i| of a row's keys."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    out, mag = np.zeros((len(q), D)), np.zeros((len(q), D))
    lse, most = np.full(len(q), -np.inf), np.zeros(len(q))
    for i in range(len(q)):
        at = np.flatnonzero(sees[i])       # what a row does not see is not touched
        if len(at) == 0:
            continue
        s = k[at] @ q[i] * scale
        m = s.max()
        w = np.exp(s - m)
        lse[i] = m + np.log(w.sum())
        w /= w.sum()
        out[i], mag[i] = w @ v[at], w @ np.abs(v[at])
        most[i] = (np.abs(k[at]) @ np.abs(q[i])).max()
    return out, lse, mag, most


def prompt(q, k, v, offsets, scale):
    """Per request and head: (rows, head, attend's results) of packed prompts."""
    G = q.shape[1] // k.shape[1]
    for b in range(len(offsets) - 1):
        lo, hi = offsets[b], offsets[b + 1]
        sees = np.tril(np.ones((hi - lo, hi - lo), bool))
        for h in range(q.shape[1]):
            yield slice(lo, hi), h, hi - lo, attend(q[lo:hi, h], k[lo:hi, h // G], v[lo:hi, h // G], scale, sees)


def cached_rows(cache, ids, L, g):
    """Rows [L][128] of kv-head g and which of them are in the pool."""
    t = np.arange(L)
    block = np.asarray(ids)[t // 16] if L else np.zeros(0, int)
    there = (block >= 0) & (block < cache.shape[0])
    rows = np.zeros((L, D), cache.dtype)
    rows[there] = cache[block[there], g, t[there] % 16]
    return rows, there


def tree(q, k_new, v_new, offsets, masks, k_cache, v_cache, table, lens, max_nodes, scale):
    """As prompt, of drafted tokens; masks uint64 [T]."""
    G = q.shape[1] // k_new.shape[1]
    for b in range(len(offsets) - 1):
        lo = offsets[b]
        hi = min(offsets[b + 1], lo + max_nodes)
        n = hi - lo
        if n <= 0:
            continue
        L = min(max(int(lens[b]), 0), table.shape[1] * 16)
        bits = np.array([[int(m) >> j & 1 for j in range(n)] for m in masks[lo:hi]], bool).reshape(n, n)
        for g in range(k_new.shape[1]):
            kc, there = cached_rows(k_cache, table[b], L, g)
            vc, _ = cached_rows(v_cache, table[b], L, g)
            k, v = np.concatenate([kc, k_new[lo:hi, g]]), np.concatenate([vc, v_new[lo:hi, g]])
            sees = np.concatenate([np.broadcast_to(there, (n, L)), bits], 1)
            for h in range(g * G, g * G + G):
                yield slice(lo, hi), h, L + n, attend(q[lo:hi, h], k, v, scale, sees)

"""Oracle of the 4-bit KV cache: its format, attention, accumulated weights and
eviction, from their definitions in numpy and 64 bits (test-only)."""
import numpy as np

BS = 16
D = 128
SLAB = 2176
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """Codes (uint8 [..., 128]) and scale bytes (uint8 [..., 4]) of fp16 rows."""
    x = np.asarray(x)
    y = x.astype(np.float64).reshape(*x.shape[:-1], 4, 32)
    bad = ~np.isfinite(y).all(-1)
    m = np.abs(np.where(bad[..., None], 0.0, y)).max(-1)
    # least e with m <= 6 2^e, by counting: fp16 has 2^-24 <= m < 2^16
    e = np.full(m.shape, -27)
    for k in range(-27, 14):
        e = np.where(m > 6 * 2.0 ** k, k + 1, e)
    e = np.where(m == 0, 0, e)
    a = np.abs(np.where(bad[..., None], 0.0, y)) / 2.0 ** e[..., None]
    d = np.abs(a[..., None] - MAGNITUDES)
    # of two equally near codes the even one
    code = np.where(d == d.min(-1, keepdims=True), np.arange(8) % 2, 9).argmin(-1)
    code = np.where(np.signbit(y) & ~bad[..., None], code + 8, code)
    code = np.where(bad[..., None], 0, code)
    return code.astype(np.uint8).reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    """float64 values of codes [..., 128] and scale bytes [..., 4]."""
    v = np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)


def row_offsets(t):
    """Byte offsets in a slab of token t's K codes [64], V codes [64], K scales
    [4], V scales [4]."""
    i = np.arange(64)
    c, r = i // 4, i % 4
    return (t * 64 + i, 1024 + (t // 4) * 256 + c * 16 + (t % 4) * 4 + r, 2048 + t * 4 + np.arange(4),
            2112 + np.arange(4) * 16 + t)


OFFSETS = np.stack([np.concatenate(row_offsets(t)) for t in range(BS)])   # [16][136]


def append(cache, k_new, v_new, slots):
    """Stores fp16 rows [T][Hkv][128] in their slots (in place)."""
    slots = np.asarray(slots, dtype=np.int64)
    t = np.flatnonzero((slots >= 0) & (slots < cache.shape[0] * BS))
    (kc, ks), (vc, vs) = quantise(np.asarray(k_new)[t]), quantise(np.asarray(v_new)[t])
    kb, vb = (c[..., 0::2] | (c[..., 1::2] << 4) for c in (kc, vc))
    cache[(slots[t] // BS)[:, None, None], np.arange(cache.shape[1])[None, :, None],
          OFFSETS[slots[t] % BS][:, None, :]] = np.concatenate([kb, vb, ks, vs], -1)


def get_rows(cache, blocks, g, L):
    """float64 K and V rows [L][128] of kv-head g at a request's blocks."""
    t = np.arange(L)
    row = cache[np.asarray(blocks, dtype=np.int64)[t // BS][:, None], g, OFFSETS[t % BS]]
    kc, vc = (np.stack([x & 15, x >> 4], -1).reshape(L, D) for x in (row[:, :64], row[:, 64:128]))
    return values(kc, row[:, 128:132]), values(vc, row[:, 132:])


def live_tokens(table_row, L, num_blocks):
    """Table positions of the tokens that take part: within the row, in blocks
    of the pool."""
    L = min(int(L), len(table_row) * BS)
    t = np.arange(max(L, 0))
    ids = np.asarray(table_row, dtype=np.int64)[t // BS]
    return t[(ids >= 0) & (ids < num_blocks)]


def attention(q, cache, table, lens, scale):
    """out [B][Hq][128] and log-sum-exp [B][Hq] in 64 bits."""
    B, Hq, _ = q.shape
    nb, Hkv, _ = cache.shape
    G = Hq // Hkv
    out, lse = np.zeros((B, Hq, D)), np.full((B, Hq), -np.inf)
    with np.errstate(invalid="ignore"):
        for b in range(B):
            t = live_tokens(table[b], lens[b], nb)
            if len(t) == 0:
                continue
            ids = np.where((table[b] >= 0) & (table[b] < nb), table[b], 0)
            for g in range(Hkv):
                k, v = (x[t] for x in get_rows(cache, ids, g, int(t[-1]) + 1))
                s = q[b, g * G:(g + 1) * G].astype(np.float64) @ k.T * float(scale)
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                l = p.sum(-1, keepdims=True)
                out[b, g * G:(g + 1) * G] = (p / l) @ v
                lse[b, g * G:(g + 1) * G] = (m + np.log(l))[:, 0]
    return out, lse


def accumulate_weights(q, cache, table, lens, scale, lse, weights):
    """weights (float64 [nb][Hkv][16]) with the step's weights added."""
    B, Hq, _ = q.shape
    nb, Hkv, _ = cache.shape
    G = Hq // Hkv
    w = weights.astype(np.float64)
    for b in range(B):
        t = live_tokens(table[b], lens[b], nb)
        if len(t) == 0:
            continue
        ids = np.where((table[b] >= 0) & (table[b] < nb), table[b], 0)
        for g in range(Hkv):
            k, _ = get_rows(cache, ids, g, int(t[-1]) + 1)
            s = q[b, g * G:(g + 1) * G].astype(np.float64) @ k[t].T * float(scale)
            add = np.exp(s - lse[b, g * G:(g + 1) * G, None].astype(np.float64)).sum(0)
            w[table[b][t // BS], g, t % BS] += add
    return w


def kept_tokens(w, pos, keep, sinks, recent):
    """Mask of the tokens that one (request, kv-head) keeps: protected ones,
    all alike, then by weight; equal ones in slot order."""
    w, pos = np.asarray(w, dtype=np.float64), np.asarray(pos, dtype=np.int64)
    w = np.where(np.isnan(w), -np.inf, w)
    safe = (pos < sinks) | (pos > pos.max() - recent)
    kept = np.zeros(len(w), bool)
    kept[np.lexsort((np.arange(len(w)), np.where(safe, 0.0, -w), ~safe))[:keep]] = True
    return kept


def evict(cache, table, lens, weights, positions, keep, sinks, recent):
    """In place on cache, weights and positions.  Tokens and slots are those of
    the pool, in the order of the table row."""
    for b, L in enumerate(lens):
        t = live_tokens(table[b], L, cache.shape[0])
        if len(t) <= keep:
            continue
        block, at = table[b][t // BS], t % BS
        for g in range(cache.shape[1]):
            kept = kept_tokens(weights[block, g, at], positions[block, g, at], keep, sinks, recent)
            to, src = np.flatnonzero(~kept[:keep]), keep + np.flatnonzero(kept[keep:])
            cache[block[to][:, None], g, OFFSETS[at[to]]] = cache[block[src][:, None], g, OFFSETS[at[src]]]
            weights[block[to], g, at[to]] = weights[block[src], g, at[src]]
            positions[block[to], g, at[to]] = positions[block[src], g, at[src]]

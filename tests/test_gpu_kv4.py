"""The 4-bit KV cache on the GPU against its oracle (oracle/kv4.py, 64 bits).

Rows are quantised and moved exactly, so append, gather and evict are compared
bit for bit.  Tolerances of the attention and of the accumulated weights, from
their arithmetic:
  score    a digit expansion of q ends at 2^(E - 18) with 2^E the row's largest
           binade, so q_i is off by at most 2^(E - 19); the products are summed
           to fp32 precision, 2^-21 of the sum of their magnitudes with room
           for the four digits' sum and the scale;
  weight   2 x the score's error, relative (it enters the numerator and the
           sum), and 2^-15 for its two bf16 parts, cut off after 16 bits;
  out      that times max |V|, and half an fp16 step, 2^-11 of the value (or
           half the smallest subnormal, 2^-25);
  lse      the score's error, 2^-21 of itself, and the sum's roundings, one
           2^-24 for each of the tokens that a lane adds up.
"""
import numpy as np
import pytest

from oracle import kv4 as O

pytestmark = pytest.mark.gpu
BS, D, SLAB = 16, 128, 2176


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.fixture(scope="module")
def kv4():
    from paper_2506_03296_amd import kv4 as K
    K.load_library()
    return K


def dev(torch, *arrays):
    return [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def poisoned(nb, Hkv, seed):
    """A cache of random bytes whose scales are NaN: nothing unwritten may count."""
    c = np.random.default_rng(seed).integers(0, 256, (nb, Hkv, SLAB), dtype=np.uint8)
    c[..., 2048:] = 255
    return c


def case(lens, Hq, Hkv, seed, width=None, spare=3, offset=0.5):
    """q, cache, table, lens: rows of normal values at scattered blocks, the
    rest of the pool poisoned, table entries past a request's end out of range."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    nblk = [max(0, -(-int(L) // BS)) for L in lens]
    nb = sum(nblk) + spare
    width = width or max(1, max(nblk))
    ids = rng.permutation(nb).astype(np.int32)
    table = np.full((len(lens), width), -7, np.int32)
    cache = poisoned(nb, Hkv, seed + 1)
    i = 0
    shift = rng.standard_normal((Hkv, D)) * offset
    for b, n in enumerate(nblk):
        table[b, :n] = ids[i:i + n]
        i += n
    slots = [table[b, t // BS].astype(np.int64) * BS + t % BS for b, L in enumerate(lens) for t in range(int(L))]
    k = (rng.standard_normal((len(slots), Hkv, D)) + shift).astype(np.float16)
    v = rng.standard_normal((len(slots), Hkv, D)).astype(np.float16)
    O.append(cache, k, v, slots)
    q = rng.standard_normal((len(lens), Hq, D)).astype(np.float16)
    return q, cache, table, lens


def score_error(q, k, scale):
    """Bound on a score's error for one q row and K rows [L][128]."""
    top = np.abs(q.astype(np.float64)).max()
    E = np.floor(np.log2(top)) if top > 0 else -24.0
    return abs(scale) * (np.abs(k).sum(-1) * 2.0 ** (E - 19) + np.abs(k * q.astype(np.float64)).sum(-1) * 2.0 ** -21).max()


def check_attention(got, lse, q, cache, table, lens, scale):
    out, ref = O.attention(q, cache, table, lens, scale)
    B, Hq, _ = q.shape
    Hkv = cache.shape[1]
    worst = 0.0
    for b in range(B):
        t = O.live_tokens(table[b], lens[b], cache.shape[0])
        ids = np.where((table[b] >= 0) & (table[b] < cache.shape[0]), table[b], 0)
        for h in range(Hq):
            if len(t) == 0:
                assert not got[b, h].any() and (lse is None or lse[b, h] == -np.inf)
                continue
            if h % (Hq // Hkv) == 0:
                k, v = (x[t] for x in O.get_rows(cache, ids, h // (Hq // Hkv), int(t[-1]) + 1))
            err = score_error(q[b, h], k, scale)
            tol = (2 * err + 2.0 ** -15) * np.abs(v).max() + np.maximum(np.abs(out[b, h]) * 2.0 ** -11, 2.0 ** -25)
            diff = np.abs(got[b, h].astype(np.float64) - out[b, h])
            worst = max(worst, float((diff / tol).max()))
            assert np.all(diff <= tol), (b, h, float((diff / tol).max()))
            if lse is not None:
                lt = err + abs(ref[b, h]) * 2.0 ** -21 + (len(t) / 16 + 64) * 2.0 ** -24
                assert abs(float(lse[b, h]) - ref[b, h]) <= lt, (b, h, float(lse[b, h]), ref[b, h], lt)
    return worst


# --- append and gather ---------------------------------------------------------

@pytest.mark.parametrize("T,nb,Hkv,pad", [(1, 1, 1, 0), (3, 2, 2, 1), (16, 1, 8, 0), (17, 40, 3, 2), (33, 5, 32, 4),
                                          (300, 50, 8, 17), (1000, 70, 1, 0)])
def test_append_and_gather_bitwise(torch, kv4, T, nb, Hkv, pad):
    rng = np.random.default_rng(T)
    slots = rng.permutation(nb * BS)[:T].astype(np.int64)
    T = len(slots)
    if pad:
        slots[rng.permutation(T)[:pad]] = rng.choice([-1, -(1 << 40), nb * BS, 1 << 50], pad)
    k, v = (rng.standard_normal((2, T, Hkv, D)) * 10.0 ** rng.integers(-5, 4, (2, T, Hkv, 1))).astype(np.float16)
    cache = poisoned(nb, Hkv, T)
    pos, w = rng.integers(0, 99, (nb, Hkv, BS)).astype(np.int32), rng.random((nb, Hkv, BS)).astype(np.float32)
    tp = rng.integers(0, 1 << 30, T).astype(np.int32)
    dk, dv, dc, ds, dp, dw, dt = dev(torch, k, v, cache, slots, pos, w, tp)
    kv4.append(dk, dv, dc, ds, token_positions=dt, positions=dp, weights=dw)
    O.append(cache, k, v, slots)
    for t, s in enumerate(slots):
        if 0 <= s < nb * BS:
            pos[s // BS, :, s % BS], w[s // BS, :, s % BS] = tp[t], 0
    assert np.array_equal(dc.cpu().numpy(), cache)
    assert np.array_equal(dp.cpu().numpy(), pos) and np.array_equal(dw.cpu().numpy(), w)
    # back again: every slot of the pool, some twice, some outside
    back = np.concatenate([np.arange(nb * BS), slots]).astype(np.int64)
    gk, gv = (x.cpu().numpy() for x in kv4.gather(dc, torch.from_numpy(back).cuda()))
    for i, s in enumerate(back):
        for g in range(Hkv):
            if not 0 <= s < nb * BS:
                assert not gk[i, g].any() and not gv[i, g].any()
                continue
            for got, j in ((gk, 0), (gv, 1)):
                o = O.row_offsets(s % BS)
                byte = cache[s // BS, g, o[j]]
                want = O.values(np.stack([byte & 15, byte >> 4], -1).reshape(D), cache[s // BS, g, o[2 + j]])
                assert np.array_equal(got[i, g].astype(np.float64), want, equal_nan=True)


def test_append_every_fp16_value(torch, kv4):
    # each value beside a largest one that gives it scales of many sizes
    bits = np.arange(65536, dtype=np.uint16).view(np.float16)
    x = bits.reshape(512, 1, 128).copy()
    small = np.sort(bits[np.isfinite(bits)])[: 63488 // 128 * 128].reshape(-1, 1, 128)
    rng = np.random.default_rng(1)
    mixed = rng.permutation(bits[np.isfinite(bits)])[:63488].reshape(-1, 1, 128)
    rows = np.concatenate([x, small, mixed])
    T = len(rows)
    nb = -(-T // BS)
    cache = np.zeros((nb, 1, SLAB), np.uint8)
    dk, dv, dc = dev(torch, rows, rows[::-1], cache)
    kv4.append(dk, dv, dc, torch.arange(T, device="cuda"))
    O.append(cache, rows, rows[::-1], range(T))
    assert np.array_equal(dc.cpu().numpy(), cache)
    got = kv4.gather(dc, torch.arange(T, device="cuda"))[0].cpu().numpy()
    code, scale = O.quantise(rows)
    with np.errstate(over="ignore"):
        want = np.clip(O.values(code, scale), -65504, 65504).astype(np.float16)
    assert np.array_equal(got, want, equal_nan=True)


def test_append_from_a_fused_projection_and_on_another_stream(torch, kv4):
    rng = np.random.default_rng(2)
    T, Hkv = 48, 4
    fused = rng.standard_normal((T, 16 + 2 * Hkv, D)).astype(np.float16)
    slots = rng.permutation(12 * BS)[:T].astype(np.int64)
    cache = poisoned(12, Hkv, 3)
    df, dc, ds = dev(torch, fused, cache, slots)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    kv4.append(df[:, 16:16 + Hkv], df[:, 16 + Hkv:], dc, ds, stream=s)
    k, _ = kv4.gather(dc, ds, stream=s)
    s.synchronize()
    O.append(cache, fused[:, 16:16 + Hkv], fused[:, 16 + Hkv:], slots)
    assert np.array_equal(dc.cpu().numpy(), cache)


def test_rows_past_32_bits(torch, kv4):
    # a pool of 5.2 GB: its last blocks lie past 2^32 bytes
    nb, Hkv = 300000, 8
    cache = torch.zeros((nb, Hkv, SLAB), dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(4)
    lens = [100, 37]
    q, small, table, lens = case(lens, 32, Hkv, 5)
    high = nb - 1 - np.arange(small.shape[0], dtype=np.int64)
    cache[torch.from_numpy(high).cuda()] = torch.from_numpy(small).cuda()
    big = np.where(table >= 0, nb - 1 - table, table).astype(np.int32)
    dq, db, dl = dev(torch, q, big, lens)
    lse = torch.empty((2, 32), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, cache, db, dl, 0.1, lse_out=lse).cpu().numpy()
    check_attention(out, lse.cpu().numpy(), q, small, table, lens, 0.1)
    w = torch.zeros((nb, Hkv, BS), dtype=torch.float32, device="cuda")
    kv4.accumulate_weights(dq, cache, db, dl, 0.1, lse, w)
    assert abs(float(w.sum()) - 2 * 32) < 1e-3
    k = rng.standard_normal((5, Hkv, D)).astype(np.float16)
    slots = torch.arange(nb * BS - 5, nb * BS, device="cuda")
    dk, = dev(torch, k)
    kv4.append(dk, dk, cache, slots)
    code, scale = O.quantise(k)
    assert np.array_equal(kv4.gather(cache, slots)[1].cpu().numpy().astype(np.float64), O.values(code, scale))


# --- attention -------------------------------------------------------------------

LENS = [[1], [15, 16, 17], [0, 1, 0, 33, 0], [5, 64, 100, 257], [1000, 3, 130], [0, 0]]


@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (4, 2), (8, 2), (16, 2), (1, 1), (8, 1), (24, 3)])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_attention(torch, kv4, Hq, Hkv, lens):
    q, cache, table, lens = case(lens, Hq, Hkv, seed=Hq * 100 + Hkv)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.full((len(lens), Hq), 7.0, dtype=torch.float32, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    r = kv4.attention(dq, dc, dt, dl, 0.088, out=out, lse_out=lse)
    assert r is out
    worst = check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, 0.088)
    print(f"[kv4] {Hq}/{Hkv} {lens.tolist()}: {worst:.3f} of the tolerance", flush=True)
    # the same without the log-sum-exp, bit for bit
    assert torch.equal(out, kv4.attention(dq, dc, dt, dl, 0.088))


@pytest.mark.parametrize("lens", [[9000], [4100, 2, 3000, 77], [700] * 40, list(range(1, 300)), [20] * 700 + [1500]],
                         ids=["long", "ragged", "alike", "many", "bulk"])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (4, 1), (8, 1), (2, 1)])
def test_attention_over_many_work_groups(torch, kv4, Hq, Hkv, lens):
    q, cache, table, lens = case(lens, Hq, Hkv, seed=len(lens))
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((len(lens), Hq), dtype=torch.float32, device="cuda")
    for _ in range(3):      # the counters are left as they were found
        out = kv4.attention(dq, dc, dt, dl, 0.09, lse_out=lse)
    check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, 0.09)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0, 3e-5])
def test_attention_scales(torch, kv4, scale):
    q, cache, table, lens = case([40, 333, 1], 8, 2, seed=9)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((3, 8), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, scale, lse_out=lse)
    check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, scale)


@pytest.mark.parametrize("size", [2.0 ** -24, 1e-4, 300.0, 60000.0])
def test_attention_sizes_of_q_and_of_rows(torch, kv4, size):
    """q of one size (and of elements over many binades), rows near the ends of
    fp16: the largest stand for 65536, which fp16 does not hold."""
    rng = np.random.default_rng(3)
    q, cache, table, lens = case([50, 200], 8, 2, seed=11)
    q = (np.sign(q) * np.minimum(np.abs(q.astype(np.float64)) * size, 65504)).astype(np.float16)
    q[0] *= (2.0 ** -rng.integers(0, 20, q[0].shape)).astype(np.float16)
    rows = (rng.standard_normal((50, 2, D)) * 1e-6).astype(np.float16)
    rows[7], rows[8] = 65504, -65504
    slots = table[0, np.arange(50) // BS].astype(np.int64) * BS + np.arange(50) % BS
    O.append(cache, (rows * np.float16(0.01)).astype(np.float16), rows, slots)
    scale = 0.05 / max(size, 1e-3)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((2, 8), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, scale, lse_out=lse)
    check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, scale)


def test_attention_peaked_softmax(torch, kv4):
    """Scores hundreds apart, rising and falling along the context."""
    q, cache, table, lens = case([600, 600], 4, 1, seed=13, offset=0.0)
    t = np.arange(600)
    for b, ramp in ((0, t), (1, 600 - t)):
        k = (np.sign(q[b, 0].astype(np.float64)) * (ramp[:, None] / 100.0)).astype(np.float16)[:, None]
        v = np.random.default_rng(b).standard_normal((600, 1, D)).astype(np.float16)
        O.append(cache, k, v, table[b, t // BS].astype(np.int64) * BS + t % BS)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((2, 4), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, 1.0, lse_out=lse)
    check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, 1.0)


def test_attention_blocks_outside_the_pool_and_lengths_past_the_row(torch, kv4):
    q, cache, table, lens = case([100, 64, 40, 16], 8, 2, seed=15)
    table[0, 1], table[0, 6] = cache.shape[0], -1     # a hole in the middle, the last (partial) block gone
    table[3, 0] = 1 << 30                             # nothing left
    lens = np.array([100, 1 << 30, 2 ** 31 - 1, 16], np.int32)
    table[1:3, :] = np.where(table[1:3] < 0, -1, table[1:3])
    table = table[:, :7]
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    # rows 1 and 2: entries past their blocks are out of range, so all tokens of the blocks count
    keep = cache.copy()
    rng = np.random.default_rng(0)
    for b, (lo, hi) in ((1, (64, 64)), (2, (40, 48))):
        t = np.arange(lo, hi)
        x = rng.standard_normal((len(t), 2, D)).astype(np.float16)
        O.append(keep, x, x, table[b, t // BS].astype(np.int64) * BS + t % BS)
    dc = torch.from_numpy(keep).cuda()
    lse = torch.empty((4, 8), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, 0.1, lse_out=lse)
    check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, keep, table, lens, 0.1)
    assert not out[3].any()
    w = torch.zeros((keep.shape[0], 2, BS), dtype=torch.float32, device="cuda")
    kv4.accumulate_weights(dq, dc, dt, dl, 0.1, lse, w)
    ref = O.accumulate_weights(q, keep, table, lens, 0.1, lse.cpu().numpy(), np.zeros(w.shape))
    assert np.allclose(w.cpu().numpy(), ref, rtol=1e-4, atol=0) and abs(ref.sum() - 3 * 8) < 1e-3


def test_attention_non_finite(torch, kv4):
    q, cache, table, lens = case([40, 40, 40], 4, 2, seed=17)
    q[0, 1, 5], q[0, 2, 127] = np.nan, np.inf
    x = np.ones((1, 2, D), np.float16)
    x[0, 1, 3] = np.inf                                  # kv-head 1 of request 1
    O.append(cache, np.ones_like(x), x, [int(table[1, 1]) * BS + 2])
    O.append(cache, x, np.ones_like(x), [int(table[2, 0]) * BS + 9])
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((3, 4), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, 0.1, lse_out=lse).cpu().numpy()
    lse = lse.cpu().numpy()
    assert np.isfinite(out[0, [0, 3]]).all() and np.isnan(out[0, [1, 2]]).all() and np.isnan(lse[0, [1, 2]]).all()
    assert np.isfinite(out[1, :2]).all() and np.isnan(out[1, 2:, :32]).all() and np.isfinite(out[1, 2:, 32:]).all()
    assert np.isfinite(lse[1]).all()
    assert np.isfinite(out[2, :2]).all() and np.isnan(out[2, 2:]).all() and np.isnan(lse[2, 2:]).all()


def test_attention_longest_row(torch, kv4):
    """A million tokens, one block over and over: the result is the block's."""
    q, cache, table, lens = case([16], 4, 1, seed=19)
    reps = 1 << 16
    dq, dc = dev(torch, q, cache)
    dt = torch.full((1, reps), int(table[0, 0]), dtype=torch.int32, device="cuda")
    dl = torch.tensor([reps * BS - 5], dtype=torch.int32, device="cuda")
    lse = torch.empty((1, 4), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, 0.1, lse_out=lse).cpu().numpy().astype(np.float64)
    ref, rlse = O.attention(q, cache, table, lens, 0.1)
    k, v = O.get_rows(cache, table[0], 0, 16)
    for h in range(4):
        err = score_error(q[0, h], k, 0.1)
        # the five tokens that the last block lacks: 5 of a million, at most e^12 apart
        tol = (2 * err + 2.0 ** -15 + 5 / reps) * np.abs(v).max() + np.abs(ref[0, h]) * 2.0 ** -11
        assert np.all(np.abs(out[0, h] - ref[0, h]) <= tol)
        # 2^20 tokens over at most 4096 waves, a 64th of a wave's to a lane's chain
        assert abs(float(lse[0, h]) - rlse[0, h] - np.log(reps)) <= err + 1e-4


# --- accumulated weights -----------------------------------------------------------

@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (4, 2), (8, 2), (16, 2), (24, 3)])
@pytest.mark.parametrize("lens", LENS + [[3000, 1, 500]], ids=str)
def test_accumulate_weights(torch, kv4, Hq, Hkv, lens):
    q, cache, table, lens = case(lens, Hq, Hkv, seed=Hq * 10 + Hkv)
    rng = np.random.default_rng(1)
    w0 = rng.random((cache.shape[0], Hkv, BS)).astype(np.float32)
    _, lse = O.attention(q, cache, table, lens, 0.088)
    lse = lse.astype(np.float32)
    dq, dc, dt, dl, dlse, dw = dev(torch, q, cache, table, lens, lse, w0)
    kv4.accumulate_weights(dq, dc, dt, dl, 0.088, dlse, dw)
    got, ref = dw.cpu().numpy(), O.accumulate_weights(q, cache, table, lens, 0.088, lse, w0)
    err = 0.0
    for b in range(len(lens)):
        for h in range(Hq):
            if lens[b] > 0:
                k, _ = O.get_rows(cache, np.maximum(table[b], 0), h // (Hq // Hkv), int(lens[b]))
                err = max(err, score_error(q[b, h], k, 0.088) + 2.0 ** -21 * (1 + abs(lse[b, h])))
    tol = np.abs(ref - w0) * (2 * err + Hq / Hkv * 2.0 ** -23) + np.abs(ref) * 2.0 ** -24 * 2
    assert np.all(np.abs(got - ref) <= tol), float((np.abs(got - ref) / np.maximum(tol, 1e-30)).max())
    # slots of no live token are as they were
    dead = np.ones(w0.shape, bool)
    for b, L in enumerate(lens):
        t = np.arange(int(L))
        dead[table[b, t // BS], :, t % BS] = False
    assert np.array_equal(got[dead], w0[dead])


# --- eviction ------------------------------------------------------------------------

def evict_case(lens, Hkv, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    _, cache, table, lens = case(lens, Hkv, Hkv, seed)
    shape = (cache.shape[0], Hkv, BS)
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 3, shape).astype(np.float32) * np.where(rng.random(shape) < 0.5, -1, 1)   # (-0 among them)
    elif kind == "equal":
        w[:] = 0
    elif kind == "wild":
        w = np.where(rng.random(shape) < 0.3, -w, w)
        for x in (np.nan, np.inf, -np.inf, 3e38, 1e-42):
            w[rng.random(shape) < 0.05] = x
    pos = np.zeros(shape, np.int32)
    for b, L in enumerate(lens):
        t = np.arange(int(L))
        for g in range(Hkv):
            pos[table[b, t // BS], g, t % BS] = rng.permutation(int(L)) if b % 2 else t + 1000 * (b % 3)
    return cache, table, lens, w.astype(np.float32), pos


def run_evict(torch, kv4, cache, table, lens, w, pos, *budget):
    dc, dt, dl, dw, dp = dev(torch, cache, table, lens, w, pos)
    kv4.evict(dc, dt, dl, dw, dp, *budget)
    return [x.cpu().numpy() for x in (dc, dw, dp)]


def same(a, b):
    return all(np.array_equal(x.view(np.uint8), y.view(np.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "wild"])
@pytest.mark.parametrize("lens,keep,sinks,recent", [
    ([2], 1, 0, 0), ([2], 1, 1, 0), ([2], 1, 0, 1), ([17, 16, 15, 0, 1], 16, 4, 4), ([64, 65, 63, 128], 64, 0, 0),
    ([200, 300, 150], 128, 128, 0), ([200, 300, 150], 129, 9, 120), ([1500, 40, 1023, 1025], 1000, 4, 200),
    ([3000], 37, 4, 9), ([3001, 2500], 2499, 4, 1000), ([5000], 2500, 0, 0)], ids=str)
def test_evict(torch, kv4, kind, lens, keep, sinks, recent):
    cache, table, lens, w, pos = evict_case(lens, 3, seed=len(lens) + keep, kind=kind)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, sinks, recent)
    O.evict(cache, table, lens, w, pos, keep, sinks, recent)
    assert same(got, (cache, w, pos))


def test_evict_positions_of_any_size(torch, kv4):
    """Negative positions, the type's ends, the same one twice."""
    cache, table, lens, w, pos = evict_case([500, 400], 2, seed=3)
    pos[...] = np.random.default_rng(0).choice([-2 ** 31, -5, 0, 3, 77, 2 ** 31 - 3, 2 ** 31 - 1], pos.shape)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, 300, 50, 200)
    O.evict(cache, table, lens, w, pos, 300, 50, 200)
    assert same(got, (cache, w, pos))


@pytest.mark.parametrize("keep", [1, 255, 256, 257, 1500, 2047, 4999])
def test_evict_of_equal_keys(torch, kv4, keep):
    """All protected alike, all weights alike, and a few among many alike: the
    slots decide."""
    for kind in range(3):
        cache, table, lens, w, pos = evict_case([5000, 300], 1, seed=7)
        w[...] = 1.5
        if kind == 0:
            pos[...] = 0
        if kind == 2:
            w[np.random.default_rng(1).random(w.shape) < 0.02] = 2.0
            w[np.random.default_rng(2).random(w.shape) < 0.02] = -1.0
        budget = (keep, 1 if kind == 0 else 0, 0)
        got = run_evict(torch, kv4, cache, table, lens, w, pos, *budget)
        O.evict(cache, table, lens, w, pos, *budget)
        assert same(got, (cache, w, pos))


@pytest.mark.parametrize("kind", ["normal", "ties"])
@pytest.mark.parametrize("L,keep,sinks,recent", [(33000, 5000, 4, 1000), (70001, 69000, 0, 0), (40000, 33000, 0, 32768)])
def test_evict_of_long_pairs(torch, kv4, kind, L, keep, sinks, recent):
    cache, table, lens, w, pos = evict_case([L], 1, seed=L, kind=kind)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, sinks, recent)
    O.evict(cache, table, lens, w, pos, keep, sinks, recent)
    assert same(got, (cache, w, pos))


@pytest.mark.parametrize("keep,sinks,recent", [(1, 1, 0), (8192, 0, 0), (20000, 4, 9000), (33000, 0, 32000)])
@pytest.mark.parametrize("kind", ["normal", "ties"])
def test_evict_of_long_and_short_pairs_together(torch, kv4, kind, keep, sinks, recent):
    """Lengths on both sides of what a work group's registers hold, of its chunks
    and of the budget."""
    lens = [40961, 100, 32769, 32768, 0, 8193]
    cache, table, lens, w, pos = evict_case(lens, 2, seed=keep, kind=kind)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, sinks, recent)
    O.evict(cache, table, lens, w, pos, keep, sinks, recent)
    assert same(got, (cache, w, pos))


@pytest.mark.parametrize("keep", [1, 8191, 8192, 16500])
def test_evict_of_equal_keys_in_a_long_pair(torch, kv4, keep):
    """The slots decide, in any chunk."""
    for kind in range(3):
        cache, table, lens, w, pos = evict_case([40960], 1, seed=11)
        w[...] = 0.0
        if kind == 0:
            pos[...] = 0
        if kind == 2:
            w[np.random.default_rng(1).random(w.shape) < 0.02] = 2.0
            w[np.random.default_rng(2).random(w.shape) < 0.02] = -1.0
        budget = (keep, 1 if kind == 0 else 0, 0)
        got = run_evict(torch, kv4, cache, table, lens, w, pos, *budget)
        O.evict(cache, table, lens, w, pos, *budget)
        assert same(got, (cache, w, pos))


def test_evict_of_a_long_pair_among_many(torch, kv4):
    """Too many pairs to spread."""
    lens = np.random.default_rng(3).integers(0, 120, 70)
    lens[31] = 33333
    cache, table, lens, w, pos = evict_case(lens, 1, seed=9)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, 20000, 4, 3000)
    O.evict(cache, table, lens, w, pos, 20000, 4, 3000)
    assert same(got, (cache, w, pos))


def test_evict_of_many_pairs(torch, kv4):
    """More pairs than four for every CU, most of them short of the budget."""
    lens = np.random.default_rng(3).integers(0, 120, 300)
    lens[7] = 9000
    cache, table, lens, w, pos = evict_case(lens, 4, seed=9)
    got = run_evict(torch, kv4, cache, table, lens, w, pos, 50, 2, 10)
    O.evict(cache, table, lens, w, pos, 50, 2, 10)
    assert same(got, (cache, w, pos))


def test_evict_leaves_blocks_outside_the_pool_alone(torch, kv4):
    cache, table, lens, w, pos = evict_case([400, 100], 2, seed=5)
    table[0, 3], table[0, 20] = -1, cache.shape[0] + 5
    got = run_evict(torch, kv4, cache, table, lens, w, pos, 150, 4, 20)
    # the other request is as it was, and nothing outside the first one's blocks changed
    assert np.array_equal(got[0][table[1]], cache[table[1]])
    used = table[0, :25][(table[0, :25] >= 0) & (table[0, :25] < cache.shape[0])]
    others = np.setdiff1d(np.arange(cache.shape[0]), used)
    assert same([x[others] for x in got], [x[others] for x in (cache, w, pos)])


def test_evict_of_a_long_pair_leaves_blocks_outside_the_pool_alone(torch, kv4):
    """Tokens outside the pool weigh less than any in it; with as many in it as the
    budget keeps, those past the budget go to slots that are not there."""
    cache, table, lens, w, pos = evict_case([33600, 50], 1, seed=5)
    keep = 33600 - 3 * BS
    w[table[0, :3]] = -1.0
    out = [500, 1000, 2099]
    table[0, out] = -1, cache.shape[0], 2 ** 31 - 1
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, 0, 0)
    inside = np.setdiff1d(np.arange(2100), out)
    used = table[0, inside]
    others = np.setdiff1d(np.arange(cache.shape[0]), used)
    assert same([x[others] for x in got], [x[others] for x in (cache, w, pos)])
    # (the tokens of entries 2097 and 2098 go to entries 500 and 1000)
    assert same([x[used] for x in got], [x[used] for x in (cache, w, pos)])


# --- together ---------------------------------------------------------------------------

def test_a_run_of_decode_steps(torch, kv4):
    """Prompts, then steps of append, attention, accumulation and, when a
    request passes its budget, eviction, as an engine runs them, against the
    same steps of the oracle.  The accumulated weights decide what is evicted,
    so from the first eviction on both go by the GPU's."""
    rng = np.random.default_rng(21)
    B, Hq, Hkv, keep = 3, 8, 2, 40
    lens = np.array([37, 12, 41], np.int32)
    nb, width = 20, 4
    table = rng.permutation(nb)[:B * width].reshape(B, width).astype(np.int32)
    cache = poisoned(nb, Hkv, 1)
    w, pos = np.full((nb, Hkv, BS), 9.0, np.float32), np.full((nb, Hkv, BS), -1, np.int32)
    dc, dt, dw, dp = dev(torch, cache, table, w, pos)
    seq = lens.copy()       # tokens of each request so far

    def add(k, v, slots, tp):
        ds, dtp, dk, dv = dev(torch, slots, tp, k, v)
        kv4.append(dk, dv, dc, ds, token_positions=dtp, positions=dp, weights=dw)
        O.append(cache, k, v, slots)
        w[slots // BS, :, slots % BS] = 0
        pos[slots // BS, :, slots % BS] = tp[:, None]

    def rows(n):
        return (rng.standard_normal((n, Hkv, D)).astype(np.float16) for _ in range(2))

    t = np.concatenate([np.arange(L) for L in lens])
    b = np.repeat(np.arange(B), lens)
    add(*rows(len(t)), table[b, t // BS].astype(np.int64) * BS + t % BS, t.astype(np.int32))
    evicted = 0
    for step in range(12):
        lens += 1
        t = lens - 1
        add(*rows(B), table[np.arange(B), t // BS].astype(np.int64) * BS + t % BS, seq)
        seq += 1
        q = rng.standard_normal((B, Hq, D)).astype(np.float16)
        dq, dl = dev(torch, q, lens)
        lse = torch.empty((B, Hq), dtype=torch.float32, device="cuda")
        out = kv4.attention(dq, dc, dt, dl, 0.3, lse_out=lse)
        kv4.accumulate_weights(dq, dc, dt, dl, 0.3, lse, dw)
        check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, 0.3)
        ref = O.accumulate_weights(q, cache, table, lens, 0.3, lse.cpu().numpy(), w)
        got = dw.cpu().numpy()
        assert np.allclose(got, ref, rtol=1e-5, atol=1e-6)
        w[...] = got
        if (lens >= keep + 4).any():
            evicted += 1
            kv4.evict(dc, dt, dl, dw, dp, keep, 2, 10)
            O.evict(cache, table, lens, w, pos, keep, 2, 10)
            lens = np.minimum(lens, keep)
            assert same([x.cpu().numpy() for x in (dc, dw, dp)], (cache, w, pos))
    assert evicted >= 2
    # what is left of request 0, read back: its positions are distinct and hold the last ten
    t = np.arange(lens[0])
    for g in range(Hkv):
        p = pos[table[0, t // BS], g, t % BS]
        assert len(set(p.tolist())) == lens[0] and set(range(seq[0] - 10, seq[0])) <= set(p.tolist())


def test_captured_and_replayed(torch, kv4):
    """A step in a graph, replayed between eager calls; two graphs with a
    workspace each."""
    q, cache, table, lens = case([300, 700, 5], 8, 2, seed=23)
    dq, dt, dl = dev(torch, q, table, lens)
    k, v = (torch.randn((3, 2, D), device="cuda").half() for _ in range(2))
    slots = torch.from_numpy(table[np.arange(3), (lens - 1) // BS].astype(np.int64) * BS + (lens - 1) % BS).cuda()
    first = torch.from_numpy(cache).cuda()
    state = [first.clone(), torch.zeros((cache.shape[0], 2, BS), device="cuda"),
             torch.arange(cache.shape[0] * 2 * BS, dtype=torch.int32, device="cuda").view(-1, 2, BS)]
    keep = 64

    def step(c, w, p, out, lse, ws, we):
        kv4.append(k, v, c, slots, weights=w)
        kv4.attention(dq, c, dt, dl, 0.1, out=out, lse_out=lse, workspace=ws)
        kv4.accumulate_weights(dq, c, dt, dl, 0.1, lse, w)
        kv4.evict(c, dt, dl, w, p, keep, 1, 8, workspace=we)

    def buffers():
        return [x.clone() for x in state] + [
            torch.empty_like(dq), torch.empty((3, 8), device="cuda"),
            torch.zeros(kv4.attention_workspace_bytes(3, 8, 2), dtype=torch.uint8, device="cuda"),
            torch.empty(kv4.evict_workspace_bytes(3, 2, table.shape[1]), dtype=torch.uint8, device="cuda")]

    want = buffers()
    step(*want)
    graphs = []
    for _ in range(2):
        buf = buffers()
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=s):
            step(*buf)
        graphs.append((g, buf))
    for i in range(6):
        for g, buf in graphs:
            for x, y in zip(buf, state):
                x.copy_(y)
            g.replay()
        kv4.attention(dq, first, dt, dl, 0.1)
        if i % 2:
            torch.cuda.synchronize()
        for _, buf in graphs:
            for x, y in zip(buf[:5], want[:5]):
                assert torch.equal(x, y)


def test_an_eviction_of_long_pairs_captured_and_replayed(torch, kv4):
    """Steps in several launches, over what the workspace holds from before."""
    cache, table, lens, w, pos = evict_case([33001, 700], 2, seed=31, kind="ties")
    budget = (20000, 4, 5000)
    dt, dl = dev(torch, table, lens)
    first = dev(torch, cache, w, pos)
    O.evict(cache, table, lens, w, pos, *budget)
    ws = torch.full((kv4.evict_workspace_bytes(2, 2, table.shape[1]),), 255, dtype=torch.uint8, device="cuda")
    buf = [x.clone() for x in first]
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        kv4.evict(buf[0], dt, dl, buf[1], buf[2], *budget, workspace=ws)
    for i in range(4):
        for x, y in zip(buf, first):
            x.copy_(y)
        if i == 2:
            ws.fill_(255)
        g.replay()
        assert same([x.cpu().numpy() for x in buf], (cache, w, pos))
        own = [x.clone() for x in first]
        kv4.evict(own[0], dt, dl, own[1], own[2], *budget)
        assert all(torch.equal(x, y) for x, y in zip(own, buf))


def test_capture_without_a_workspace_is_refused(torch, kv4):
    q, cache, table, lens = case([30], 4, 1, seed=1)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    w, p = torch.zeros((cache.shape[0], 1, BS), device="cuda"), torch.zeros((cache.shape[0], 1, BS), dtype=torch.int32,
                                                                            device="cuda")
    out = torch.empty_like(dq)
    raised = []
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        for call in (lambda: kv4.attention(dq, dc, dt, dl, 0.1, out=out), lambda: kv4.evict(dc, dt, dl, w, p, 8)):
            try:
                call()
            except RuntimeError as e:
                raised.append(str(e))
        out.zero_()
    assert len(raised) == 2 and all("capture" in r for r in raised)


def test_two_streams_with_a_workspace_each(torch, kv4):
    q, cache, table, lens = case([3000, 2000, 100, 1], 8, 2, seed=25)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    want = kv4.attention(dq, dc, dt, dl, 0.1)
    torch.cuda.synchronize()
    runs = []
    for _ in range(2):
        runs.append((torch.cuda.Stream(), torch.zeros(kv4.attention_workspace_bytes(4, 8, 2), dtype=torch.uint8,
                                                      device="cuda"), torch.empty_like(dq)))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, ws, out in runs:
            kv4.attention(dq, dc, dt, dl, 0.1, out=out, workspace=ws, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for _, _, out in runs)


def test_one_workspace_for_calls_of_many_shapes(torch, kv4):
    """Partials of one call lie where no other call looks for its counters."""
    ws = torch.zeros(kv4.attention_workspace_bytes(700, 8, 8), dtype=torch.uint8, device="cuda")
    for lens, Hq, Hkv in (([3000], 8, 1), ([40] * 700, 8, 8), ([2000, 5, 900], 4, 4), ([1500] * 40, 8, 4), ([9000], 2, 1),
                          ([3000], 8, 1)):
        q, cache, table, lens = case(lens, Hq, Hkv, seed=len(lens) + Hq)
        dq, dc, dt, dl = dev(torch, q, cache, table, lens)
        own = torch.zeros(kv4.attention_workspace_bytes(len(lens), Hq, Hkv), dtype=torch.uint8, device="cuda")
        for _ in range(2):
            assert torch.equal(kv4.attention(dq, dc, dt, dl, 0.1, workspace=ws), kv4.attention(dq, dc, dt, dl, 0.1, workspace=own))


def test_empty_tables_and_pools(torch, kv4):
    q = torch.randn((2, 4, D), device="cuda").half()
    lens = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    wide, none = (torch.zeros((2, n), dtype=torch.int32, device="cuda") for n in (3, 0))
    lse = torch.zeros((2, 4), device="cuda")
    for nb, table in ((3, none), (0, wide), (0, none)):
        c = torch.full((nb, 2, SLAB), 255, dtype=torch.uint8, device="cuda")
        out = kv4.attention(q, c, table, lens, 0.1, lse_out=lse)
        assert not out.any() and torch.isinf(lse).all()
        w, p = torch.ones((nb, 2, BS), device="cuda"), torch.zeros((nb, 2, BS), dtype=torch.int32, device="cuda")
        kv4.accumulate_weights(q, c, table, lens, 0.1, lse, w)
        kv4.evict(c, table, lens, w, p, 2)
        assert (w == 1).all() and (c == 255).all()
    k, v = kv4.gather(c, torch.tensor([0, -1, 70], device="cuda"))
    assert not k.any() and not v.any()
    kv4.append(torch.ones((2, 2, D), device="cuda").half(), torch.ones((2, 2, D), device="cuda").half(), c,
               torch.tensor([0, 1], device="cuda"))


def test_growing_and_releasing_the_librarys_workspace(torch, kv4):
    for lens in ([100], [50] * 600, [3000, 1]):
        q, cache, table, lens = case(lens, 4, 1, seed=27)
        dq, dc, dt, dl = dev(torch, q, cache, table, lens)
        ws = torch.zeros(kv4.attention_workspace_bytes(len(lens), 4, 1), dtype=torch.uint8, device="cuda")
        assert torch.equal(kv4.attention(dq, dc, dt, dl, 0.1), kv4.attention(dq, dc, dt, dl, 0.1, workspace=ws))
    kv4.release_workspace()
    assert torch.equal(kv4.attention(dq, dc, dt, dl, 0.1), kv4.attention(dq, dc, dt, dl, 0.1, workspace=ws))


# --- the binding ---------------------------------------------------------------------------

BREAK = {
    "dtype": lambda t: t.double() if t.is_floating_point() else t.long() if str(t.dtype) != "torch.int64" else t.int(),
    "host": lambda t: t.cpu(),
    "shape": lambda t: t[..., :-1].contiguous() if t.dim() > 1 else t[:-1],
    "gaps": lambda t: t.repeat_interleave(2, dim=-1)[..., ::2],
}


@pytest.mark.parametrize("how", list(BREAK))
def test_binding_refuses(torch, kv4, how):
    q, cache, table, lens = case([40, 17], 4, 2, seed=29)
    good = dict(zip("q cache table lens".split(), dev(torch, q, cache, table, lens)))
    nb = cache.shape[0]
    good.update(k=torch.zeros((5, 2, D), dtype=torch.float16, device="cuda"), slots=torch.arange(5, device="cuda"),
                w=torch.zeros((nb, 2, BS), device="cuda"), p=torch.zeros((nb, 2, BS), dtype=torch.int32, device="cuda"),
                tp=torch.zeros(5, dtype=torch.int32, device="cuda"), lse=torch.zeros((2, 4), device="cuda"),
                out=torch.zeros((2, 4, D), dtype=torch.float16, device="cuda"),
                rows=torch.zeros((5, 2, D), dtype=torch.float16, device="cuda"),
                rows2=torch.zeros((5, 2, D), dtype=torch.float16, device="cuda"),
                ws=torch.zeros(kv4.attention_workspace_bytes(2, 4, 2), dtype=torch.uint8, device="cuda"),
                we=torch.zeros(1 << 16, dtype=torch.uint8, device="cuda"))
    good["v"] = good["k"].clone()
    calls = {
        "append": (lambda a: kv4.append(a["k"], a["v"], a["cache"], a["slots"], a["tp"], a["p"], a["w"]),
                   "k v cache slots tp p w"),
        "gather": (lambda a: kv4.gather(a["cache"], a["slots"], a["rows"], a["rows2"]), "cache slots rows rows2"),
        "attention": (lambda a: kv4.attention(a["q"], a["cache"], a["table"], a["lens"], 0.1, a["out"], a["lse"], a["ws"]),
                      "q cache table lens out lse ws"),
        "weights": (lambda a: kv4.accumulate_weights(a["q"], a["cache"], a["table"], a["lens"], 0.1, a["lse"], a["w"]),
                    "q cache table lens lse w"),
        "evict": (lambda a: kv4.evict(a["cache"], a["table"], a["lens"], a["w"], a["p"], 8, 1, 2, a["we"]),
                  "cache table lens w p we"),
    }
    for name, (call, args) in calls.items():
        call(good)
        for x in args.split():
            # any row width is a table, and one byte less is workspace enough
            if how == "shape" and x in ("table", "we"):
                continue
            with pytest.raises((TypeError, ValueError, RuntimeError)):
                call({**good, x: BREAK[how](good[x])})
    torch.cuda.synchronize()


def test_binding_pairs_of_arguments(torch, kv4):
    c = kv4.empty_cache(3, 2, "cuda")
    k = torch.zeros((5, 2, D), dtype=torch.float16, device="cuda")
    s = torch.arange(5, device="cuda")
    with pytest.raises(ValueError):
        kv4.append(k, k, c, s, positions=torch.zeros((3, 2, BS), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        kv4.append(k, k[:, :1], c, s)
    with pytest.raises(ValueError):
        kv4.append(k, torch.zeros((5, 4, D), dtype=torch.float16, device="cuda")[:, :2], c, s)
    with pytest.raises(ValueError):
        kv4.append(k[:1].expand(5, 2, D), k[:1].expand(5, 2, D), c, s)     # no stride between tokens
    b = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    n = torch.full((1,), 40, dtype=torch.int32, device="cuda")
    w, p = torch.zeros((3, 2, BS), device="cuda"), torch.zeros((3, 2, BS), dtype=torch.int32, device="cuda")
    for budget in ((0,), (-1,), (1 << 32,), (8, -1), (8, 0, -1), (8, 5, 4)):
        with pytest.raises(ValueError):
            kv4.evict(c, b, n, w, p, *budget)
    kv4.append(k[:0], k[:0], c, s[:0])
    assert kv4.gather(c, s[:0])[0].shape == (0, 2, D)
    e = torch.empty((0, 4, D), dtype=torch.float16, device="cuda")
    i = torch.empty((0, 3), dtype=torch.int32, device="cuda")
    assert kv4.attention(e, c, i, i[:, 0], 0.1).shape == (0, 4, D)

"""Evictions from the 4-bit KV cache where table rows hold ids outside the pool.

Only tokens and slots of the pool count: a request with more than `keep` of them
keeps `keep`, in the first `keep` of its row's slots of the pool, so none that the
order of keeping names is lost, whichever of its blocks are elsewhere.  Rows move
as they are, so all of it is compared bit for bit.
"""
import numpy as np
import pytest

from oracle import kv4 as O
from test_gpu_kv4 import BS, case, evict_case, kv4, run_evict, same, torch  # noqa: F401  (two are fixtures)

OUTSIDE = (-1, 2 ** 31 - 1, -2 ** 31, None)   # (None: the pool's size)


def lose(cache, table, lens, entries, seed=0):
    """Puts ids outside the pool at `entries` (a list for every request)."""
    rng = np.random.default_rng(seed)
    for b, of in enumerate(entries):
        for e in of:
            x = OUTSIDE[rng.integers(len(OUTSIDE))]
            table[b, e] = cache.shape[0] if x is None else x


def check_definition(before, after, table, lens, keep, sinks, recent):
    """The outcome, token by token, against the definition: the tokens kept are
    those that come first by (protected, weight, slot), all of them lie in the first
    `keep` slots of the pool, and all other slots are as they were."""
    (c0, w0, p0), (c1, w1, p1) = before, after
    touched = np.zeros(w0.shape, bool)
    for b, L in enumerate(lens):
        t = O.live_tokens(table[b], L, c0.shape[0])
        if len(t) <= keep:
            continue
        block, at = table[b][t // BS], t % BS
        for g in range(c0.shape[1]):
            rows = [x[block[:, None], g, O.OFFSETS[at]] for x in (c0, c1)]
            w, pos = (np.stack([x[block, g, at] for x in y]) for y in ((w0, w1), (p0, p1)))
            safe = (pos[0] < sinks) | (pos[0] > int(pos[0].max()) - recent)
            order = sorted(range(len(t)), key=lambda i: (not safe[i], 0.0 if safe[i] else -float(w[0, i]), i))
            token = [(rows[j][i].tobytes(), w[j, i].tobytes(), int(pos[j, i])) for j in (0, 1) for i in range(len(t))]
            assert sorted(token[i] for i in order[:keep]) == sorted(token[len(t):len(t) + keep])
            assert token[keep:len(t)] == token[len(t) + keep:]
        touched[block[:keep], :, at[:keep]] = True
    assert np.array_equal(w1[~touched], w0[~touched]) and np.array_equal(p1[~touched], p0[~touched])


# entries of the first request outside the pool; of 48 tokens 32 are left, of 50 34, ...
SMALL = [([48], 31, 2, 8, [[0]]), ([48], 32, 0, 32, [[0]]), ([48], 24, 2, 8, [[0]]), ([48], 1, 0, 1, [[1]]),
         ([50], 33, 0, 20, [[1]]), ([50], 16, 0, 3, [[3]]), ([50], 20, 0, 0, [[0, 1, 2]]), ([50], 2, 0, 0, [[0, 1, 2]]),
         ([50], 1, 0, 0, [[0, 1, 2]]), ([50], 20, 0, 0, [[0, 1, 2, 3]]), ([64], 16, 0, 16, [[1, 2]]),
         ([64, 64], 16, 0, 16, [[0, 3], []]), ([400, 100], 150, 4, 20, [[3, 20], []]), ([400, 300], 200, 4, 100, [[0, 1, 2, 12], [18]])]


@pytest.mark.parametrize("lens,keep,sinks,recent,entries", SMALL, ids=str)
def test_oracle_keeps_what_the_order_names(lens, keep, sinks, recent, entries):
    cache, table, lens, w, pos = evict_case(lens, 2, seed=keep)
    lose(cache, table, lens, entries)
    before = [x.copy() for x in (cache, w, pos)]
    O.evict(cache, table, lens, w, pos, keep, sinks, recent)
    check_definition(before, (cache, w, pos), table, lens, keep, sinks, recent)


def on_gpu(torch, kv4, state, *budget):  # noqa: F811
    cache, table, lens, w, pos = state
    got = run_evict(torch, kv4, cache, table, lens, w, pos, *budget)
    O.evict(cache, table, lens, w, pos, *budget)
    assert same(got, (cache, w, pos))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["normal", "ties"])
@pytest.mark.parametrize("lens,keep,sinks,recent,entries", SMALL, ids=str)
def test_evict(torch, kv4, kind, lens, keep, sinks, recent, entries):  # noqa: F811
    state = evict_case(lens, 2, seed=keep, kind=kind)
    lose(*state[:3], entries)
    on_gpu(torch, kv4, state, keep, sinks, recent)


# lengths for every number of tokens that a thread holds, for work groups of either
# size, for those that read their tokens again, and for pairs spread over work groups
@pytest.mark.gpu
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
@pytest.mark.parametrize("lens,Hkv,keep", [
    ([500, 33], 2, 200), ([2000, 400, 0], 2, 700), ([4000, 2049], 1, 1500), ([8000, 7000], 1, 6000),
    ([2000, 8200], 1, 900), ([16000, 9000], 1, 4096), ([32768, 17000], 1, 15000), ([9000] + [5] * 1030, 1, 3000),
    ([33000, 700], 1, 20000), ([40960, 33333, 8192], 1, 8192), ([33333] + [40] * 70, 1, 20000)],
                         ids=lambda x: str(x)[:24])
def test_evict_of_lengths(torch, kv4, lens, Hkv, keep, share):  # noqa: F811
    cache, table, lens, w, pos = evict_case(lens, Hkv, seed=keep, kind="ties" if share == 0.5 else "normal")
    rng = np.random.default_rng(keep)
    lose(cache, table, lens, [np.flatnonzero(rng.random(-(-L // BS)) < share) for L in lens])
    n = len(O.live_tokens(table[0], lens[0], cache.shape[0]))
    # a budget of its own, and those that the tokens of the pool just exceed, equal
    # and do not reach
    for k in (keep, n - 1, n, n + 1):
        if k > 0:
            on_gpu(torch, kv4, (cache.copy(), table, lens, w.copy(), pos.copy()), k, 4 if k > 20 else 0, k // 3)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,keep", [([700], 300), ([33000], 18000)], ids=str)
def test_attention_afterwards(torch, kv4, lens, keep):  # noqa: F811
    """The length that a request has after the call: up to the keep-th slot of the
    pool.  Its attention is that over the kept tokens."""
    cache, table, lens, w, pos = evict_case(lens, 1, seed=5)
    lose(cache, table, lens, [[0, 7, keep // BS]])
    t = O.live_tokens(table[0], lens[0], cache.shape[0])
    kept = O.kept_tokens(w[table[0][t // BS], 0, t % BS], pos[table[0][t // BS], 0, t % BS], keep, 4, 50)
    ids = np.where((table[0] >= 0) & (table[0] < cache.shape[0]), table[0], 0)
    k, v = (x[t][kept] for x in O.get_rows(cache, ids, 0, int(lens[0])))
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, 4, 50)
    q = np.random.default_rng(1).standard_normal((1, 2, 128)).astype(np.float16)
    length = np.array([t[keep - 1] + 1], np.int32)
    dq, dc, dt, dl = (torch.from_numpy(x).cuda() for x in (q, got[0], table, length))
    out = kv4.attention(dq, dc, dt, dl, 0.09).cpu().numpy().astype(np.float64)
    s = q[0].astype(np.float64) @ k.T * float(np.float32(0.09))
    p = np.exp(s - s.max(-1, keepdims=True))
    want = p / p.sum(-1, keepdims=True) @ v
    # scores 2^-19 of q's largest binade (below 8) times sum |K| times the scale, twice;
    # weights 2^-15; half an fp16 step
    tol = (2 * 0.09 * np.abs(k).sum(-1).max() * 8 * 2.0 ** -18 + 2.0 ** -15) * np.abs(v).max() + np.abs(want) * 2.0 ** -11
    assert np.all(np.abs(out[0] - want) <= tol)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,keep", [([3000, 60], 1000), ([33001, 700], 20000)], ids=str)
def test_captured_and_replayed(torch, kv4, lens, keep):  # noqa: F811
    """Rows with and without ids outside the pool by turns, in one graph."""
    states = []
    for share in (0.0, 0.3, 0.0, 0.9):
        cache, table, lens_, w, pos = evict_case(lens, 2, seed=len(states))
        rng = np.random.default_rng(len(states))
        lose(cache, table, lens_, [np.flatnonzero(rng.random(-(-L // BS)) < share) for L in lens])
        first = [torch.from_numpy(x).cuda() for x in (cache, table, w, pos)]
        O.evict(cache, table, lens_, w, pos, keep, 4, keep // 4)
        states.append((first, (cache, w, pos)))
    buf = [x.clone() for x in states[0][0]]
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.full((kv4.evict_workspace_bytes(len(lens), 2, buf[1].shape[1]),), 255, dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        kv4.evict(buf[0], buf[1], dl, buf[2], buf[3], keep, 4, keep // 4, workspace=ws)
    for first, want in states + states:
        for x, y in zip(buf, first):
            x.copy_(y)
        g.replay()
        assert same([buf[i].cpu().numpy() for i in (0, 2, 3)], want)

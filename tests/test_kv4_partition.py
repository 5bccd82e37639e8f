"""How the attention over the 4-bit KV cache cuts a batch: which batches of these
tests reach which way (CPU, with the constants read from the source), and their
results against the oracle (GPU).

The plan here follows the rules beside plan_of in kv4_attention.hip for a device of
256 compute units, in whole numbers and by explicit positions.
"""
import functools
import os
import re

import numpy as np
import pytest

from oracle import kv4 as O
from test_gpu_kv4 import BS, D, check_attention, dev, kv4, poisoned, score_error, torch  # noqa: F401  (two are fixtures)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
W = 256          # work groups: compute units of an MI355X
WAVES = 8


@functools.lru_cache(maxsize=None)
def constants():
    text = open(os.path.join(ROOT, "paper_2506_03296_amd", "csrc", "kv4", "kv4_attention.hip")).read()
    found = {}
    for line in re.findall(r"^constexpr (?:unsigned|int) (\w[^;]*);", text, re.M):
        for name, value in re.findall(r"(k\w+) = (\d+)", line):
            found[name] = int(value)
    return found


def start(V, w):
    per, rest = divmod(V, W)
    return w * per + w * rest // W


def plan(lens, Hkv):
    """way, and for every request its pairs' contributors (for the line: the most
    over its kv-heads)."""
    c = constants()
    K, least_part, most_part = c["kPairCost"], c["kMinPart"], c["kMaxPart"]
    nb = [max(0, -(-int(L) // BS)) for L in lens]
    pairs, U, longest = sum(n > 0 for n in nb) * Hkv, sum(nb) * Hkv, max(nb)
    if U == 0:
        return "line", [0] * len(nb)
    if pairs > W and longest <= c["kMostWhole"]:
        per, rounds = U // W, -(-pairs // (WAVES * W))
        if longest <= c["kWholeBlocks"] or max(3 * longest * rounds, per + per // 8) + 32 < per + K * pairs // W:
            return "whole", [int(n > 0) for n in nb]
    if pairs <= W:
        room = W - pairs
        least = longest if longest <= 2 * least_part else -(-U // room) if room > 0 else U
        if least <= most_part:
            parts = []
            for n in nb:
                t = max(least_part, least_part // 2 + n // 64, least)
                count = -(-n // t)
                parts.append(-(-n // -(-n // count)) if n else 0)
                assert parts[-1] <= count
            return "parts", parts
    V = U + K * pairs
    owner = np.repeat(np.arange(W), np.diff([start(V, w) for w in range(W + 1)]))
    contributors, at = [], 0
    for n in nb:
        most = 0
        for _ in range(Hkv if n else 0):
            most = max(most, int(owner[at + K + n - 1] - owner[at + K]) + 1)
            at += K + n
        contributors.append(most)
    assert at == V
    return "line", contributors


# lens, Hkv, way, the most contributors of a pair
BATCHES = {
    "line, one long among many": ([20000] + [400] * 300, 1, "line", 13),
    "line, three to a pair": ([2500] + [1] * 300, 1, "line", 3),
    "line, up to 64 requests": ([9000] + [700] * 30 + [5000, 40], 8, "line", 5),
    "line, as many pairs as work groups": (list(range(300, 8300, 250)), 8, "line", 3),
    "line, empty requests among 64": ([0, 0, 6000] + [300, 0, 2600] * 18 + [0], 8, "line", 3),
    "line, empty requests among many": ([0, 0, 0] + [1000, 0] * 150 + [0, 5, 0, 0], 2, "line", 2),
    "whole, empty requests among many": ([0, 20] * 300, 1, "whole", 1),
    "whole, empty requests among 64": ([0, 400, 17] * 20, 8, "whole", 1),
    "whole, more pairs than waves": ([0, 90, 16, 1] * 150 + [0], 8, "whole", 1),
    "parts, empty requests among many": ([0, 3000] + [0, 30] * 60 + [0], 2, "parts", 6),
    "parts, empty requests among 64": ([0, 0, 5000, 0, 17, 0], 4, "parts", 10),
    "a part a pair": ([700, 0, 1024, 1] * 20, 4, "parts", 1),
}


@pytest.mark.parametrize("name", list(BATCHES))
def test_the_batches_reach_their_ways(name):
    lens, Hkv, way, most = BATCHES[name]
    got, contributors = plan(lens, Hkv)
    assert (got, max(contributors)) == (way, most)


def test_parts_fit_the_work_groups():
    rng = np.random.default_rng(0)
    seen = set()
    for _ in range(3000):
        B, Hkv = int(rng.integers(1, 120)), int(rng.choice([1, 2, 4, 8, 32]))
        lens = np.exp(rng.uniform(0, rng.uniform(1, 11.8), B)).astype(int) * (rng.random(B) < 0.9)
        way, contributors = plan(lens, Hkv)
        seen.add(way)
        if way == "parts":
            assert sum(contributors) * Hkv <= W
    assert seen == {"line", "parts", "whole"}


@functools.lru_cache(maxsize=1)
def batch(name):
    """cache, table, lens: any codes with scales of 2^-3 to 2^-1 in the slots of the
    requests, NaN scales in all others, table entries past a request's end out of
    range."""
    lens, Hkv, _, _ = BATCHES[name]
    lens = np.asarray(lens, np.int32)
    rng = np.random.default_rng(len(lens))
    nblk = -(-lens // BS)
    nb, width = int(nblk.sum()) + 3, int(nblk.max())
    table = np.full((len(lens), width), -7, np.int32)
    ids = rng.permutation(nb)
    cache = poisoned(nb, Hkv, 1)
    for b, L in enumerate(lens):
        first = int(nblk[:b].sum())
        table[b, :nblk[b]] = ids[first:first + nblk[b]]
        t = np.arange(L)
        offsets = O.OFFSETS[t % BS][:, 128:]   # of the scales
        cache[table[b, t // BS][:, None, None], np.arange(Hkv)[None, :, None], offsets[:, None, :]] = rng.integers(
            124, 127, (L, Hkv, 8), dtype=np.uint8)
    return cache, table, lens


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("name", list(BATCHES))
def test_attention(torch, kv4, name, G):  # noqa: F811
    assert torch.cuda.get_device_properties(0).multi_processor_count == W
    cache, table, lens = batch(name)
    q = np.random.default_rng(G).standard_normal((len(lens), cache.shape[1] * G, D)).astype(np.float16)
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    kv4.attention(dq, dc, dt, dl, 0.09, out=out, lse_out=lse)
    worst = check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, 0.09)
    print(f"[kv4] {name}, G = {G}: {worst:.3f} of the tolerance", flush=True)
    again = kv4.attention(dq, dc, dt, dl, 0.09)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("scale", [0.09, 0.0, -0.07])
@pytest.mark.parametrize("name", ["line, empty requests among many", "whole, empty requests among many",
                                  "parts, empty requests among 64"])
def test_accumulated_weights(torch, kv4, name, scale, G):  # noqa: F811
    """Batches of more and of fewer than 64 requests, any sign of the scale."""
    cache, table, lens = batch(name)
    B, Hkv = len(lens), cache.shape[1]
    rng = np.random.default_rng(G)
    q = rng.standard_normal((B, Hkv * G, D)).astype(np.float16)
    w0 = rng.random((cache.shape[0], Hkv, BS)).astype(np.float32)
    lse = O.attention(q, cache, table, lens, scale)[1].astype(np.float32)
    dq, dc, dt, dl, dlse, dw = dev(torch, q, cache, table, lens, lse, w0)
    kv4.accumulate_weights(dq, dc, dt, dl, scale, dlse, dw)
    got, ref = dw.cpu().numpy(), O.accumulate_weights(q, cache, table, lens, scale, lse, w0)
    # a weight: e to the score's error and to 2^-21 of the lse's size, then sums of G
    # and of the old value
    err = 0.0
    for b in np.flatnonzero(lens > 0):
        for h in range(0, Hkv * G, G):
            k, _ = O.get_rows(cache, np.maximum(table[b], 0), h // G, int(lens[b]))
            for i in range(h, h + G):
                err = max(err, score_error(q[b, i], k, scale) + 2.0 ** -21 * (1 + abs(float(lse[b, i]))))
    tol = np.abs(ref - w0) * (2 * err + G * 2.0 ** -23) + np.abs(ref) * 2.0 ** -23
    assert np.all(np.abs(got - ref) <= tol), float((np.abs(got - ref) / np.maximum(tol, 1e-30)).max())
    dead = np.ones(w0.shape, bool)
    for b, L in enumerate(lens):
        t = np.arange(int(L))
        dead[table[b, t // BS], :, t % BS] = False
    assert np.array_equal(got[dead], w0[dead])

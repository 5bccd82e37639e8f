"""The softmax's weights in prompt attention and tree attention: keys far below a
row's largest, against the oracle in 64 bits.

Tolerance, as in test_gpu_steps.py but for the term of the smallest weights.  Weights
are held 2^11 times what the softmax defines, or more, so that what lies among
fp16's subnormal numbers is off by half of 2^-24, 2^-36 of the row's largest weight.
With sum |V| over the keys that a row attends, and the sum of its weights in units of
the largest one, e^(lse - the largest score): 2^-36 sum |V| / that sum.
"""
import numpy as np
import pytest

from oracle import steps as O
from test_gpu_steps import D, oracle, prompts, run_prompts, run_trees, steps, torch, trees  # noqa: F401

pytestmark = pytest.mark.gpu
FLOOR = 2.0 ** -36
GAPS = [12, 14, 15.5, 16.5, 17, 17.016, 18, 19.5, 21, 22, 24]


def tolerance(n, scale, most, mag, out, sum_v, total_w, weight):
    err = abs(scale) * most * (2.0 ** -17 + 2.0 ** -22)
    total = n * 2.0 ** -24 + 2.0 ** -20
    rel = 2 * err + 2 * 2.0 ** -22 + weight + 2 * total
    return np.asarray(rel)[:, None] * mag + FLOOR * sum_v / total_w[:, None] + np.maximum(np.abs(out) * 2.0 ** -11, 2.0 ** -25)


def one_key_above(q, k, v, gap, size):
    """Scores of 0 but for one key, whose score is the gap and whose values are 0."""
    q[:], k[:], v[:] = 0, 0, size
    q[:, :, 0] = 1
    k[0, :, 0], v[0] = gap, 0


@pytest.mark.parametrize("size", [1, 200])
@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("n,Hq", [(3000, 1), (200, 4)])
def test_prompt_weights_far_below_the_largest(torch, steps, n, Hq, gap, size):  # noqa: F811
    q, k, v, offsets = prompts([n], Hq, 1, 61)
    one_key_above(q, k, v, gap, size)
    got, _ = run_prompts(torch, steps, q, k, v, offsets, 1.0)
    for _, h, _, (out, lse, mag, most) in O.prompt(q[:, :1], k, v, offsets, 1.0):
        tol = tolerance(n, 1.0, most, mag, out, size * np.arange(n)[:, None], np.exp(lse - most), 2.0 ** -11)
        for head in range(Hq):
            diff = np.abs(got[:, head].astype(np.float64) - out)
            assert np.all(diff <= tol), float((diff / tol).max())


@pytest.mark.parametrize("size", [1, 200])
@pytest.mark.parametrize("gap", GAPS)
@pytest.mark.parametrize("nodes", [3, 16, 32, 64])
def test_tree_weights_far_below_the_largest(torch, steps, nodes, gap, size):  # noqa: F811
    L = 2000
    c = trees([L], [nodes], 4, 1, 62, masks=[0] * nodes)
    c["q"][:], c["kc"][:], c["vc"][:] = 0, 0, size
    c["q"][:, :, 0] = 1
    c["kc"][:, 0, 0, 0], c["vc"][:, 0, 0] = gap, 0      # a block's first token: every wave has such a key
    got, _ = run_trees(torch, steps, c, 1.0)
    for at, h, _, (out, lse, mag, most) in oracle(c, 1.0):
        tol = tolerance(L, 1.0, most, mag, out, size * L, np.exp(lse - most), 2.0 ** -11)
        diff = np.abs(got[at, h].astype(np.float64) - out)
        assert np.all(diff <= tol), (h, float((diff / tol).max()))


# Trees take the weights in two parts.  Rows here attend few keys, whose scores are
# exact (one product a row), so that little but the weights and the output's rounding is
# left: the score times c = log2 e and the exponential's argument, 2^-24 of up to 8 log2 e
# each and c's own rounding as much, 3 x 12 x 2^-24 x ln 2 of a weight; the exponential
# and the factors that join parts 4 x 2^-22; the weight's parts 2^-21; sums of n numbers
# (n + 8) x 2^-24.  Numerator and denominator: twice that.
@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("Hq,Hkv,nodes", [(4, 1, [8, 3, 5]), (4, 2, [1, 7, 8]), (4, 1, [16, 9, 12]), (4, 1, [32, 17, 20]), (4, 1, [64, 33, 50]),
                                          (8, 1, [64, 40, 64])])
def test_tree_outputs_are_the_nearest_but_for_fp32(torch, steps, Hq, Hkv, nodes, negative):  # noqa: F811
    rng = np.random.default_rng(Hq + nodes[0])
    c = trees([20, 0, 3], nodes, Hq, Hkv, 63 + nodes[0])
    c["q"][:] = 0
    c["q"][:, :, 0] = rng.choice([0.5, 1, 2], c["q"].shape[:2])
    for k in (c["k"], c["kc"]):
        k[..., 0] = rng.uniform(-4, 4, k.shape[:-1])
    for v in (c["v"], c["vc"]):
        v[:] = 4 * v
    scale = -1.0 if negative else 1.0
    got, _ = run_trees(torch, steps, c, scale)
    for at, h, n, (out, _, mag, _) in oracle(c, scale):
        rel = 2 * (36 * 2.0 ** -24 * np.log(2) + 4 * 2.0 ** -22 + 2.0 ** -21 + (n + 8) * 2.0 ** -24)
        with np.errstate(over="ignore"):
            step = np.spacing(np.abs(out).astype(np.float16)).astype(np.float64)
        tol = rel * mag + FLOOR * n * 16 + step / 2
        diff = np.abs(got[at, h].astype(np.float64) - out)
        assert np.all(diff <= tol), (h, n, float((diff / tol).max()), float((diff - step / 2).max()))

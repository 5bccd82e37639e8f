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

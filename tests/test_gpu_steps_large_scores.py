"""Prompt attention and tree attention where scores are large: a row's largest keys have
all the weight, however coarse fp32 is at their scores.

Scores are one product each and exact; steps between different ones are 2^7 and more,
so that smaller ones weigh less than e^-128.  What is left is the mean of the values
of the keys that share the maximum: their weights, alike, rounded to fp16, 2^-11; the sums,
2^-20; half an output step.  The log-sum-exp is the largest score, 2^-22 of it, and
the logarithm of how many keys share it.
"""
import numpy as np
import pytest

from oracle import steps as O
from test_gpu_steps import oracle, prompts, run_prompts, run_trees, steps, torch, trees  # noqa: F401

pytestmark = pytest.mark.gpu
SIZES = [2.0 ** e for e in (7, 10, 13, 15, 18, 22, 26)]      # the smallest step; the largest score is up to 2^11 of it


def check(results, got, lse):
    rows = np.zeros(got.shape[:2], bool)
    for at, h, _, (out, ref, mag, _) in results:
        rows[at, h] = True
        tol = (2.0 ** -11 + 2.0 ** -20) * mag + np.maximum(np.abs(out) * 2.0 ** -11, 2.0 ** -25)
        diff = np.abs(got[at, h].astype(np.float64) - out)
        assert np.all(diff <= tol), (at, h, float(diff.max()))
        empty = np.isneginf(ref)
        assert np.isneginf(lse[at, h][empty]).all()
        off = np.abs(lse[at, h][~empty] - ref[~empty])
        assert np.all(off <= 2.0 ** -22 * (np.abs(ref[~empty]) + 12) + 2.0 ** -18), (at, h)
    return rows


def scores(rng, q, keys, size, low):
    """scale q . k = size x a whole number of 11 bits and a sign, from `low` on."""
    q[:], q[..., 0] = 0, 2.0 ** 15
    for k in keys:
        k[..., 0] = rng.integers(low, 2 ** 11 if low < 0 else low + 40, k.shape[:-1]) * (size / 2.0 ** 23)
    return 2.0 ** 8      # the scale


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("low", [-2 ** 11 + 1, 1000])      # far apart, and with many that share the maximum
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("lens,Hq,Hkv", [([200, 70], 4, 2), ([700], 2, 1)])
def test_prompt_large_scores(torch, steps, lens, Hq, Hkv, size, low, negative):  # noqa: F811
    rng = np.random.default_rng(int(np.log2(size)))
    q, k, v, offsets = prompts(lens, Hq, Hkv, 81)
    scale = scores(rng, q, [k], size, low)
    scale = -scale if negative else scale
    got, lse = run_prompts(torch, steps, q, k, v, offsets, scale)
    assert check(O.prompt(q, k, v, offsets, scale), got, lse).all()
    v[40, 0, 3] = np.nan                               # key by key
    bad, _ = run_prompts(torch, steps, q, k, v, offsets, scale)
    assert np.array_equal(bad[:40], got[:40]) or np.allclose(bad[:40].astype(float), got[:40].astype(float), rtol=2 ** -9, atol=2 ** -24)


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("low", [-2 ** 11 + 1, 1000])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("lens,nodes", [([900, 0, 33], [8, 5, 3]), ([900, 0, 33], [16, 5, 3]), ([900, 0, 33], [32, 5, 3]),
                                        ([900, 0, 33], [64, 5, 3])])
def test_tree_large_scores(torch, steps, lens, nodes, size, low, negative):  # noqa: F811
    rng = np.random.default_rng(int(np.log2(size)))
    c = trees(lens, nodes, 4, 1, 82)
    scale = scores(rng, c["q"], [c["k"], c["kc"]], size, low)
    scale = -scale if negative else scale
    got, lse = run_trees(torch, steps, c, scale)
    assert check(oracle(c, scale), got, lse).all()

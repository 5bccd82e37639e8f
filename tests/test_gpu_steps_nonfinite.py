"""Infinities and NaNs in prompt attention and tree attention: they reach the rows
that attend them and no others, and cost a call nothing but the keys beside them."""
import numpy as np
import pytest

from oracle import steps as O
from test_gpu_steps import SCALE, check, oracle, prompts, run_prompts, run_trees, steps, torch, trees  # noqa: F401

pytestmark = pytest.mark.gpu


def check_finite(results, got, lse, scale):
    """As check; what is not finite in the oracle's results is not in `got`, and nothing else."""
    clean, clean_lse = got.copy(), lse.copy()

    def finite():
        for at, h, n, (out, ref, mag, most) in results:
            bad, lost = ~np.isfinite(out), np.isnan(ref)
            assert np.array_equal(~np.isfinite(got[at, h]), bad), (at, h)
            assert np.array_equal(np.isnan(lse[at, h]), lost), (at, h)
            clean[at, h][bad] = 0
            clean_lse[at, h][lost] = 0
            yield at, h, n, (np.where(bad, 0, out), np.where(lost, 0, ref), np.where(bad, 0, mag), np.where(np.isfinite(most), most, 0))

    with np.errstate(all="ignore"):
        return check(finite(), clean, clean_lse, scale)


def spoil(rng, k, v, tokens, values):
    """Some tokens' K or V with a number that is not finite, one head and dim each."""
    for i, t in enumerate(tokens):
        h, d = rng.integers(0, k.shape[1]), rng.integers(0, 128)
        # k: NaN only, an infinite score would depend on a sum's order
        if i % 3 == 0:
            k[t, h, d] = np.nan
        else:
            v[t, h, d] = values[i % len(values)]


VALUES = [np.nan, np.inf, -np.inf]


@pytest.mark.parametrize("scale", [SCALE, -SCALE, 0.0])
@pytest.mark.parametrize("lens,Hq,Hkv", [([40], 1, 1), ([200, 90, 1], 4, 2), ([130, 61], 7, 1), ([300], 8, 1), ([257, 64, 300], 40, 1),
                                         ([300], 4, 2), ([700], 2, 1)])
def test_prompt_numbers_that_are_not_finite(torch, steps, lens, Hq, Hkv, scale):  # noqa: F811
    rng = np.random.default_rng(sum(lens) + Hq)
    q, k, v, offsets = prompts(lens, Hq, Hkv, sum(lens) + Hq, pad=3)
    late = [hi - 1 - int(x) for lo, hi in zip(offsets[:-1], offsets[1:]) for x in rng.integers(0, min(hi - lo, 40), 4)]
    spoil(rng, k, v, late, VALUES)
    got, lse = run_prompts(torch, steps, q, k, v, offsets, scale)
    assert check_finite(O.prompt(q, k, v, offsets, scale), got, lse, scale)[:-3].all()
    assert (got[-3:] == 7).all()


def test_prompt_every_value_not_finite(torch, steps):  # noqa: F811
    # whole rows of every second token, from some token on
    q, k, v, offsets = prompts([190], 3, 1, 50)
    v[100::2] = np.inf
    v[101::4] = np.nan
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert check_finite(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE).all()


@pytest.mark.parametrize("value", [0.0, np.nan])
def test_prompt_of_subnormal_keys_and_values(torch, steps, value):  # noqa: F811
    # by the products of whole tiles (0) and key by key (NaN)
    q, k, v, offsets = prompts([150], 4, 2, 51, offset=0)
    q *= np.float16(4000)
    k *= np.float16(2 ** -17)
    v *= np.float16(2 ** -17)
    v[-1, :, 7] = value
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert check_finite(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE).all()


@pytest.mark.parametrize("scale", [SCALE, -SCALE, 0.0])
@pytest.mark.parametrize("lens,nodes,Hq,Hkv", [([70, 0, 300], [8, 5, 3], 4, 1), ([70, 0, 300], [16, 9, 12], 4, 1),
                                               ([70, 513, 0], [32, 20, 31], 4, 1), ([70, 257, 0], [64, 50, 33], 8, 1),
                                               ([40, 4000], [64, 64], 2, 2)])
def test_tree_numbers_that_are_not_finite(torch, steps, lens, nodes, Hq, Hkv, scale):  # noqa: F811
    rng = np.random.default_rng(sum(lens) + Hq)
    c = trees(lens, nodes, Hq, Hkv, sum(lens) + Hq, pad=2)
    spoil(rng, c["k"], c["v"], rng.integers(0, sum(nodes), 6), VALUES)
    c["vc"][c["table"][0, 2], 0, 3, 17] = np.inf      # a cached token, attended by its whole request
    got, lse = run_trees(torch, steps, c, scale)
    assert check_finite(oracle(c, scale), got, lse, scale)[:-2].all()


# A number that is not finite in a token that everybody attends is everybody's: such
# a call takes as long as another.  The factor is far from both sides: 1 here, 10 and
# more where the keys are taken one by one.
FACTOR = 3


def shortest(torch, call):  # noqa: F811
    times = []
    for _ in range(8):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times[2:])


@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_prompt_takes_no_longer_after_a_number_that_is_not_finite(torch, steps, value):  # noqa: F811
    n, Hq, Hkv = 4096, 8, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((n, h, 128), generator=g, device="cuda", dtype=torch.float16) for h in (Hq, Hkv, Hkv))
    offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    clean = shortest(torch, lambda: steps.prompt_attention(q, k, v, offsets, SCALE))
    assert shortest(torch, lambda: steps.prompt_attention(q, k, v, offsets, 0.0)) < FACTOR * clean
    for x, at in ((v, 0), (v, n // 2), (k, 0), (q, n // 2)):
        keep = x[at, :, 3].clone()
        x[at, :, 3] = value
        assert shortest(torch, lambda: steps.prompt_attention(q, k, v, offsets, SCALE)) < FACTOR * clean
        x[at, :, 3] = keep


@pytest.mark.parametrize("nodes", [4, 16, 32, 64])
def test_tree_takes_no_longer_after_a_number_that_is_not_finite(torch, steps, nodes):  # noqa: F811
    B, blocks, Hq, Hkv = 16, 500, 32, 8
    g = torch.Generator(device="cuda").manual_seed(2)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float16)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    T = B * nodes
    q, k, v, kc, vc = normal(T, Hq, 128), normal(T, Hkv, 128), normal(T, Hkv, 128), normal(blocks, Hkv, 16, 128), normal(blocks, Hkv, 16, 128)
    table, lens = ints([list(range(blocks))] * B), ints([blocks * 16] * B)
    mask = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    args = [q, k, v, ints(range(0, T + 1, nodes)), mask, kc, vc, table, lens, nodes]
    clean = shortest(torch, lambda: steps.tree_attention(*args, SCALE))
    assert shortest(torch, lambda: steps.tree_attention(*args, 0.0)) < FACTOR * clean
    vc[::50, :, 5, 9] = np.nan
    assert shortest(torch, lambda: steps.tree_attention(*args, SCALE)) < FACTOR * clean
    q[:, 0, 0] = np.nan
    assert shortest(torch, lambda: steps.tree_attention(*args, SCALE)) < FACTOR * clean

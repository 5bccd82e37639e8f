"""The attention over the 4-bit KV cache rounds its probabilities to nearest: its
results are not pulled to one side.

The mean of (result - exact) / exact over N results.  A result is rounded to fp16,
uniformly within 2^-11 of itself at most: a standard deviation of 2^-11 / sqrt(3),
and of 2^-11 / sqrt(3 N) for the mean; six of these are allowed, 1.7e-6 for N =
2^20.  The other roundings are of fp32 sums (2^-24 of a result, a few times) and the
probabilities', 16 bits to nearest, 2^-16 at most each and to either side: their
means are far below.  (Cut off instead, the second part's 8 bits lose half their last one
on average, 2^-17 of the binade's start, times 4/3 for where the second part's first
bit lies, over a mean weight of 1.44 binade's starts: 7e-6 to one side.)
"""
import numpy as np
import pytest

from oracle import kv4 as O
from test_gpu_kv4 import BS, D, SLAB, dev, kv4, torch  # noqa: F401  (two are fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv", [(32, 32), (32, 16), (64, 16), (128, 16)])
def test_results_are_not_pulled_to_one_side(torch, kv4, Hq, Hkv):  # noqa: F811
    B = (1 << 20) // (Hq * D)
    rng = np.random.default_rng(Hq)
    width = 5
    lens = rng.integers(30, width * BS, B).astype(np.int32)
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    q = rng.standard_normal((B, Hq, D)).astype(np.float16)
    # K of any codes, at most 3 in magnitude; V from 0.5 to 6: a relative error means
    # something
    cache = rng.integers(0, 256, (B * width, Hkv, SLAB), dtype=np.uint8)
    low, high = rng.integers(1, 8, (2, B * width, Hkv, 1024), dtype=np.uint8)
    cache[..., 1024:2048] = low | high << 4
    cache[..., 2048:2112] = 126
    cache[..., 2112:] = 127
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    got = kv4.attention(dq, dc, dt, dl, 0.09).cpu().numpy().astype(np.float64)
    want, _ = O.attention(q, cache, table, lens, np.float32(0.09))
    mean = float(((got - want) / want).mean())
    print(f"[kv4] {Hq}/{Hkv}: mean relative error {mean:.2e}", flush=True)
    assert abs(mean) <= 6 * 2.0 ** -11 / np.sqrt(3 * want.size)

"""Scores of rows whose four groups of 32 dims have scales far apart, as a model's
outlier channels make them: the groups' sums are joined to fp32 precision.

A request of one token has its score for its log-sum-exp, so the score is seen as it
is.  The bounds are those of test_gpu_kv4.py: 2^-21 of the sum of the products'
magnitudes, and q's last digit.
"""
import numpy as np
import pytest

from oracle import kv4 as O
from test_gpu_kv4 import BS, D, check_attention, dev, kv4, poisoned, torch  # noqa: F401  (two are fixtures)

pytestmark = pytest.mark.gpu
B = 96


def rows_of(kind, rng, shape):
    """K rows [...][128] and the scale of q's groups [...][4]."""
    k = rng.standard_normal((*shape, 4, 32))
    if kind == "outlier group":
        return k * 2.0 ** np.array([0, 9, 0, -6])[:, None], np.ones(4)
    if kind == "any scales":
        return k * 2.0 ** rng.integers(-12, 13, (*shape, 4, 1)), np.ones(4)
    if kind == "small values times large ones":
        # every group's products of one size: q falls as K rises (within q's 2^-8)
        e = np.array([0, 6, 3, -1])
        return k * 2.0 ** e[:, None], 2.0 ** -np.maximum(e, 0.0)
    assert kind == "large groups cancel"
    k *= np.array([2.0 ** 10, 1, 2.0 ** 10, 1])[:, None]
    k[..., 2, :] = -k[..., 0, :]                       # (q is the same in both)
    return k, np.ones(4)


@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("kind", ["outlier group", "any scales", "small values times large ones", "large groups cancel"])
def test_scores(torch, kv4, kind, Hq, Hkv):  # noqa: F811
    rng = np.random.default_rng(Hq)
    lens = np.concatenate([np.ones(B - 4), [40, 17, 300, 5]]).astype(np.int32)
    width = int(-(-lens.max() // BS))
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    cache = poisoned(B * width, Hkv, 1)
    slots = np.concatenate([table[b, t // BS].astype(np.int64) * BS + t % BS for b, t in enumerate(map(np.arange, lens))])
    k, of_q = rows_of(kind, rng, (len(slots), Hkv))
    v = rng.standard_normal((len(slots), Hkv, D)).astype(np.float16)
    O.append(cache, k.reshape(len(slots), Hkv, D).astype(np.float16), v, slots)
    q = rng.standard_normal((B, Hq, 4, 32)) * of_q[:, None]
    if kind == "large groups cancel":
        q[:, :, 2] = q[:, :, 0]
    q = q.reshape(B, Hq, D).astype(np.float16)
    scale = 0.09 if kind in ("small values times large ones", "large groups cancel") else 2.0 ** -10
    dq, dc, dt, dl = dev(torch, q, cache, table, lens)
    lse = torch.empty((B, Hq), dtype=torch.float32, device="cuda")
    out = kv4.attention(dq, dc, dt, dl, scale, lse_out=lse)
    worst = check_attention(out.cpu().numpy(), lse.cpu().numpy(), q, cache, table, lens, scale)
    _, ref = O.attention(q, cache, table, lens, scale)
    print(f"[kv4] {kind}, {Hq}/{Hkv}: {worst:.3f} of the tolerance; scores up to {np.abs(ref).max():.3g}, the log-sum-exp off by up "
          f"to {np.abs(lse.cpu().numpy() - ref).max():.2g}", flush=True)

"""Prompt attention and tree attention on the GPU against their oracle
(oracle/steps.py, 64 bits).

Tolerances, from the arithmetic, for a row that sees n keys:
  score    128 products summed in fp32: 128 x 2^-24 of the sum of their
           magnitudes, times |scale|; scale x log2 e and the product with it round
           by 2^-24 each, of a score that is no larger than that sum: 2^-22 more;
  weight   the score's error, relative; the exponential 2^-22; as fp16 half a step,
           2^-11; weights are held 2^7 or more above the row's largest one's
           definition, so what lies among the subnormals is off by 2^-25 x 2^-7 of it;
  sums     of the weights and of weight x V in fp32, rescaled now and then:
           n x 2^-24 + 2^-20 each;
  out      the numerator's and the denominator's errors times sum(weight |V|), and
           half an fp16 step, 2^-11 of the value (or half the smallest, 2^-25);
  lse      the score's error, that of the sum of the weights, 2^-22 of itself.
"""
import numpy as np
import pytest

from oracle import steps as O

pytestmark = pytest.mark.gpu
D, BS = 128, 16
SCALE = float(np.float32(1 / np.sqrt(128)))


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.fixture(scope="module")
def steps():
    from paper_2506_03296_amd import steps as S
    S.load_library()
    return S


def dev(torch, *arrays):
    out = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]
    return out if len(out) > 1 else out[0]


def check(results, got, lse, scale):
    """Every row that the oracle yields within its tolerance; returns the rows."""
    rows = np.zeros(got.shape[:2], bool)
    for at, h, n, (out, ref, mag, most) in results:
        rows[at, h] = True
        err = abs(scale) * most * (2.0 ** -17 + 2.0 ** -22)
        total = n * 2.0 ** -24 + 2.0 ** -20
        rel = 2 * err + 2 * 2.0 ** -22 + 2.0 ** -11 + n * 2.0 ** -32 + 2 * total
        tol = rel[:, None] * mag + np.maximum(np.abs(out) * 2.0 ** -11, 2.0 ** -25)
        diff = np.abs(got[at, h].astype(np.float64) - out)
        assert np.all(diff <= tol), (at, h, n, float((diff / tol).max()))
        if lse is not None:
            empty = np.isneginf(ref)
            assert np.all(np.isneginf(lse[at, h][empty]))
            lt = err + 2.0 ** -22 * (1 + np.abs(ref)) + total
            with np.errstate(invalid="ignore"):
                off = np.abs(lse[at, h].astype(np.float64) - ref)
            assert np.all(off[~empty] <= lt[~empty]), (at, h, n, off[~empty].max())
    return rows


def normal(rng, *shape):
    return rng.standard_normal(shape).astype(np.float16)


def offsets_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


# --- prompts ---------------------------------------------------------------------

def prompts(lens, Hq, Hkv, seed, pad=0, offset=0.5):
    """q, k, v, offsets; `pad` rows of NaNs behind the last request."""
    rng = np.random.default_rng(seed)
    T = int(sum(lens)) + pad
    q, k, v = normal(rng, T, Hq, D), normal(rng, T, Hkv, D) + np.float16(offset) * normal(rng, 1, Hkv, D), normal(rng, T, Hkv, D)
    if pad:
        q[-pad:], k[-pad:], v[-pad:] = np.nan, np.nan, np.nan
    return q, k, v, offsets_of(lens)


def run_prompts(torch, steps, q, k, v, offsets, scale=SCALE, stream=None):
    dq, dk, dv, do = dev(torch, q, k, v, offsets)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    assert steps.prompt_attention(dq, dk, dv, do, scale, out=out, lse_out=lse, stream=stream) is out
    torch.cuda.synchronize()
    return out.cpu().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (2, 1), (4, 1), (16, 2), (6, 2), (7, 1), (40, 1)])
@pytest.mark.parametrize("lens", [[1], [2], [33], [64], [65], [1, 0, 31, 32, 0, 1], [127, 63, 3], [257, 129, 64]])
def test_prompts(torch, steps, lens, Hq, Hkv):
    q, k, v, offsets = prompts(lens, Hq, Hkv, sum(lens) + Hq, pad=3)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    rows = check(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE)
    assert rows[:-3].all()
    assert (got[-3:] == 7).all() and (lse[-3:] == 7).all()      # padding is left as it was


@pytest.mark.parametrize("seed", range(4))
def test_prompts_at_random(torch, steps, seed):
    rng = np.random.default_rng(100 + seed)
    lens = rng.integers(0, 400, rng.integers(1, 9)).tolist() + [int(rng.integers(1, 700))]
    Hkv = int(rng.integers(1, 4))
    Hq = Hkv * int(rng.integers(1, 10))
    q, k, v, offsets = prompts(lens, Hq, Hkv, seed)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert check(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE).all()


@pytest.mark.parametrize("B,Hq,Hkv,most", [(64, 4, 1, 40), (65, 4, 1, 40), (65, 8, 8, 130), (300, 3, 1, 9), (4200, 2, 2, 3)])
def test_prompts_of_many_requests(torch, steps, B, Hq, Hkv, most):
    rng = np.random.default_rng(B)
    lens = rng.integers(0, most, B)
    lens[rng.permutation(B)[:2]] = [300, 0]
    q, k, v, offsets = prompts(lens.tolist(), Hq, Hkv, B)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert check(O.prompt(q, k, v, offsets, SCALE), got, lse, SCALE).all()


@pytest.mark.parametrize("scale", [0.0, -SCALE, 1.0, -3.0, 1e-6])
def test_prompt_scales(torch, steps, scale):
    scale = float(np.float32(scale))
    q, k, v, offsets = prompts([150, 70], 4, 2, 11)
    got, lse = run_prompts(torch, steps, q, k, v, offsets, scale)
    assert check(O.prompt(q, k, v, offsets, scale), got, lse, scale).all()


def test_prompt_whose_maximum_keeps_rising(torch, steps):
    # scores grow along the keys, by more and by less than the running maximum's slack
    q, k, v, offsets = prompts([700], 2, 1, 12, offset=0)
    q[:], k[:] = 0.25, 0
    k[:, 0, 0] = np.linspace(0, 2000, 700).astype(np.float16)
    k[300:, 0, 1] = -500
    got, lse = run_prompts(torch, steps, q, k, v, offsets, 0.125)
    assert check(O.prompt(q, k, v, offsets, 0.125), got, lse, 0.125).all()


def test_prompt_weights_far_below_the_largest(torch, steps):
    # one key above all others by 2^24 and more: what the many small ones add up to still counts
    n = 3000
    q, k, v, offsets = prompts([n], 1, 1, 13, offset=0)
    q[:], k[:], v[:] = 0, 0, 1
    q[:, 0, 0], k[0, 0, 0], v[0] = 1, 17.0, 0
    got, lse = run_prompts(torch, steps, q, k, v, offsets, 1.0)
    assert check(O.prompt(q, k, v, offsets, 1.0), got, lse, 1.0).all()


def test_prompt_out_of_a_fused_projection(torch, steps):
    rng = np.random.default_rng(14)
    lens, Hq, Hkv = [90, 1, 200], 8, 2
    x = normal(rng, sum(lens), Hq + 2 * Hkv + 1, D)
    dx, do = dev(torch, x, offsets_of(lens))
    q, k, v = dx[:, :Hq], dx[:, Hq:Hq + Hkv], dx[:, Hq + Hkv:Hq + 2 * Hkv]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    lse = torch.empty((sum(lens), Hq), dtype=torch.float32, device="cuda")
    out = steps.prompt_attention(q, k, v, do, SCALE, lse_out=lse, stream=s)
    s.synchronize()
    got = check(O.prompt(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:Hq + 2 * Hkv], offsets_of(lens), SCALE),
                out.cpu().numpy(), lse.cpu().numpy(), SCALE)
    assert got.all()


@pytest.mark.parametrize("stride", [(1 << 23) - 8, (1 << 23) + 8])
@pytest.mark.parametrize("lens", [[300], [100, 130, 69]])
def test_prompt_rows_far_apart(torch, steps, lens, stride):
    """Tokens 16 MiB apart: a tile's rows span 2^30 bytes and more, the batch 2^32."""
    T, Hq, Hkv = sum(lens), 4, 2
    q, k, v, offsets = prompts(lens, Hq, Hkv, T + stride % 16)
    base = torch.empty(T * stride, dtype=torch.float16, device="cuda")
    views, at = [], 0
    for x in (q, k, v):
        view = base.as_strided(x.shape, (stride, D, 1), at)
        view.copy_(dev(torch, x))
        views.append(view)
        at += x.shape[1] * D
    lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
    out = steps.prompt_attention(*views, dev(torch, offsets), SCALE, lse_out=lse)
    assert check(O.prompt(q, k, v, offsets, SCALE), out.cpu().numpy(), lse.cpu().numpy(), SCALE).all()


def test_tree_of_rows_far_apart(torch, steps):
    c = trees([70, 0, 300], [40, 64, 3], 4, 2, 41)
    args = list(device(torch, c))
    T, stride = c["q"].shape[0], (1 << 25) + 8
    base, at = torch.empty(T * stride, dtype=torch.float16, device="cuda"), 0
    for i in range(3):
        x = args[i]
        args[i] = base.as_strided(x.shape, (stride, D, 1), at)
        args[i].copy_(x)
        at += x.shape[1] * D
    lse = torch.empty((T, 4), dtype=torch.float32, device="cuda")
    out = steps.tree_attention(*args, SCALE, lse_out=lse)
    check(oracle(c), out.cpu().numpy(), lse.cpu().numpy(), SCALE)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("which", ["k", "v"])
def test_prompt_later_tokens_do_not_count(torch, steps, which, value):
    lens, Hq, Hkv = [200, 90], 4, 2
    q, k, v, offsets = prompts(lens, Hq, Hkv, 15)
    clean, clean_lse = run_prompts(torch, steps, q, k, v, offsets)
    bad = {"k": k, "v": v}[which]
    bad[140, 0, 5] = value
    bad[200 + 3, 1, 100] = value
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    G = Hq // Hkv
    for h, first, end in ((0, 140, 200), (1, 203, 290)):
        heads = slice(h * G, h * G + G)
        other = np.ones(290, bool)
        other[first:end] = False
        sees = np.isclose(got[other, heads], clean[other, heads], rtol=2 ** -9, atol=2 ** -12)
        assert sees.all()
        if which == "v":
            dim = 5 if h == 0 else 100
            assert not np.isfinite(got[first:end, heads, dim]).any()
            assert np.isfinite(np.delete(got[first:end, heads], dim, -1)).all()
            assert np.allclose(lse, clean_lse, rtol=0, atol=2 ** -15)


def test_prompt_all_scores_minus_infinity(torch, steps):
    q, k, v, offsets = prompts([70], 1, 1, 16)
    q[:] = 1
    k[:, 0, 0] = -np.inf
    k[40:, 0, 0] = 0
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    assert (got[:40] == 0).all() and np.isneginf(lse[:40]).all()
    k[:40] = 0
    q0, k0, v0 = q[40:], k[40:], v[40:]
    assert check(O.prompt(q0, k0, v0, [0, 30], SCALE), got[40:], lse[40:], SCALE).all()


def test_prompt_offsets_out_of_order_stay_in_bounds(torch, steps):
    q, k, v, _ = prompts([300], 4, 2, 17)
    for offsets in ([0, 200, 100, 300], [-5, 1000, 300, 300], [300, 0, 0, 0], [250, 250, 300, 2 ** 31 - 1]):
        got, _ = run_prompts(torch, steps, q, k, v, np.array(offsets, np.int32))
        assert np.isfinite(got).all()


def test_prompt_long_against_fp32(torch, steps):
    # 9001 tokens: rows here and there against a plain product in 64 bits
    n, Hq, Hkv = 9001, 8, 2
    q, k, v, offsets = prompts([n], Hq, Hkv, 18)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    G = Hq // Hkv
    for r in [0, 1, 63, 64, 4095, 4096, 6000, 8959, 8960, 9000]:
        for h in range(Hq):
            one = O.attend(q[r:r + 1, h], k[:r + 1, h // G], v[:r + 1, h // G], SCALE, np.ones((1, r + 1), bool))
            check([(slice(0, 1), 0, r + 1, one)], got[r:r + 1, h:h + 1], lse[r:r + 1, h:h + 1], SCALE)


def plain64(torch, q, k, v, offsets, scale):
    """out, lse and the sums of weight x |V| of packed prompts, in 64 bits on the GPU."""
    G = q.shape[1] // k.shape[1]
    out, lse, mag, most = [], [], [], []
    for lo, hi in zip(offsets[:-1], offsets[1:]):
        a, b, c = (x[lo:hi].double().transpose(0, 1) for x in (q, k, v))
        b, c = b.repeat_interleave(G, 0), c.repeat_interleave(G, 0)
        bt = b.transpose(1, 2).contiguous()
        s = (a @ bt * scale).masked_fill(torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").triu(1), -np.inf)
        w = torch.softmax(s, -1)
        out.append((w @ c).transpose(0, 1))
        mag.append((w @ c.abs()).transpose(0, 1))
        lse.append(torch.logsumexp(s, -1).transpose(0, 1))
        most.append((a.abs() @ bt.abs()).tril().amax(-1).transpose(0, 1))
    return [torch.cat(x).cpu().numpy() for x in (out, lse, mag, most)]


@pytest.mark.parametrize("B,n,Hq,Hkv", [(64, 200, 32, 32), (40, 300, 16, 16), (20, 300, 32, 8), (7, 500, 64, 32), (150, 70, 12, 12),
                                        (1, 3000, 64, 8)])
def test_prompts_of_many_tiles(torch, steps, B, n, Hq, Hkv):
    """Several tiles a work group: 1 to 14 to a compute unit."""
    rng = np.random.default_rng(B)
    lens = rng.integers(n // 2, n + 1, B).tolist()
    lens[-1] = n
    q, k, v, offsets = prompts(lens, Hq, Hkv, B)
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    out, ref, mag, most = plain64(torch, *dev(torch, q, k, v), offsets.tolist(), SCALE)
    for h in range(Hq):
        check([(slice(0, sum(lens)), h, n, (out[:, h], ref[:, h], mag[:, h], most[:, h]))], got, lse, SCALE)


@pytest.mark.parametrize("lens,Hq,Hkv", [([256], 1, 1), ([257], 4, 1), ([511], 3, 3), ([1100], 2, 2), ([2051], 4, 2), ([1, 0, 900], 8, 2),
                                         ([64, 449], 16, 2), ([300, 320, 257], 6, 2), ([1500], 32, 4)])
def test_prompts_whose_keys_two_waves_share(torch, steps, lens, Hq, Hkv):
    """Few prompts of some length: every second 64 keys are another wave's."""
    q, k, v, offsets = prompts(lens, Hq, Hkv, sum(lens) + Hq, pad=2)
    k[64:128] *= np.float16(4)                  # some rows' largest weights in either's keys
    got, lse = run_prompts(torch, steps, q, k, v, offsets, -SCALE)
    assert (got[-2:] == 7).all() and (lse[-2:] == 7).all()
    out, ref, mag, most = plain64(torch, *dev(torch, q, k, v), np.unique(offsets).tolist(), -SCALE)
    for h in range(Hq):
        check([(slice(0, sum(lens)), h, max(lens), (out[:, h], ref[:, h], mag[:, h], most[:, h]))], got, lse, SCALE)


@pytest.mark.parametrize("dead", [range(0, 64), range(64, 128), range(0, 300), [i for i in range(500) if i // 64 % 2], range(0, 500)])
def test_prompt_scores_of_minus_infinity_among_shared_keys(torch, steps, dead):
    n, dead = 500, list(dead)
    q, k, v, offsets = prompts([n], 2, 1, 19)
    q[:, :, 0] = 1
    k[:, :, 0] = 0
    sees = np.ones(n, bool)
    sees[dead] = False
    k[dead, :, 0] = -np.inf
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    k[:, :, 0] = 0
    for r in list(range(0, n, 7)) + [n - 1]:
        keys = np.flatnonzero(sees[:r + 1])
        for h in range(2):
            if not len(keys):
                assert (got[r, h] == 0).all() and np.isneginf(lse[r, h])
                continue
            one = O.attend(q[r:r + 1, h], k[keys, 0], v[keys, 0], SCALE, np.ones((1, len(keys)), bool))
            check([(slice(0, 1), 0, len(keys), one)], got[r:r + 1, h:h + 1], lse[r:r + 1, h:h + 1], SCALE)


@pytest.mark.parametrize("key", [70, 130, 299])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_prompt_later_values_do_not_count_where_keys_are_shared(torch, steps, key, value):
    q, k, v, offsets = prompts([300], 4, 2, 20)
    clean, _ = run_prompts(torch, steps, q, k, v, offsets)
    v[key, 0, 5] = value
    got, lse = run_prompts(torch, steps, q, k, v, offsets)
    before, heads = np.arange(300) < key, slice(0, 2)
    assert np.isclose(got[before], clean[before], rtol=2 ** -9, atol=2 ** -12).all()
    assert np.isclose(got[:, 2:], clean[:, 2:], rtol=2 ** -9, atol=2 ** -12).all()
    assert not np.isfinite(got[~before, heads, 5]).any()
    assert np.isfinite(np.delete(got[:, heads], 5, -1)).all() and np.isfinite(lse).all()


def test_attention_refuses_what_it_cannot_read(torch, steps):
    c = trees([20, 5], [3, 4], 4, 2, 40)
    a = device(torch, c)
    q, k, v, o = a[:4]
    for bad in ((q.float(), k, v, o), (q, k.bfloat16(), v, o), (q[:5], k, v, o), (q, k[:, :1], v, o), (q[..., :64], k, v, o),
                (q, k, v, o.long()), (q, k, v, o.cpu()), (q.cpu(), k, v, o), (q, k.cpu(), v, o), (q, k, v[:6], o),
                (q.transpose(1, 2).contiguous().transpose(1, 2), k, v, o), (q, k, torch.cat([v, v], 1)[:, :2], o)):
        with pytest.raises((ValueError, TypeError)):
            steps.prompt_attention(*bad, SCALE)
        with pytest.raises((ValueError, TypeError)):
            steps.tree_attention(*bad, *a[4:], SCALE)
    for i, bad in ((4, a[4].int()), (4, a[4][:3]), (5, a[5].float()), (5, a[5][:, :1]), (6, a[6][1:]), (7, a[7].long()),
                   (7, a[7][:1]), (8, a[8][:1]), (8, a[8].cpu())):
        with pytest.raises((ValueError, TypeError)):
            steps.tree_attention(*a[:i], bad, *a[i + 1:], SCALE)
    for kw in (dict(out=torch.empty_like(q)[:2]), dict(out=q.float()), dict(lse_out=torch.empty(7, 3, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            steps.prompt_attention(q, k, v, o, SCALE, **kw)
    import paper_2506_03296_amd as A
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    for kw in (dict(workspace=small),):
        with pytest.raises(A.ApexError):
            steps.tree_attention(*a, SCALE, **kw)
    with pytest.raises(A.ApexError):
        steps.prompt_attention(q, k, v, o, SCALE, out=q)
    with pytest.raises(A.ApexError, match="capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            steps.tree_attention(*a, SCALE)


def test_prompt_captured_and_replayed(torch, steps):
    q, k, v, offsets = prompts([130, 0, 61], 4, 1, 19)
    dq, dk, dv, do = dev(torch, q, k, v, offsets)
    out = torch.zeros_like(dq)
    lse = torch.zeros(q.shape[:2], dtype=torch.float32, device="cuda")
    eager = steps.prompt_attention(dq, dk, dv, do, SCALE)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps.prompt_attention(dq, dk, dv, do, SCALE, out=out, lse_out=lse)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    # other lengths in the same buffers
    do.copy_(torch.tensor([0, 5, 100, 191], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert check(O.prompt(q, k, v, [0, 5, 100, 191], SCALE), out.cpu().numpy(), lse.cpu().numpy(), SCALE).all()


def test_prompts_whose_keys_two_waves_share_replayed_with_other_lengths(torch, steps):
    q, k, v, offsets = prompts([600, 100], 4, 2, 21)
    dq, dk, dv, do = dev(torch, q, k, v, offsets)
    out = torch.zeros_like(dq)
    lse = torch.zeros(q.shape[:2], dtype=torch.float32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps.prompt_attention(dq, dk, dv, do, SCALE, out=out, lse_out=lse)
    for other in ([0, 600, 700], [0, 0, 700], [0, 700, 700], [0, 1, 129], [0, 64, 640]):
        do.copy_(torch.tensor(other, dtype=torch.int32))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        rows = check(O.prompt(q, k, v, other, SCALE), got, lse.cpu().numpy(), SCALE)
        assert rows[:other[-1]].all() and (got[other[-1]:] == 7).all()


# --- trees -----------------------------------------------------------------------

def random_tree(rng, n):
    """uint64 [n]: a node sees itself and its ancestors."""
    m = [0] * n
    for i in range(n):
        p = int(rng.integers(-1, i)) if i else -1
        m[i] = (m[p] if p >= 0 else 0) | 1 << i
    return m


def trees(lens, nodes, Hq, Hkv, seed, width=None, spare=3, pad=0, masks=None):
    """Everything of a call: the cache's rows of a request at scattered blocks, the
    rest of the pool NaN, table entries behind a request's end out of range."""
    rng = np.random.default_rng(seed)
    nblk = [max(0, -(-int(L) // BS)) for L in lens]
    nb = sum(nblk) + spare
    width = max(1, max(nblk)) if width is None else width
    ids = rng.permutation(nb).astype(np.int32)
    table = np.full((len(lens), width), -9, np.int32)
    kc, vc = (np.full((nb, Hkv, BS, D), np.nan, np.float16) for _ in range(2))
    shift = np.float16(0.5) * normal(rng, Hkv, 1, D)
    i = 0
    for b, n in enumerate(nblk):
        table[b, :min(n, width)] = ids[i:i + n][:width]
        for t in range(int(max(lens[b], 0))):
            kc[ids[i + t // BS], :, t % BS] = normal(rng, Hkv, D) + shift[:, 0]
            vc[ids[i + t // BS], :, t % BS] = normal(rng, Hkv, D)
        i += n
    T = int(sum(nodes)) + pad
    q, k, v = normal(rng, T, Hq, D), normal(rng, T, Hkv, D) + shift[None, :, 0], normal(rng, T, Hkv, D)
    if pad:
        q[-pad:], k[-pad:], v[-pad:] = np.nan, np.nan, np.nan
    if masks is None:
        masks = [w for n in nodes for w in random_tree(rng, n)]
    masks = np.array(list(masks) + [2 ** 64 - 1] * pad, np.uint64)
    return dict(q=q, k=k, v=v, offsets=offsets_of(nodes), masks=masks, kc=kc, vc=vc, table=table,
                lens=np.array(lens, np.int32), max_nodes=max(max(nodes), 1))


def oracle(c, scale=SCALE):
    return O.tree(c["q"], c["k"], c["v"], c["offsets"], c["masks"], c["kc"], c["vc"], c["table"], c["lens"],
                  c["max_nodes"], scale)


def device(torch, c):
    q, k, v, o, m, kc, vc, t, n = dev(torch, c["q"], c["k"], c["v"], c["offsets"], c["masks"].view(np.int64), c["kc"],
                                      c["vc"], c["table"], c["lens"])
    return [q, k, v, o, m, kc, vc, t, n, c["max_nodes"]]


def run_trees(torch, steps, c, scale=SCALE, workspace=None, stream=None):
    args = device(torch, c)
    out = torch.full(c["q"].shape, 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full(c["q"].shape[:2], 7.0, dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    steps.tree_attention(*args, scale, out=out, lse_out=lse, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return out.cpu().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 2), (4, 1), (8, 1), (6, 2), (7, 1), (24, 2)])
@pytest.mark.parametrize("lens,nodes", [
    ([0], [1]), ([1], [1]), ([0, 5], [3, 64]), ([16, 17, 15], [5, 1, 8]), ([127, 128, 129], [8, 8, 8]),
    ([63, 64, 65], [16, 33, 64]), ([500, 0, 1], [2, 0, 64]), ([1000], [7])])
def test_trees(torch, steps, lens, nodes, Hq, Hkv):
    c = trees(lens, nodes, Hq, Hkv, sum(lens) + sum(nodes) + Hq, pad=2)
    got, lse = run_trees(torch, steps, c)
    rows = check(oracle(c), got, lse, SCALE)
    assert rows[:-2].all()
    assert (got[-2:] == 7).all() and (lse[-2:] == 7).all()


@pytest.mark.parametrize("seed", range(6))
def test_trees_at_random(torch, steps, seed):
    rng = np.random.default_rng(200 + seed)
    B = int(rng.integers(1, 20))
    Hkv = int(rng.integers(1, 4))
    Hq = Hkv * int(rng.integers(1, 9))
    most = int(rng.integers(1, 65))
    nodes = rng.integers(0, most + 1, B).tolist()
    nodes[0] = most
    c = trees(rng.integers(0, 900, B).tolist(), nodes, Hq, Hkv, seed)
    workspace = torch.full((steps.tree_workspace_bytes(most, Hq, Hkv),), 255, dtype=torch.uint8, device="cuda")
    got, lse = run_trees(torch, steps, c, workspace=workspace)      # whatever the workspace holds
    assert check(oracle(c), got, lse, SCALE).all()


@pytest.mark.parametrize("B,nodes,Hq,Hkv", [(70, 4, 4, 1), (300, 1, 2, 1), (150, 20, 8, 2), (600, 2, 8, 8)])
def test_trees_of_many_requests(torch, steps, B, nodes, Hq, Hkv):
    rng = np.random.default_rng(B)
    c = trees(rng.integers(0, 60, B).tolist(), rng.integers(1, nodes + 1, B).tolist(), Hq, Hkv, B)
    c["max_nodes"] = nodes
    got, lse = run_trees(torch, steps, c)
    assert check(oracle(c), got, lse, SCALE).all()


def test_tree_masks_of_any_kind(torch, steps):
    # nothing at all, all, itself only, others only, bits past the request's nodes
    nodes = [6, 3, 64, 2]
    masks = [0, 63, 4, 8 | 1 << 60, 2 ** 64 - 1, 1 << 6, 0, 1 << 3, 2 ** 63] + [2 ** 64 - 1 >> i for i in range(64)] + [0, 0]
    for lens in ([40, 0, 130, 0], [0, 0, 0, 0]):
        c = trees(lens, nodes, 4, 2, 21, masks=masks)
        got, lse = run_trees(torch, steps, c)
        assert check(oracle(c), got, lse, SCALE).all()
    assert (got[0] == 0).all() and np.isneginf(lse[0]).all()       # the last: no context, no bits


def test_tree_blocks_outside_the_pool_and_short_tables(torch, steps):
    for bad in (-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31):
        c = trees([300, 40, 16, 70], [9, 2, 4, 5], 4, 2, 22)
        c["table"][0, 3], c["table"][0, 17], c["table"][1, 0], c["table"][2, 0] = bad, bad, bad, bad
        got, lse = run_trees(torch, steps, c)
        assert check(oracle(c), got, lse, SCALE).all()
    c = trees([300, 40], [9, 2], 4, 2, 23, width=4)
    c["lens"][:] = [300, 2 ** 31 - 1]
    c["table"][1] = c["table"][0]
    got, lse = run_trees(torch, steps, c)
    assert check(oracle(c), got, lse, SCALE).all()
    c = trees([0, 0], [9, 2], 4, 2, 24)
    c["lens"][:] = [-4, -2 ** 31]
    got, lse = run_trees(torch, steps, c)
    assert check(oracle(c), got, lse, SCALE).all()


def test_tree_without_a_table_or_a_pool(torch, steps):
    c = trees([0, 0], [5, 30], 4, 2, 25)
    c["table"] = c["table"][:, :0]
    c["lens"][:] = 100
    got, lse = run_trees(torch, steps, c)
    assert check(oracle(c), got, lse, SCALE).all()
    c["kc"], c["vc"], c["table"] = c["kc"][:0], c["vc"][:0], np.zeros((2, 7), np.int32)
    got, lse = run_trees(torch, steps, c)
    assert check(oracle(c), got, lse, SCALE).all()


def test_tree_rows_behind_max_nodes_are_padding(torch, steps):
    c = trees([100, 30], [20, 10], 4, 2, 26)
    c["max_nodes"] = 12
    got, lse = run_trees(torch, steps, c)
    rows = check(oracle(c), got, lse, SCALE)
    assert (~rows).any(1).sum() == 8
    assert (got[12:20] == 7).all() and (lse[12:20] == 7).all()


@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("lens,nodes,Hq", [([140, 33], [5, 7], 4), ([140, 33], [12, 30], 4), ([300, 33], [40, 64], 8)])
def test_tree_tokens_out_of_sight_do_not_count(torch, steps, lens, nodes, Hq, value):
    c = trees(lens, nodes, Hq, 2, 27)
    c["masks"][:] = [1 << i | 1 for n in nodes for i in range(n)]      # all see the first, and themselves
    clean, clean_lse = run_trees(torch, steps, c)
    c["v"][2, 1, 9] = value                      # seen by row 2 only
    c["k"][nodes[0] + 3, 0, 0] = np.nan          # seen by its own row only
    c["vc"][c["table"][1, 0], 1, 4, 17] = value  # seen by all of the second request
    got, lse = run_trees(torch, steps, c)
    G, n0 = Hq // 2, nodes[0]
    bad = np.zeros(got.shape, bool)
    bad[2, G:, 9] = True
    bad[n0 + 3, :G] = True
    bad[n0:, G:, 17] = True
    assert np.array_equal(~np.isfinite(got), bad)
    assert np.allclose(got[~bad], clean[~bad], rtol=2 ** -9, atol=2 ** -12)
    keep = np.ones(lse.shape, bool)
    keep[n0 + 3, :G] = False
    assert np.allclose(lse[keep], clean_lse[keep], rtol=0, atol=2 ** -15) and np.isnan(lse[~keep]).all()


def test_tree_scales_and_negative_scales(torch, steps):
    c = trees([200, 3], [9, 4], 4, 2, 28)
    for scale in (0.0, -SCALE, 2.0):
        got, lse = run_trees(torch, steps, c, scale)
        assert check(oracle(c, scale), got, lse, scale).all()


def test_tree_rows_past_32_bits(torch, steps):
    # a pool of 9.8 GB a cache: its last blocks lie past 2^33 bytes
    nb, Hkv = 300000, 8
    c = trees([100, 37], [9, 3], 32, Hkv, 29)
    small = device(torch, c)
    n = c["kc"].shape[0]
    kc = torch.zeros((nb, Hkv, BS, D), dtype=torch.float16, device="cuda")
    vc = torch.zeros_like(kc)
    high = torch.from_numpy(nb - 1 - np.arange(n)).cuda()
    kc[high], vc[high] = small[5], small[6]
    table = torch.where(small[7] >= 0, nb - 1 - small[7], small[7])
    lse = torch.empty((12, 32), dtype=torch.float32, device="cuda")
    out = steps.tree_attention(*small[:5], kc, vc, table, *small[8:], SCALE, lse_out=lse)
    assert check(oracle(c), out.cpu().numpy(), lse.cpu().numpy(), SCALE).all()


def test_tree_captured_and_replayed(torch, steps):
    c = trees([700, 20, 0], [8, 4, 3], 4, 1, 30)
    args = device(torch, c)
    eager = steps.tree_attention(*args, SCALE)
    out = torch.zeros_like(args[0])
    size = steps.tree_workspace_bytes(c["max_nodes"], 4, 1)
    workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps.tree_attention(*args, SCALE, out=out, workspace=workspace)
    other = trees([650, 9, 8], [8, 4, 3], 4, 1, 31)
    for case in (c, other, c):
        for dst, src in zip(args[:9], device(torch, case)[:9]):
            if dst.shape == src.shape:
                dst.copy_(src)
        now = dict(case, kc=args[5].cpu().numpy(), vc=args[6].cpu().numpy(), table=args[7].cpu().numpy())
        out.zero_()
        workspace.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        if case is c:
            assert torch.equal(out, eager)
        else:
            live = now["lens"] <= now["table"].shape[1] * BS
            assert live.all()
        ref = steps.tree_attention(*args, SCALE)
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(ref))


def test_tree_two_calls_at_once(torch, steps):
    cases = [trees([900, 40], [8, 3], 8, 2, 32), trees([30, 600, 7], [20, 33, 64], 8, 2, 33)]
    args = [device(torch, c) for c in cases]
    alone = [steps.tree_attention(*a, SCALE) for a in args]
    streams = [torch.cuda.Stream() for _ in cases]
    spaces = [torch.empty(steps.tree_workspace_bytes(a[9], 8, 2), dtype=torch.uint8, device="cuda") for a in args]
    torch.cuda.synchronize()
    outs = [torch.empty_like(a[0]) for a in args]
    for _ in range(5):
        for a, s, w, o in zip(args, streams, spaces, outs):
            steps.tree_attention(*a, SCALE, out=o, workspace=w, stream=s)
    torch.cuda.synchronize()
    for o, ref in zip(outs, alone):
        assert torch.equal(o, ref)

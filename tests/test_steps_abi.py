"""Steps of several tokens a request without a GPU: symbols, refusals, and the
oracle against brute force.

Refusals come before any HIP call, so fake (never dereferenced) addresses do.
"""
import math
import os
import re

import numpy as np
import pytest

from oracle import steps as O

A = pytest.importorskip("paper_2506_03296_amd")
from paper_2506_03296_amd import steps  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(steps.LIB_PATH):
        from paper_2506_03296_amd import build
        build.build(quiet=True)
    return steps.load_library()


def test_header_symbols_are_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "apex_steps.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(apex_steps_\w+)\s*\(", text))
    assert declared == set(steps.EXPORTED_SYMBOLS)
    assert all(hasattr(lib, n) for n in declared)
    assert int(re.search(r"APEX_STEPS_MAX_NODES (\d+)", text).group(1)) == steps.MAX_NODES


def at(i):
    return FAKE + (i << 36)      # 64 GiB apart


def extend(lib, **kw):
    a = dict(lens=at(0), news=at(1), table=at(2), stride=10, free=at(3), state=at(4), offsets=at(5), totals=at(6),
             slots=at(7), positions=at(8), B=4, T=9, bs=16, nb=100)
    a.update(kw)
    return lib.apex_steps_extend(*a.values(), None)


def release(lib, **kw):
    a = dict(lens=at(0), keeps=at(1), table=at(2), stride=10, free=at(3), state=at(4), B=4, bs=16, nb=100)
    a.update(kw)
    return lib.apex_steps_release(*a.values(), None)


def prompt(lib, **kw):
    a = dict(q=at(0), qs=0, k=at(1), v=at(2), ks=0, offsets=at(3), out=at(4), lse=at(5), B=4, T=50, Hq=32, Hkv=8, d=128,
             scale=0.1)
    a.update(kw)
    return lib.apex_steps_prompt_attention(*a.values(), None)


def tree(lib, **kw):
    a = dict(q=at(0), qs=0, k=at(1), v=at(2), ks=0, offsets=at(3), mask=at(6), kc=at(7), vc=at(8), table=at(9), stride=10,
             lens=at(10), out=at(4), lse=at(5), B=4, T=50, most=16, Hq=32, Hkv=8, d=128, bs=16, nb=100, scale=0.1, ws=None,
             ws_bytes=0)
    a.update(kw)
    return lib.apex_steps_tree_attention(*a.values(), None)


BAD, UNSUP = A.APEX_ERR_INVALID_ARG, A.APEX_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,kw,rc", [
    (extend, dict(B=-1), BAD), (extend, dict(T=-1), BAD), (extend, dict(bs=0), BAD), (extend, dict(nb=-1), BAD),
    (extend, dict(stride=-1), BAD), (extend, dict(nb=1 << 31), UNSUP), (extend, dict(stride=1 << 31), UNSUP),
    (extend, dict(B=(1 << 22) + 1), UNSUP), (extend, dict(lens=None), BAD), (extend, dict(news=None), BAD),
    (extend, dict(table=None), BAD), (extend, dict(free=None), BAD), (extend, dict(state=None), BAD),
    (extend, dict(offsets=None), BAD), (extend, dict(totals=None), BAD), (extend, dict(slots=None), BAD),
    (extend, dict(positions=None), BAD), (extend, dict(slots=at(7) + 4), BAD), (extend, dict(lens=at(0) + 2), BAD),
    (extend, dict(totals=at(0)), BAD), (extend, dict(offsets=at(4) + 4), BAD), (extend, dict(table=at(3) + 396), BAD),
    (extend, dict(positions=at(7) + 64), BAD), (extend, dict(state=at(2) + 156), BAD),
    (release, dict(B=-1), BAD), (release, dict(bs=-16), BAD), (release, dict(nb=-1), BAD), (release, dict(stride=-2), BAD),
    (release, dict(lens=None), BAD), (release, dict(keeps=None), BAD), (release, dict(table=None), BAD),
    (release, dict(free=None), BAD), (release, dict(state=None), BAD), (release, dict(table=at(1)), BAD),
    (release, dict(free=at(2) + 100), BAD), (release, dict(state=at(3) + 396), BAD), (release, dict(keeps=at(1) + 1), BAD),
    (prompt, dict(B=-1), BAD), (prompt, dict(T=-1), BAD), (prompt, dict(Hkv=0), BAD), (prompt, dict(Hq=0), BAD),
    (prompt, dict(Hq=30), BAD), (prompt, dict(d=64), UNSUP), (prompt, dict(scale=math.nan), BAD),
    (prompt, dict(scale=math.inf), BAD), (prompt, dict(qs=4095), BAD), (prompt, dict(qs=4088), BAD),
    (prompt, dict(ks=1028), BAD), (prompt, dict(ks=1 << 31), UNSUP), (prompt, dict(T=1 << 25), UNSUP),
    (prompt, dict(B=(1 << 22) + 1), UNSUP), (prompt, dict(q=None), BAD), (prompt, dict(k=None), BAD),
    (prompt, dict(v=None), BAD), (prompt, dict(offsets=None), BAD), (prompt, dict(out=None), BAD),
    (prompt, dict(q=at(0) + 8), BAD), (prompt, dict(out=at(4) + 8), BAD), (prompt, dict(offsets=at(3) + 2), BAD),
    (prompt, dict(lse=at(5) + 2), BAD), (prompt, dict(out=at(0)), BAD), (prompt, dict(out=at(1) + 1024), BAD),
    (prompt, dict(out=at(3) - 4096), BAD), (prompt, dict(lse=at(4) + 400), BAD), (prompt, dict(lse=at(2)), BAD),
    (tree, dict(B=-1), BAD), (tree, dict(most=0), BAD), (tree, dict(most=65), UNSUP), (tree, dict(d=256), UNSUP),
    (tree, dict(bs=32), UNSUP), (tree, dict(nb=-1), BAD), (tree, dict(stride=-1), BAD), (tree, dict(nb=1 << 27), UNSUP),
    (tree, dict(stride=1 << 27), UNSUP), (tree, dict(stride=(1 << 27) - 1), UNSUP), (tree, dict(scale=-math.inf), BAD),
    (tree, dict(mask=None), BAD), (tree, dict(kc=None), BAD), (tree, dict(vc=None), BAD), (tree, dict(table=None), BAD),
    (tree, dict(lens=None), BAD), (tree, dict(out=None), BAD), (tree, dict(mask=at(6) + 4), BAD),
    (tree, dict(kc=at(7) + 2), BAD), (tree, dict(ws=at(11) + 16, ws_bytes=1 << 40), BAD), (tree, dict(out=at(7) + 4096), BAD),
    (tree, dict(out=at(9)), BAD), (tree, dict(lse=at(10)), BAD), (tree, dict(out=at(6)), BAD),
    (tree, dict(ks=1000), BAD), (tree, dict(Hq=1 << 22, Hkv=1), UNSUP), (tree, dict(Hq=(1 << 16) + 1, Hkv=1), UNSUP),
    (prompt, dict(Hq=1 << 17, T=100), UNSUP), (prompt, dict(B=1 << 22, Hq=1 << 10, Hkv=1 << 10), UNSUP),
])
def test_refusals(lib, call, kw, rc):
    assert call(lib, **kw) == rc
    assert steps.last_error() != ""


def test_no_ops(lib):
    assert prompt(lib, B=0) == prompt(lib, T=0, q=None) == tree(lib, B=0) == tree(lib, T=0, k=None) == A.APEX_OK
    assert release(lib, B=0) == release(lib, nb=0) == release(lib, stride=0) == A.APEX_OK
    assert steps.last_error() == ""
    assert steps.release_workspace() is None


def test_workspace_of_bad_shapes(lib):
    for bad in ((0, 32, 8), (65, 32, 8), (4, 30, 8), (4, 0, 8), (4, 32, 0), (4, -8, -8)):
        assert steps.tree_workspace_bytes(*bad) == 0


def test_binding_wants_gpu_tensors():
    torch = pytest.importorskip("torch")
    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros((4, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        steps.extend(i, i, torch.zeros((2, 3), dtype=torch.int32), i, i, 4)
    with pytest.raises(ValueError, match="GPU"):
        steps.release(i, i, torch.zeros((2, 3), dtype=torch.int32), i, i)
    with pytest.raises(ValueError, match="GPU"):
        steps.prompt_attention(x, x, x, i, 0.1)
    free, state = steps.new_pool(5, "cpu")
    assert free.tolist() == [4, 3, 2, 1, 0] and state.tolist() == [5, 0]
    plan = steps.empty_plan(3, 7, "cpu")
    assert [tuple(t.shape) for t in plan] == [(4,), (3,), (7,), (7,)]
    plan.slot_mapping.fill_(-1)
    for t in plan:
        t.zero_()


# --- the oracle ------------------------------------------------------------------

def test_oracle_extend_by_hand():
    # 4-token blocks: request 0 has 5 tokens (blocks 2, 0) and gets 4, request 1 gets 3 (refused: one block left)
    table = np.array([[2, 0, -1], [-1, -1, -1], [4, -1, -1]], np.int32)
    free = np.array([1, 3, 9, 9, 9], np.int32)
    t, height, offsets, totals, slots, positions = O.extend([5, 0, 2], [4, 5, 1], table, free, 2, 11, 5, 4)
    assert t.tolist() == [[2, 0, 3], [-1, -1, -1], [4, -1, -1]] and height == 1
    assert offsets.tolist() == [0, 4, 9, 10] and totals.tolist() == [9, 0, 3]
    assert slots.tolist() == [1, 2, 3, 12, -1, -1, -1, -1, -1, 18, -1]
    assert positions.tolist() == [5, 6, 7, 8, 0, 0, 0, 0, 0, 2, 0]
    t, free, height = O.release([9, 0, 3], [3, 0, 0], t, free, 1, 5, 4)
    assert t.tolist() == [[2, -1, -1], [-1, -1, -1], [-1, -1, -1]] and free[:4].tolist() == [1, 0, 3, 4] and height == 4


def test_oracle_attention_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 9, 128))
    sees = np.tril(np.ones((9, 9), bool))
    out, lse, mag, most = O.attend(q, k, v, 0.1, sees)
    t = [torch.from_numpy(x)[None, None] for x in (q, k, v)]
    ref = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=True, scale=0.1)[0, 0].numpy()
    assert np.abs(out - ref).max() < 1e-12
    assert abs(lse[0] - 0.1 * q[0] @ k[0]) < 1e-12 and (mag >= np.abs(out) - 1e-12).all() and (most > 0).all()
    none = O.attend(q, np.full_like(k, np.nan), v, 0.1, np.zeros((9, 9), bool))
    assert not none[0].any() and np.isneginf(none[1]).all()


def test_oracle_tree_of_a_chain_is_a_prompt():
    rng = np.random.default_rng(2)
    n, L, Hq, Hkv = 5, 21, 4, 2
    q, k, v = rng.standard_normal((L + n, Hq, 128)), rng.standard_normal((L + n, Hkv, 128)), rng.standard_normal((L + n, Hkv, 128))
    ids = np.array([[3, 1]], np.int32)
    kc, vc = np.zeros((4, Hkv, 16, 128)), np.zeros((4, Hkv, 16, 128))
    for t in range(L):
        kc[ids[0, t // 16], :, t % 16], vc[ids[0, t // 16], :, t % 16] = k[t], v[t]
    chain = [(1 << (i + 1)) - 1 for i in range(n)]
    whole = {h: r for _, h, _, r in O.prompt(q, k, v, [0, L + n], 0.2)}
    for _, h, seen, r in O.tree(q[L:], k[L:], v[L:], [0, n], chain, kc, vc, ids, [L], 64, 0.2):
        assert seen == L + n
        for a, b in zip(r, whole[h]):
            assert np.abs(a - b[L:]).max() < 1e-12

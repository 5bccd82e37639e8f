"""4-bit KV cache without a GPU: symbols, refusals, workspace sizes, and the
oracle's format against a search over all codes.

Refusals come before any HIP call, so fake (never dereferenced) addresses do.
"""
import os
import re

import numpy as np
import pytest

from oracle import kv4 as O

A = pytest.importorskip("paper_2506_03296_amd")
from paper_2506_03296_amd import kv4  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kv4.LIB_PATH):
        from paper_2506_03296_amd import build
        build.build(quiet=True)
    return kv4.load_library()


def test_header_symbols_are_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "apex_kv4.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(apex_kv4_\w+)\s*\(", text))
    assert declared == set(kv4.EXPORTED_SYMBOLS)
    assert all(hasattr(lib, n) for n in declared)
    assert int(re.search(r"APEX_KV4_SLAB_BYTES (\d+)", text).group(1)) == kv4.SLAB_BYTES == O.SLAB


def at(i):
    return FAKE + (i << 36)


# buffers of every call 64 GiB apart: k_new, v_new, cache, slots, ...
def append(lib, **kw):
    a = dict(k=at(0), v=at(1), stride=0, cache=at(2), slots=at(3), tp=at(4), pos=at(5), w=at(6), T=4, Hkv=8, d=128,
             bs=16, nb=100)
    a.update(kw)
    return lib.apex_kv4_append(*a.values(), None)


def gather(lib, **kw):
    a = dict(cache=at(2), slots=at(3), k=at(0), v=at(1), T=4, Hkv=8, d=128, bs=16, nb=100)
    a.update(kw)
    return lib.apex_kv4_gather(*a.values(), None)


def attention(lib, **kw):
    a = dict(q=at(0), cache=at(2), bt=at(3), stride=10, lens=at(4), out=at(5), lse=at(6), B=4, Hq=32, Hkv=8, d=128, bs=16,
             nb=100, scale=0.1, ws=None, ws_bytes=0)
    a.update(kw)
    return lib.apex_kv4_attention(*a.values(), None)


def accumulate(lib, **kw):
    a = dict(q=at(0), cache=at(2), bt=at(3), stride=10, lens=at(4), lse=at(5), w=at(6), B=4, Hq=32, Hkv=8, d=128, bs=16,
             nb=100, scale=0.1)
    a.update(kw)
    return lib.apex_kv4_accumulate_weights(*a.values(), None)


def evict(lib, **kw):
    a = dict(cache=at(2), bt=at(3), stride=10, lens=at(4), w=at(5), pos=at(6), B=4, Hkv=8, d=128, bs=16, nb=100, keep=64,
             sinks=4, recent=16, ws=None, ws_bytes=0)
    a.update(kw)
    return lib.apex_kv4_evict(*a.values(), None)


BAD, UNSUP, MEM = A.APEX_ERR_INVALID_ARG, A.APEX_ERR_UNSUPPORTED, A.APEX_ERR_OUT_OF_MEMORY


@pytest.mark.parametrize("call,kw,rc", [
    (append, dict(T=-1), BAD), (append, dict(Hkv=0), BAD), (append, dict(d=64), UNSUP), (append, dict(bs=32), UNSUP),
    (append, dict(nb=-1), BAD), (append, dict(nb=1 << 31), UNSUP), (append, dict(stride=1000), BAD),
    (append, dict(stride=1028), BAD), (append, dict(k=None), BAD), (append, dict(v=None), BAD),
    (append, dict(cache=None), BAD), (append, dict(slots=None), BAD), (append, dict(k=at(0) + 8), BAD),
    (append, dict(cache=at(2) + 8), BAD), (append, dict(w=at(6) + 4), BAD), (append, dict(slots=at(3) + 4), BAD),
    (append, dict(pos=at(5) + 2), BAD), (append, dict(tp=None), BAD), (append, dict(pos=None), BAD),
    (append, dict(T=1 << 25), UNSUP), (append, dict(k=at(2) + 2176 * 799), BAD), (append, dict(slots=at(2)), BAD),
    (append, dict(pos=at(2)), BAD), (append, dict(w=at(5)), BAD), (append, dict(tp=at(5)), BAD),
    (append, dict(k=at(6)), BAD),
    (gather, dict(T=-1), BAD), (gather, dict(Hkv=-2), BAD), (gather, dict(d=256), UNSUP), (gather, dict(bs=8), UNSUP),
    (gather, dict(k=None), BAD), (gather, dict(v=None), BAD), (gather, dict(cache=None), BAD),
    (gather, dict(slots=None), BAD), (gather, dict(k=at(0) + 4), BAD), (gather, dict(v=at(0) + 4 * 2048 - 16), BAD),
    (gather, dict(k=at(2)), BAD), (gather, dict(v=at(3)), BAD), (gather, dict(T=1 << 25), UNSUP),
    (attention, dict(B=-1), BAD), (attention, dict(Hq=30), BAD), (attention, dict(Hq=0), BAD),
    (attention, dict(Hq=24), UNSUP), (attention, dict(Hq=128), UNSUP), (attention, dict(d=64), UNSUP),
    (attention, dict(bs=32), UNSUP), (attention, dict(stride=-1), BAD), (attention, dict(stride=1 << 27), UNSUP),
    (attention, dict(stride=1 << 26, B=64), UNSUP), (attention, dict(q=None), BAD), (attention, dict(out=None), BAD),
    (attention, dict(bt=None), BAD), (attention, dict(lens=None), BAD), (attention, dict(cache=None), BAD),
    (attention, dict(q=at(0) + 2), BAD), (attention, dict(out=at(5) + 8), BAD), (attention, dict(lse=at(6) + 2), BAD),
    (attention, dict(bt=at(3) + 2), BAD), (attention, dict(out=at(0)), BAD), (attention, dict(out=at(2) + 2176 * 700), BAD),
    (attention, dict(out=at(3) + 144), BAD), (attention, dict(lse=at(5)), BAD), (attention, dict(lse=at(4)), BAD),
    (attention, dict(ws=at(0), ws_bytes=1 << 30), BAD), (attention, dict(out=at(7), ws=at(7), ws_bytes=1 << 30), BAD),
    (accumulate, dict(B=-1), BAD), (accumulate, dict(Hq=20), BAD), (accumulate, dict(d=1), UNSUP),
    (accumulate, dict(lse=None), BAD), (accumulate, dict(w=None), BAD), (accumulate, dict(w=at(6) + 4), BAD),
    (accumulate, dict(lse=at(5) + 1), BAD), (accumulate, dict(w=at(2)), BAD), (accumulate, dict(lse=at(6)), BAD),
    (evict, dict(B=-1), BAD), (evict, dict(Hkv=0), BAD), (evict, dict(d=64), UNSUP), (evict, dict(bs=1), UNSUP),
    (evict, dict(keep=0), BAD), (evict, dict(keep=-5), BAD), (evict, dict(sinks=-1), BAD), (evict, dict(recent=-1), BAD),
    (evict, dict(sinks=40, recent=25), BAD), (evict, dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), BAD),
    (evict, dict(w=None), BAD), (evict, dict(pos=None), BAD), (evict, dict(cache=None), BAD), (evict, dict(lens=None), BAD),
    (evict, dict(w=at(6)), BAD), (evict, dict(pos=at(2)), BAD), (evict, dict(cache=at(4) - 2176), BAD),
    (evict, dict(ws=at(7) + 64, ws_bytes=1 << 30), BAD), (evict, dict(ws=at(7), ws_bytes=100), MEM),
    (evict, dict(ws=at(2), ws_bytes=1 << 30), BAD), (evict, dict(B=1 << 19, stride=1), UNSUP),
])
def test_refusals(lib, call, kw, rc):
    assert call(lib, **kw) == rc
    assert kv4.last_error() != ""


def test_an_eviction_of_too_wide_a_table_is_refused(lib):
    assert evict(lib, B=1, Hkv=1, stride=1 << 24) == UNSUP and "2^24" in kv4.last_error()
    assert kv4.evict_workspace_bytes(1, 1, 1 << 24) == 0 and kv4.evict_workspace_bytes(1, 1, (1 << 24) - 1) > 0
    # a token's bit, a pair's count
    assert kv4.evict_workspace_bytes(65, 1, 2049) == 512 + -(-65 * 513 * 8 // 256) * 256
    # where pairs may be spread, also two counts of 2048 digits for every chunk
    assert kv4.evict_workspace_bytes(64, 1, 2049) >= 64 * 5 * 2 * 2048 * 2


def test_nothing_to_do(lib):
    assert append(lib, T=0, k=None, v=None, cache=None, slots=None) == A.APEX_OK
    assert gather(lib, T=0, k=None, v=None, cache=None, slots=None) == A.APEX_OK
    assert attention(lib, B=0, q=None, out=None) == A.APEX_OK
    assert accumulate(lib, B=0, q=None, w=None) == A.APEX_OK
    assert evict(lib, B=0, cache=None) == A.APEX_OK
    assert append(lib, nb=0) == A.APEX_OK
    assert accumulate(lib, nb=0) == A.APEX_OK
    assert evict(lib, nb=0) == A.APEX_OK
    assert evict(lib, stride=0, bt=None) == A.APEX_OK
    # no request can be longer than `keep`
    assert evict(lib, keep=160, ws=at(7), ws_bytes=1 << 30) == A.APEX_OK
    assert kv4.last_error() == ""


def test_workspace_sizes(lib):
    assert kv4.evict_workspace_bytes(0, 8, 10) == 0
    # a count per pair and a bit per slot
    assert kv4.evict_workspace_bytes(4, 8, 10) == 256 + 32 * 3 * 8
    assert kv4.evict_workspace_bytes(4, 8, -1) == 0 and kv4.evict_workspace_bytes(4, 0, 1) == 0


# ---------------------------------------------------------------------------
# the oracle's format
# ---------------------------------------------------------------------------

def test_row_layout_covers_the_slab_once():
    seen = np.concatenate([np.concatenate(O.row_offsets(t)) for t in range(16)])
    assert np.array_equal(np.sort(seen), np.arange(O.SLAB))


def test_quantise_is_the_nearest_code_of_the_least_scale():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((64, 128)) * 10.0 ** rng.integers(-6, 4, (64, 1))).astype(np.float16)
    x[0] = 0
    x[1, :32] = 0
    x[2, 5] = 65504
    x[3] = np.float16(2.0 ** -24) * rng.integers(-3, 4, 128)
    code, scale = O.quantise(x)
    v = O.values(code, scale)
    y = x.astype(np.float64)
    s = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32, -1)
    grid = np.concatenate([O.MAGNITUDES, -O.MAGNITUDES])
    assert np.array_equal(np.abs(v - y), np.abs(grid[:, None, None] * s - y).min(0))
    m = np.abs(y).reshape(64, 4, 32).max(-1)
    e = 2.0 ** (scale.astype(np.float64) - 127)
    assert np.all(m <= 6 * e) and np.all((m > 3 * e) | (m == 0)) and np.all(scale[m == 0] == 127)


@pytest.mark.parametrize("v,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (0.2502, 1),
                                    (4.99, 6), (5.01, 7), (6.0, 7), (-0.0, 8), (-0.1, 8), (-3.5, 14)])
def test_ties_go_to_the_even_code(v, code):
    x = np.zeros(128, np.float16)
    x[0], x[1] = v, 6.0
    c, s = O.quantise(x)
    assert s[0] == 127 and c[0] == code


def test_a_group_with_a_non_finite_value_is_nan():
    x = np.ones((2, 128), np.float16)
    x[0, 40], x[1, 100] = np.inf, np.nan
    c, s = O.quantise(x)
    # ones: 6 x 2^-3 = 0.75 < 1 <= 6 x 2^-2 = 1.5, so the byte is 125
    assert s.tolist() == [[125, 255, 125, 125], [125, 125, 125, 255]] and not c[s.repeat(32, -1) == 255].any()
    assert np.isnan(O.values(c, s)).sum() == 64

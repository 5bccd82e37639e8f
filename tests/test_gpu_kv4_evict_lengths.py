"""Evictions of pairs of 2049 to 32768 tokens: every number of keys that a thread of
the larger work groups keeps in its registers, moves within the selecting work group
and in the second launch.  Bit for bit against the oracle."""
import functools

import pytest

from oracle import kv4 as O
from test_gpu_kv4 import evict_case, kv4, run_evict, same, torch  # noqa: F401  (two are fixtures)

pytestmark = pytest.mark.gpu


@functools.lru_cache(maxsize=1)
def pairs(kind):
    # 2048, 8192, 16384 and 32768 tokens are where a thread takes more
    return evict_case([32768, 2049, 20000, 8192, 16385, 8193, 16384, 2048, 31000], 1, seed=37, kind=kind)


@pytest.mark.parametrize("keep,sinks,recent", [(1, 0, 0), (2040, 4, 500), (4096, 4, 1024), (8190, 0, 4096), (16384, 16384, 0),
                                               (32760, 4, 16000)])
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "wild"])
def test_evict(torch, kv4, kind, keep, sinks, recent):  # noqa: F811
    cache, table, lens, w, pos = pairs(kind)
    cache, w, pos = cache.copy(), w.copy(), pos.copy()
    got = run_evict(torch, kv4, cache, table, lens, w, pos, keep, sinks, recent)
    O.evict(cache, table, lens, w, pos, keep, sinks, recent)
    assert same(got, (cache, w, pos))

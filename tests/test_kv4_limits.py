"""The 4-bit KV cache's limits of batches: each refusal says which one it is."""
import pytest

A = pytest.importorskip("paper_2506_03296_amd")
from paper_2506_03296_amd import kv4  # noqa: E402
from test_kv4_abi import UNSUP, accumulate, attention, evict, lib  # noqa: E402, F401  (lib is a fixture)

WIDEST = (1 << 27) - 2   # a row's tokens stay below 2^31


@pytest.mark.parametrize("call,one", [(attention, dict(B=1, Hq=1, Hkv=1)), (accumulate, dict(B=1, Hq=1, Hkv=1)),
                                      (evict, dict(B=1, Hkv=1))])
def test_table_rows_of_2_31_tokens(lib, call, one):  # noqa: F811
    for stride in (WIDEST + 1, 1 << 27, 1 << 40):
        assert call(lib, stride=stride, **one) == UNSUP
        assert kv4.last_error() == f"block_table_stride {stride} reaches 2^27 - 1"


def test_the_widest_row_passes_this_check(lib):  # noqa: F811
    # refused for its pointers, which are looked at next
    assert attention(lib, stride=WIDEST, B=1, Hq=1, Hkv=1, q=None) == A.APEX_ERR_INVALID_ARG
    assert "NULL" in kv4.last_error()


def test_pairs_times_row_width(lib):  # noqa: F811
    for B, Hkv, stride in ((2, 8, WIDEST), (1 << 20, 1, 1984), (1 << 30, 1, 0), (2 ** 31 - 1, 2 ** 31 - 1, 0)):
        assert attention(lib, B=B, Hq=Hkv, Hkv=Hkv, stride=stride) == UNSUP
        assert kv4.last_error() == "B * Hkv * (block_table_stride + 64) exceeds 2^31 - 1"
    assert attention(lib, B=1 << 20, Hq=1, Hkv=1, stride=1983, q=None) == A.APEX_ERR_INVALID_ARG

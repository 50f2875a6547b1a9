"""Argument checks of attention, rotary positions and dropout at the limits that are documented (no GPU)."""
import ctypes as C

import pytest

from test_attention import ATT_B, ATT_F, ROT, heads  # noqa: F401
from test_operators import BF16, INVALID, OK, OUT_OF_MEMORY, P, TOO_LARGE, lib  # noqa: F401

MOST = (1 << 30) - 1024   # rows x heads, key rows x kv heads


@pytest.mark.parametrize("rows,keys,sequences,heads,kv_heads,status", [
    (1, 1 << 29, 1, 128, 1, OK),              # many kept keys under a large group
    (1, MOST, 1, 65536, 1, OK),
    (MOST, MOST, 65536, 1, 1, OK),
    (MOST // 65536, MOST // 16384, 65536, 65536, 16384, OK),
    (MOST // 65536, MOST // 32768, 65536, 65536, 32768, TOO_LARGE),   # 2^31 tiles, one a sequence and head at least
    (MOST + 1, 1, 1, 1, 1, TOO_LARGE),
    (1, MOST + 1, 1, 1, 1, TOO_LARGE),
    (1, MOST // 2 + 1, 1, 2, 2, TOO_LARGE),
])
@pytest.mark.parametrize("backward", [0, 1])
def test_sizes_up_to_the_documented_ones(lib, rows, keys, sequences, heads, kv_heads, status, backward):  # noqa: F811
    need = C.c_uint64()
    assert lib.pase_attention_workspace(BF16, rows, keys, sequences, heads, kv_heads, 2, backward, C.byref(need)) == status

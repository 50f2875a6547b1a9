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


@pytest.mark.parametrize("rows,heads,dim,ld,hs", [(4, 2, 8, 16, 8), (4, 2, 8, 40, 12), (4, 3, 8, 8, 40), (5, 1, 8, 11, 0), (1, 4, 6, 0, 9), (1, 1, 8, 0, 0),
                                                  (3, 4, 2, 50, 5), (6, 2, 8, 16, 120)])
def test_rotation_onto_a_part_of_x(lib, rows, heads, dim, ld, hs):  # noqa: F811
    """Refused where x and y have an element in common (here the next refusal, of the positions, stands for what passes)."""
    x = {r * ld + h * hs + e for r in range(rows) for h in range(heads) for e in range(dim)}
    assert len(x) == rows * heads * dim
    at = 1 << 20
    for d in range(-max(x) - 3, max(x) + 4):
        args = {**ROT, "rows": rows, "heads": heads, "dim": dim, "turned": 2, "x": at, "ldx": ld, "hsx": hs, "y": at + 2 * d, "ldy": ld, "hsy": hs,
                "positions": None}
        assert lib.pase_rotary(*args.values()) == INVALID
        shared = d and not x.isdisjoint({e + d for e in x})
        assert lib.pase_operator_error() == (b"y overlaps x in part" if shared else b"positions is null"), d


def apart(args):
    """The same call with arrays of its own for every pointer to P."""
    at, out = 1 << 20, {}
    for name, value in args.items():
        out[name] = value
        if value == P:
            out[name], at = at, at + (1 << 16)
    return out


@pytest.mark.parametrize("name,good,pairs", [
    ("pase_attention_forward", ATT_F, [("o", "q"), ("o", "k"), ("o", "v"), ("lse", "q"), ("lse", "k"), ("lse", "v"), ("lse", "o")]),
    ("pase_attention_backward", ATT_B, [(o, i) for o in ("dq", "dk", "dv") for i in ("do", "q", "k", "v", "o", "lse")] + [("dk", "dq"), ("dv", "dq"), ("dv", "dk")]),
])
def test_outputs_that_are_inputs(lib, name, good, pairs):  # noqa: F811
    good = apart(good)
    for output, other in pairs:
        assert getattr(lib, name)(*{**good, output: good[other]}.values()) == INVALID
        assert lib.pase_operator_error() in (b"an output is an input", b"two outputs are one"), (output, other)

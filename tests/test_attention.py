"""Argument checks of attention, rotary positions and dropout (no GPU): every refusal is made on
the host before anything is enqueued, so the pointers here are never followed."""
import ctypes as C

import pytest
import torch

from test_operators import BF16, FP16, FP32, INVALID, OK, OUT_OF_MEMORY, P, TOO_LARGE, lib  # noqa: F401

SIZES = dict(dtype=BF16, rows=4, key_rows=6, sequences=2, heads=4, kv_heads=2, dim=8)


def heads(name, n, at=P):
    return {name: at, f"ld{name}": n * 8, f"hs{name}": 8}


OFFSETS = dict(q_offsets=P, k_offsets=P, k_lengths=P, off64=0, causal=1, scale=0.5)
ATT_F = dict(**SIZES, **heads("q", 4), **heads("k", 2), **heads("v", 2), **OFFSETS, **heads("o", 4), lse=P, ws=P, ws_bytes=1 << 30, stream=None)
ATT_B = dict(**SIZES, **heads("do", 4), **heads("q", 4), **heads("k", 2), **heads("v", 2), **heads("o", 4), lse=P, **OFFSETS,
             **heads("dq", 4), **heads("dk", 2), **heads("dv", 2), ws=P, ws_bytes=1 << 30, stream=None)
ROT = dict(dtype=BF16, rows=4, heads=2, dim=8, turned=6, interleaved=0, inverse=0, **heads("x", 2), positions=P, pos64=1,
           frequencies=P, magnitude=1.0, **heads("y", 2, 2 * P), stream=None)
DROP = dict(dtype=BF16, rows=4, width=8, x=P, ldx=8, residual=P, ldr=8, p=0.1, seed=P, y=2 * P, ldy=8, stream=None)

SHARED = [dict(dtype=FP32), dict(dtype=7), dict(sequences=0), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(dim=0), dict(q=None),
          dict(q=P + 1), dict(ldq=7), dict(hsq=7), dict(ldq=31), dict(ldq=8, hsq=8), dict(ldq=(1 << 22) + 1), dict(hsq=1 << 41),
          dict(k=None), dict(ldk=15), dict(hsk=47, ldk=8), dict(v=None), dict(hsv=4), dict(q_offsets=None), dict(k_offsets=None),
          dict(q_offsets=P + 2), dict(k_offsets=P + 4, off64=1), dict(off64=2), dict(k_lengths=P + 1), dict(causal=2), dict(scale=0.0),
          dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e-40), dict(lse=None), dict(lse=P + 2), dict(o=None), dict(ldo=3)]
LARGE = [dict(dim=129), dict(sequences=65537), dict(heads=131072, kv_heads=131072), dict(rows=1 << 30), dict(key_rows=1 << 30),
         dict(rows=1 << 30, heads=1, kv_heads=1), dict(key_rows=1 << 30, heads=1, kv_heads=1), dict(sequences=65536, heads=65536, kv_heads=65536)]
REFUSALS = [
    ("pase_attention_forward", ATT_F, INVALID, SHARED + [dict(rows=1, key_rows=5000, heads=2, kv_heads=1, ws=None), dict(rows=1, key_rows=5000, ws=P + 8)]),
    ("pase_attention_forward", ATT_F, TOO_LARGE, LARGE),
    ("pase_attention_forward", ATT_F, OUT_OF_MEMORY, [dict(rows=1, key_rows=5000, ws_bytes=64)]),
    ("pase_attention_backward", ATT_B, INVALID, SHARED + [
        dict(do=None), dict(lddo=4), dict(dq=None), dict(hsdq=4), dict(dk=None), dict(lddk=4), dict(dv=P + 1), dict(hsdv=0), dict(ws=None), dict(ws=P + 4)]),
    ("pase_attention_backward", ATT_B, TOO_LARGE, LARGE),
    ("pase_attention_backward", ATT_B, OUT_OF_MEMORY, [dict(ws_bytes=0), dict(ws_bytes=127)]),
    ("pase_rotary", ROT, INVALID, [
        dict(dtype=3), dict(heads=0), dict(dim=0), dict(turned=0), dict(turned=5), dict(turned=10), dict(interleaved=2), dict(inverse=-1),
        dict(x=None), dict(x=P + 1), dict(ldx=15), dict(hsx=7), dict(y=None), dict(y=P, ldy=20), dict(positions=None), dict(positions=P + 4),
        dict(pos64=3), dict(frequencies=None), dict(frequencies=P + 4), dict(dtype=FP32, x=P + 2)]),
    ("pase_rotary", ROT, TOO_LARGE, [dict(turned=1026, dim=1026), dict(heads=1 << 20), dict(rows=1 << 41)]),
    ("pase_dropout", DROP, INVALID, [
        dict(dtype=3), dict(width=0), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(x=None), dict(x=P + 1), dict(ldx=7),
        dict(residual=P + 1), dict(ldr=7), dict(seed=None), dict(seed=P + 4), dict(y=None), dict(ldy=7), dict(y=P, ldy=9),
        dict(residual=2 * P, ldr=9)]),
    ("pase_dropout", DROP, TOO_LARGE, [dict(width=(1 << 32) + 1), dict(rows=1 << 41), dict(rows=1 << 38, width=64)]),
]


@pytest.mark.parametrize("name,good,status,change", [
    pytest.param(n, g, s, c, id=f"{n[5:]}-{'-'.join(f'{k}={v}' for k, v in c.items())}")
    for n, g, s, changes in REFUSALS for c in changes])
def test_refusals(lib, name, good, status, change):  # noqa: F811
    assert getattr(lib, name)(*{**good, **change}.values()) == status
    assert lib.pase_operator_error()


@pytest.mark.parametrize("name,good", [("pase_attention_forward", ATT_F), ("pase_rotary", ROT), ("pase_dropout", DROP),
                                       ("pase_attention_backward", {**ATT_B, "key_rows": 0})])
def test_no_rows_is_nothing_to_do(lib, name, good):  # noqa: F811
    none = {k: (None if v in (P, 2 * P) and k != "ws_bytes" else v) for k, v in good.items()}
    assert getattr(lib, name)(*{**none, "rows": 0}.values()) == OK


def test_workspace_sizes(lib):  # noqa: F811
    need = C.c_uint64(12345)

    def ask(rows, keys, n, heads, kv, dim, backward=0):
        assert lib.pase_attention_workspace(BF16, rows, keys, n, heads, kv, dim, backward, C.byref(need)) == OK
        return need.value
    assert ask(16384, 16384, 64, 16, 16, 64) == 0                 # tiles enough
    assert ask(16384, 16384, 64, 16, 16, 64, 1) == 16384 * 16 * 8
    assert ask(1, 100, 1, 4, 4, 64) == 0                          # nothing to share out
    # shares: a log-sum-exp and dim elements for each row and head
    one = ask(1, 65536, 1, 16, 2, 128)
    assert one > 0 and one % (16 * 129 * 4) == 0 and one // (16 * 129 * 4) <= 256
    odd = ask(3, 65536, 1, 5, 5, 22)
    assert odd > 0 and odd % (16 * 25 * 4) == 0
    assert lib.pase_attention_workspace(BF16, 1, 1, 1, 1, 1, 8, 0, None) == INVALID
    assert lib.pase_attention_workspace(BF16, 1, 1, 1, 1, 1, 8, 2, C.byref(need)) == INVALID
    assert lib.pase_attention_workspace(FP32, 1, 1, 1, 1, 1, 8, 0, C.byref(need)) == INVALID


def test_strides_of_either_order_are_taken(lib):  # noqa: F811
    """Rows inside heads and heads inside rows pass the checks (and reach the launch, which is not there without a
    GPU; here the next refusal, of the output's alignment, stands for that)."""
    for layout in (dict(ldq=32, hsq=8), dict(ldq=8, hsq=32), dict(ldq=40, hsq=9), dict(ldq=100, hsq=8)):
        assert lib.pase_attention_forward(*{**ATT_F, **layout, "o": P + 1}.values()) == INVALID
        assert lib.pase_operator_error() == b"out is not aligned to its element", layout


def test_host_tensors_are_refused():
    from paper_2407_04001_amd import PaseError, ops
    x, o = torch.zeros(4, 2, 8, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    pos, f, seed = torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.float64), torch.zeros(2, dtype=torch.int64)
    lse = torch.zeros(2, 4)
    for call in (lambda: ops.attention_forward(x, x, x, o, o), lambda: ops.attention(q=x, k=x, v=x, q_offsets=o, k_offsets=o),
                 lambda: ops.attention_backward(x, x, x, x, x, lse, o, o), lambda: ops.rotary_forward(x, pos, f),
                 lambda: ops.rotary_backward(dy=x, positions=pos, frequencies=f), lambda: ops.rotary(x, pos, f),
                 lambda: ops.dropout_forward(x[:, 0], 0.1, seed), lambda: ops.dropout_backward(dy=x[:, 0], p=0.1, seed=seed),
                 lambda: ops.dropout(x[:, 0], 0.1, seed)):
        with pytest.raises(PaseError) as e:
            call()
        assert e.value.status == INVALID


def philox(counter, key):
    """Philox 4x32-10, round by round (Salmon, Moraes, Dror, Shaw 2011)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xffffffff, a >> 32 ^ c[3] ^ k[1], a & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def test_the_generators_published_values():
    """The known answers that were published with the generator."""
    assert philox([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox([0xffffffff] * 4, [0xffffffff] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert philox([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]) == \
        [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_argument_checks_under_sanitizers():
    """This file's tests on the host-only build, under AddressSanitizer and UBSan."""
    import os
    import shutil
    import subprocess
    import sys
    if "libasan" in os.environ.get("LD_PRELOAD", ""):
        pytest.skip("this is that run")
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if not cxx:
        pytest.skip("no host C++ compiler")
    from paper_2407_04001_amd import build
    san = build.build_host_sanitized()
    asan = subprocess.run([cxx, "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-x", "-p", "no:cacheprovider", "--pase-lib", san],
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and " passed" in r.stdout, (r.stdout + r.stderr)[-4000:]

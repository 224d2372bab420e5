"""uc_linear_attend's outputs share memory with nothing else (CPU): what a launch
would race on is turned down, rows that merely interleave in one buffer are not.

Nothing can be launched here, so a call that passes every check ends in the
CUDA error of a machine without a GPU; the tensor maps are asked for first where
there are more than a few tokens, and end the same way."""
import ctypes as C
import itertools
import random

import pytest
import torch

from paper_2609_32831_gb300 import _lib

LIB = _lib.lib
A = 1 << 30
STATE = 9 << 40

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls over made-up addresses: no GPU")


def _rows(ptr, sb, sh, st):
    return _lib.UcRows(ptr, sb, sh, st)


def _call(B, hq, hkv, T, q, k, v, out, s_in=None, s_out=STATE):
    r = [C.byref(x) for x in (q, k, v, out)]
    return LIB().uc_linear_attend(r[0], r[1], r[2], B, hq, hkv, T, None, (C.c_float * hkv)(*[-0.1] * hkv), s_in, s_out,
                                  r[3], 8 << 40, 1 << 30, None)


def _meets(a, sa, b, sb, same=False):
    """By enumeration: rows of 256 bytes."""
    at = lambda r, s: [(i, r.ptr + 2 * (i[0] * r.stride_b + i[1] * r.stride_h + i[2] * r.stride_t))
                       for i in itertools.product(*map(range, s))]
    return any(abs(x - y) < 256 and not (same and i == j) for i, x in at(a, sa) for j, y in at(b, sb))


def _apart(B, hq, hkv, T, off=40):
    far = lambda n, h: _rows(n << off, h * T * 128, T * 128, 128)
    return far(1, hq), far(2, hkv), far(3, hkv)


@pytest.mark.parametrize("T", [3, 20])
def test_interleaved_rows_pass(T):
    B, hq, hkv = 2, 4, 2
    w = 2 * hq + 2 * hkv
    wide = [_rows(A + 256 * at, T * w * 128, 128, w * 128) for at in (0, hq, hq + hkv, hq + 2 * hkv)]
    assert _call(B, hq, hkv, T, *wide) == _lib.UC_ERR_CUDA
    # a block per sequence, tokens first in out's part
    blocks = [_rows(A + 256 * T * at, T * w * 128, T * 128, 128) for at in (0, hq, hq + hkv)]
    out = _rows(A + 256 * T * (hq + 2 * hkv), T * w * 128, 128, hq * 128)
    assert _call(B, hq, hkv, T, *blocks, out) == _lib.UC_ERR_CUDA


@pytest.mark.parametrize("T", [3, 20])
def test_shared_rows_are_refused(T):
    B, hq, hkv = 2, 4, 2
    q, k, v = _apart(B, hq, hkv, T)
    for r, h in ((q, hq), (k, hkv), (v, hkv)):
        for shift in (256, 16, -16):          # one row on, a few channels on or back
            out = _rows(r.ptr + shift, hq * T * 128, T * 128, 128)
            assert _call(B, hq, hkv, T, q, k, v, out) == _lib.UC_ERR_ARG
    assert b"uc_linear_attend" in LIB().uc_last_error()


@pytest.mark.parametrize("sb,sh,st", [(4096, 128, 128), (128, 4096, 128), (65536, 1024, 1032), (65536, 136, 128),
                                      (384, 128, 256)])
def test_out_over_itself_is_refused(sb, sh, st):
    B, hq, hkv, T = 2, 4, 2, 10
    out = _rows(4 << 40, sb, sh, st)
    assert _meets(out, (B, hq, T), out, (B, hq, T), same=True)
    assert _call(B, hq, hkv, T, *_apart(B, hq, hkv, T), out) == _lib.UC_ERR_SHAPE


def test_states_over_rows_are_refused():
    B, hq, hkv, T = 2, 4, 2, 3
    q, k, v = _apart(B, hq, hkv, T)
    out = _rows(4 << 40, hq * T * 128, T * 128, 128)
    for r in (q, k, v, out):
        assert _call(B, hq, hkv, T, q, k, v, out, s_out=r.ptr + 256) == _lib.UC_ERR_ARG
    assert _call(B, hq, hkv, T, q, k, v, out, s_in=out.ptr + 512) == _lib.UC_ERR_ARG
    assert _call(B, hq, hkv, T, q, k, v, out, s_in=q.ptr) == _lib.UC_ERR_CUDA    # (both only read)
    # one row right before the states, the next sequence's right behind them, or 16 bytes into them
    q, k, v = _apart(B, 1, 1, 1)
    size = B * 65536
    for gap, want in ((size + 256, _lib.UC_ERR_CUDA), (size + 240, _lib.UC_ERR_ARG)):
        assert _call(B, 1, 1, 1, q, k, v, _rows(STATE - 256, gap // 2, 0, 0)) == want


def test_extents_beyond_any_memory_are_refused():
    B, hq, hkv, T = 2, 4, 2, 1 << 28
    q, k, v = _apart(B, hq, hkv, T, off=50)
    out = _rows(4 << 50, 128, 128, 1 << 37)
    assert _call(B, hq, hkv, T, q, k, v, out) == _lib.UC_ERR_SHAPE


def test_against_enumeration():
    rng = random.Random(0)
    seen = set()
    for _ in range(3000):
        B, hkv, T = rng.randint(1, 3), rng.randint(1, 2), rng.randint(1, 5)
        hq = hkv * rng.randint(1, 2)
        stride = lambda: 128 + 8 * rng.randint(0, rng.choice([2, 40, 400]))
        q, out = (_rows(A + 16 * rng.randint(0, 3000), *[stride() for _ in range(3)]) for _ in range(2))
        if rng.random() < 0.5:
            out.stride_b, out.stride_h, out.stride_t = q.stride_b, q.stride_h, q.stride_t
        _, k, v = _apart(B, hq, hkv, T)
        s = (B, hq, T)
        want = _lib.UC_ERR_CUDA
        if q.ptr == out.ptr:
            want = _lib.UC_ERR_ARG
        elif _meets(out, s, out, s, same=True):
            want = _lib.UC_ERR_SHAPE
        elif _meets(out, s, q, s):
            want = _lib.UC_ERR_ARG
        assert _call(B, hq, hkv, T, q, k, v, out) == want, (s, q.ptr - A, out.ptr - A)
        seen.add(want)
    assert len(seen) == 3

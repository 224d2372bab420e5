"""Rotary positions against fp64: layouts of pairs, parts of the head, types,
strides, far positions, in place."""
import numpy as np
import pytest
import torch

from oracle import rotary as orot

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")

DEV = "cuda"
# half a step of each type, relative to the value
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half a step of the subnormal numbers: fp16's steps below 2^-14 are 2^-24 whatever the value (the others' are below 2^-132)
LEAST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def rows(g, B, H, T, layout, dtype=torch.bfloat16):
    if layout == "bthd":
        return torch.randn((B, T, H, 128), generator=g, device=DEV).to(dtype).transpose(1, 2)
    if layout == "cut":      # every second head of a wider tensor, behind an offset
        return torch.randn((B, 2 * H, T + 3, 128), generator=g, device=DEV).to(dtype)[:, ::2, 2:2 + T]
    return torch.randn((B, H, T, 128), generator=g, device=DEV).to(dtype)


def freqs_of(pairs, base=10000.0):
    return [base ** (-i / pairs) for i in range(pairs)]


def bound(x, pairs, interleaved, scale, dtype, want):
    """In fp32 a sine and a cosine are within 2^-22 (two ulp and the angle's own rounding), their scale, the
    products and their sum within 2^-23 more: of |a| + |b| times the scale. Then half a step of the type."""
    a = np.abs(x)
    size = a.copy()
    if interleaved:
        both = a[..., 0:2 * pairs:2] + a[..., 1:2 * pairs:2]
        size[..., 0:2 * pairs:2] = size[..., 1:2 * pairs:2] = both
    else:
        both = a[..., :pairs] + a[..., pairs:2 * pairs]
        size[..., :pairs] = size[..., pairs:2 * pairs] = both
    exact = np.broadcast_to(np.arange(128) >= 2 * pairs, a.shape)
    err = size * abs(scale) * (2.0 ** -22 + 2.0 ** -23)
    return np.where(exact, 0.0, err + HALF[dtype] * (np.abs(want) + err) + LEAST[dtype] + 1e-9 * abs(scale) * size)


CASES = [(B, hq, hkv, T, pairs, inter, dtype, layout, mode, start)
         for B, hq, hkv, T, layout, mode, start in ((1, 28, 4, 1, "bhtd", "first", 0), (3, 5, 1, 37, "bthd", "each", 1000000),
                                                   (2, 4, 4, 130, "cut", "first", 2 ** 31 - 200))
         for pairs in (64, 32, 24, 20, 17, 1, 63)
         for inter in (False, True)
         for dtype in (torch.bfloat16, torch.float16, torch.float32)]


@pytest.mark.parametrize("B,hq,hkv,T,pairs,inter,dtype,layout,mode,start", CASES)
def test_against_fp64(B, hq, hkv, T, pairs, inter, dtype, layout, mode, start):
    g = torch.Generator(device=DEV).manual_seed(pairs + 100 * T)
    q, k = rows(g, B, hq, T, layout, dtype), rows(g, B, hkv, T, layout, dtype)
    f, scale = freqs_of(pairs), 1.25
    first = start + torch.arange(B, device=DEV)[:, None] * 7
    pos = first if mode == "first" else first + (torch.arange(T, device=DEV) * 31) % 1000
    table = uc.Rotary(f, interleaved=inter, scale=scale)
    keep = q.clone(), k.clone()
    out = uc.rotary(table, pos.int(), q, k)
    p = pos.cpu().numpy() + (np.arange(T) if mode == "first" else 0)
    for x, y in zip((q, k), out):
        assert y.dtype == dtype and y.shape == x.shape
        xs = x.double().cpu().numpy()
        want = orot.rotary(xs, p, f, inter, scale)
        err = np.abs(y.double().cpu().numpy() - want)
        far = err - bound(xs, pairs, inter, scale, dtype, want)
        assert far.max() <= 0, (float(far.max()), float(np.abs(want).flat[far.argmax()]))
    assert torch.equal(keep[0], q) and torch.equal(keep[1], k)
    # in place, and alone
    alone, none = uc.rotary(table, pos.int(), q)
    assert none is None and torch.equal(alone, out[0])
    got = uc.rotary(table, pos.int(), q, k, out_q=q, out_k=k)
    assert got[0] is q and torch.equal(q, out[0]) and torch.equal(k, out[1])


def test_layout_is_kept():
    g = torch.Generator(device=DEV).manual_seed(1)
    q = rows(g, 2, 3, 5, "bthd")
    y, _ = uc.rotary(uc.Rotary([1.0]), torch.zeros((2, 5), dtype=torch.int32, device=DEV), q)
    assert y.stride() == q.stride()


def test_a_rotation_at_the_negative_position_turns_back():
    """The transpose of the map, what a gradient goes through."""
    g = torch.Generator(device=DEV).manual_seed(2)
    q = rows(g, 2, 3, 50, "bhtd", torch.float32)
    table = uc.Rotary(freqs_of(64))
    p = torch.randint(0, 1 << 20, (2, 50), generator=g, device=DEV, dtype=torch.int32)
    there, _ = uc.rotary(table, p, q)
    back, _ = uc.rotary(table, -p, there)
    # twice the bound of one rotation, of |a| + |b| <= sqrt(2) of the pair's length
    assert float((back - q).abs().max()) <= 4 * (2.0 ** -22 + 2.0 ** -23 + 2.0 ** -24) * float(q.abs().max()) * 2


def test_nonfinite_values_stay_in_their_pair():
    x = torch.ones((1, 1, 1, 128), device=DEV)
    x[..., 3] = float("nan")
    x[..., 127] = float("inf")
    at = torch.full((1, 1), 9, dtype=torch.int32, device=DEV)
    for inter, pair in ((False, 3 + 20), (True, 2)):
        y, _ = uc.rotary(uc.Rotary(freqs_of(20), interleaved=inter), at, x)
        bad = (~torch.isfinite(y)).nonzero()[:, 3].tolist()
        assert bad == sorted([3, pair, 127]) and float(y[..., 127]) == float("inf")

"""States of uc_linear_attend at the accuracy that their arithmetic has.

Per element, in units of the sum of the terms' magnitudes (the oracle's size):

* up to 8 tokens: each step rounds a product and two fused sums, of which decay
  forgets none: (3 T + 1) * 2^-24;
* one slice of 16 tokens on the tensor cores: the decayed values enter whole, as
  three bf16 parts (two would be up to 2^-16 off), so what is lost are the
  roundings of weight, product and final sum, three additions to the accumulator
  (a cut below one unit in the last place, 2^-23), and 16 products aligned to the
  largest of them (2^-25 each): (3 + 3 + 4) * 2^-23;
* more: 8 slices of three parts per chunk, each addition cut, and a few fp32
  roundings per chunk that decay has not forgotten: 24 * 2^-23 + 8 * 2^-24."""
import numpy as np
import pytest
import torch

from oracle import linear as olinear
from tests.test_gpu_linear import _inputs, _np

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")


def _tol(T):
    if T <= 8:
        return (3 * T + 1) * 2.0 ** -24
    return 10 * 2.0 ** -23 if T <= 16 else 24 * 2.0 ** -23 + 8 * 2.0 ** -24


@pytest.mark.parametrize("T", [1, 3, 8, 9, 12, 16, 17, 100, 128, 129, 300, 515])
@pytest.mark.parametrize("hq,hkv,B", [(28, 4, 1), (2, 2, 3), (9, 3, 2)])
@pytest.mark.parametrize("state", [False, True])
def test_states(hq, hkv, B, T, state):
    ld = np.linspace(-0.3, -0.0003, hkv).tolist()
    q, k, v, s = _inputs(31 * T + hq, B, hq, hkv, T, state=state)
    lengths = [max(1, T - b) for b in range(B)]
    _, new = uc.linear_attend(q, k, v, ld, state=s, lengths=lengths)
    # log decays as the library holds them
    ld = [float(np.float32(x)) for x in ld]
    _, ref, _, size = olinear.linear_attend(_np(q), _np(k), _np(v), ld, _np(s), lengths)
    err = np.abs(_np(new) - ref) / size
    assert err.max() <= _tol(T), (err.max(), _tol(T))

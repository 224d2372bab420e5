"""uc_beam_select's outputs share memory with nothing that its join still reads
or writes (CPU). Scores in place, where each request has as many results as
beams, are allowed: a call that passes every check ends in the CUDA error of a
machine without a GPU."""
import pytest
import torch

from paper_2609_32831_gb300 import _lib

LIB = _lib.lib
A = 1 << 30

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid calls over made-up addresses: no GPU")


def _call(n=4, scores=2 * A, fin=3 * A, os=4 * A, op=5 * A, ot=6 * A, of=7 * A, B=3, K=4):
    return LIB().uc_beam_select(A, _lib.FP32, 4000, 1000, B, K, 1000, scores, fin, 1, n, os, op, ot, of, 8 * A, 1 << 24, None)


def test_apart():
    assert _call() == _call(of=None) == _call(fin=None) == _lib.UC_ERR_CUDA
    assert _call(op=4 * A + 48, ot=4 * A + 96, of=4 * A + 144) == _lib.UC_ERR_CUDA   # next to one another
    assert _call(os=2 * A) == _lib.UC_ERR_CUDA                                       # in place


@pytest.mark.parametrize("kw", [dict(os=2 * A, n=5), dict(os=2 * A, n=3), dict(os=2 * A + 4), dict(op=2 * A),
                                dict(ot=2 * A + 44), dict(of=2 * A), dict(of=3 * A), dict(of=3 * A + 11),
                                dict(os=3 * A), dict(op=4 * A), dict(ot=4 * A + 44), dict(ot=5 * A - 4),
                                dict(of=6 * A + 47), dict(of=4 * A)])
def test_shared(kw):
    assert _call(**kw) == _lib.UC_ERR_ARG
    assert b"beam_select" in LIB().uc_last_error()

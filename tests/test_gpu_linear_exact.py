"""Prompts' outputs carry one rounding, their own to bf16.

The factors that the tensor cores take (the decayed q.k and the state) enter as
two bf16 parts each, 2^-18 of a factor at most, and sums are fp32: both are far
below the output's own rounding, 2^-9, and independent of it. So the error's
norm is that of rounding the fp64 result to bf16, within a percent (an
independent error a seventh of it; a factor rounded to bf16 once alone is as
large as it, 1.2 to 1.4 times in all)."""
import numpy as np
import pytest
import torch

from oracle import linear as olinear
from tests.test_gpu_linear import _inputs, _np

pytestmark = pytest.mark.gpu

uc = pytest.importorskip("paper_2609_32831_gb300")


@pytest.mark.parametrize("T", [1, 8, 9, 65, 128, 129, 300, 515])
@pytest.mark.parametrize("hq,hkv,B", [(28, 4, 1), (2, 2, 2), (6, 2, 1), (9, 3, 1)])
@pytest.mark.parametrize("decays", ["slow", "fast", "mixed"])
def test_one_rounding(hq, hkv, B, T, decays):
    ld = {"slow": np.linspace(-0.01, -0.0003, hkv), "fast": np.linspace(-3.0, -0.3, hkv),
          "mixed": np.linspace(-0.5, 0.0, hkv)}[decays].tolist()
    q, k, v, s = _inputs(17 * T + hq, B, hq, hkv, T, state=T % 2 == 0)
    out, _ = uc.linear_attend(q, k, v, ld, state=s)
    ref, _, _, _ = olinear.linear_attend(_np(q), _np(k), _np(v), [float(np.float32(x)) for x in ld], _np(s))
    own = torch.from_numpy(ref).to(torch.bfloat16).double().numpy() - ref
    assert np.linalg.norm(_np(out) - ref) <= 1.01 * np.linalg.norm(own)

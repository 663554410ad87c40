"""conf_kv_attend_pages over tensors that are not dense: weights that are a slice of wider rows, and pages whose rows lie gigabytes apart.
Formulas and tolerances of the call's own tests."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_pages import _Case, torch_cuda  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,G,new,context", [(128, 4, [1, 3], [700, 5]), (128, 2, [40, 2], [30, 700]), (64, 8, [30], [600]), (64, 2, [2], [9])])
def test_weights_as_a_projection_leaves_them(lib, torch_cuda, D, G, new, context):
    c = _Case(lib, torch_cuda, D, G, 2, 16, new, context, diff=True)
    wide = torch_cuda.full((c.R, 3 * G + 5), float("nan"), device="cuda")
    lam = wide[:, G + 1:2 * G + 1]
    lam.copy_(c.on(c.lam))
    c.run(lam=lam)

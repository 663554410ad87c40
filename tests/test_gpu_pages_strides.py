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


@pytest.mark.parametrize("apart", [(1 << 26) - 8, 1 << 26, 1 << 29])
@pytest.mark.parametrize("D,G,new,context", [
    (128, 4, [1, 2], [300, 7]), (128, 4, [70, 1], [200, 129]), (128, 2, [200], [700]), (64, 8, [40, 9], [130, 0]), (64, 1, [3], [100]), (64, 4, [300], [5])])
def test_rows_that_lie_far_apart(lib, torch_cuda, D, G, new, context, apart):
    """Slots of a page `apart` values from one to the next, pages side by side: the rows of one load of a wavefront are up to a gigabyte
    apart, or so far that the distance takes more than 32 bits."""
    c = _Case(lib, torch_cuda, D, G, 2, 8, new, context, seed=2)
    step = 2 * D
    room = [torch_cuda.empty(7 * apart + c.n_pages * step, dtype=torch_cuda.float16, device="cuda") for _ in range(2)]
    far = [x.as_strided((c.n_pages, 8, 2, D), (step, apart, D, 1)) for x in room]
    for pages, x in zip(c.pages, far):
        x.copy_(pages)
    c.pages = far
    c.run()

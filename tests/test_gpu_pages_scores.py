"""conf_kv_attend_pages with scores far beyond what the exponential's argument resolves: 2^30 and more, from finite queries and keys.

Keys and queries that have one channel each make scores that are single products, exact in float32, so that the tolerance holds none of a
score's error: a probability is rounded to fp16 once as an operand (2^-11 of it) and so is the result; scores times log2(e) sm
are off by 2^-23 of their distance from the row's largest, of which those beyond 128 weigh less than 2^-128: 2^-15 of the others' size with
everything behind it; operands hold probabilities lifted, half a step of the smallest fp16 numbers is 2^-29 of the row's largest
(n of them), as in the tests of ordinary scores."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_pages import _Case, torch_cuda  # noqa: E402,F401

pytestmark = pytest.mark.gpu

_CALLS = [
    # D, G, new, context: a single token and parts of it, up to 32 rows, chunks, parts of them
    (128, 4, [1], [40]), (128, 4, [1, 5], [1000, 700]), (128, 16, [2], [300]), (64, 8, [1, 4], [700, 9]), (64, 1, [31], [3]),
    (128, 4, [40], [30]), (128, 5, [64, 3], [700, 0]), (64, 4, [130], [66]), (128, 2, [300], [400]),
]


def _first_channel(c, queries):
    """Scores queries[row][head] * sm * key: every key of a head another multiple of 16 below 2^15."""
    c.q[:] = 0
    c.q[:, :, 0] = queries
    for k in c.k:
        k[:] = 0
        for g in range(c.H):
            k[:, g, 0] = 16 * (1024 + c.rng.permutation(1024)[:len(k)])


def _check(c):
    got = c.out.cpu().numpy().astype(np.float64)
    sm, J = float(np.float32(1 / math.sqrt(c.D))), c.G // (2 if c.diff else 1)
    for b, (n, first, s) in enumerate(zip(c.new, c.context, c.starts)):
        for g in range(c.H):
            q, k, v = (x.astype(np.float64) for x in (c.q[s:s + n, g * c.G:(g + 1) * c.G, 0], c.k[b][:, g, 0], c.v[b][:, g]))
            score = q[..., None] * k * sm
            score[np.broadcast_to(np.arange(len(k)) > first + np.arange(n)[:, None, None], score.shape)] = -np.inf
            p = np.exp(score - score.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out, tol = p @ v, (2.0 ** -11 + 2.0 ** -15) * (p @ np.abs(v)) + len(k) * 2.0 ** -29 * np.abs(v).max()
            if c.diff:
                lam = c.lam[s:s + n, g * J:(g + 1) * J, None].astype(np.float64)
                out, tol = out[:, 0::2] - lam * out[:, 1::2], tol[:, 0::2] + np.abs(lam) * tol[:, 1::2]
            err = np.abs(got[s:s + n, g * J:(g + 1) * J] - out) / (tol + 2.0 ** -11 * np.abs(out) + 2.0 ** -25)
            assert np.all(err <= 1.0), f"sequence {b} head {g}: off by {np.nanmax(err):.3g} x tolerance at {np.argwhere(~(err <= 1))[:3]}"


@pytest.mark.parametrize("D,G,new,context,diff", [c + (d,) for c in _CALLS for d in (False, True) if not (d and c[1] % 2)])
def test_scores_of_all_sizes(lib, torch_cuda, D, G, new, context, diff):
    """Rows whose largest score is 2^27, -2^27 and of every size between, next to each other in one block."""
    c = _Case(lib, torch_cuda, D, G, 2, 16, new, context, diff=diff, seed=5)
    sizes = np.ldexp(1.0, c.rng.integers(-24, 16, c.q.shape[:2]))
    _first_channel(c, np.minimum(sizes, 2.0 ** 15) * c.rng.choice([-1.0, 1.0], c.q.shape[:2]))
    c.upload()
    c.call()
    _check(c)
    c.kv.close()


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("D,G,new,context", _CALLS)
def test_references_that_move_by_much(lib, torch_cuda, D, G, new, context, order):
    """Keys in rising and falling order, of both signs: a row's largest score goes from -2^27 to 2^27, or is the first one."""
    c = _Case(lib, torch_cuda, D, G, 1, 16, new, context, seed=6)
    _first_channel(c, c.rng.choice([1.0, -1.0, 2.0 ** 15, -2.0 ** 15], c.q.shape[:2]))
    for k in c.k:
        values = np.concatenate([-np.arange(2047, 1023, -1), np.arange(1024, 2048)]) * 16.0
        k[:, 0, 0] = np.sort(c.rng.choice(values, len(k), replace=False))[::order]
    c.upload()
    c.call()
    _check(c)
    c.kv.close()


@pytest.mark.parametrize("size", [3000.0, 65504.0])
@pytest.mark.parametrize("D,G,new,context", _CALLS)
def test_the_largest_numbers(lib, torch_cuda, D, G, new, context, size):
    """All channels: whatever a score of that size is rounded to, a row stays between the values that it sees."""
    c = _Case(lib, torch_cuda, D, G, 1, 16, new, context, seed=7)
    sign = lambda x: np.where(x < 0, -size, size).astype(np.float16)
    c.q, c.k = sign(c.q), [sign(k) for k in c.k]
    c.q[:, 0] = size
    for k in c.k:
        k[::3] = size
    c.upload()
    c.call()
    got = c.out.cpu().numpy().astype(np.float64)
    for b, (n, first, s) in enumerate(zip(new, context, c.starts)):
        for t in range(n):
            v = c.v[b][:first + t + 1, 0].astype(np.float64)
            slack = 2.0 ** -10 * np.abs(v).max() + 2.0 ** -25
            assert np.all(got[s + t] >= v.min(0) - slack) and np.all(got[s + t] <= v.max(0) + slack), (b, t)
    c.kv.close()

"""conf_kv_attend_pages and keys, values and queries that are infinite or NaN, in all forms of the call: both head widths, groups
of one to sixteen heads, two kv-heads, single tokens and chunks, sequences cut into parts, tokens that the pages hold already (slots
behind the last token NaN), differences of two maps.

A key whose score is NaN or infinite upwards leaves a row that sees it no number; one that is infinite downwards has no weight.  A value
that is no number makes its channel what such values add up to, in the rows that see it.  Everything else is what it is without
them, to the tolerance of the call's own tests, which is taken over what a row sees."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_pages import _Case, torch_cuda  # noqa: E402,F401

pytestmark = pytest.mark.gpu

_CONFIGS = [(128, 1, False), (128, 5, False), (128, 16, False), (64, 1, False), (64, 4, False), (64, 8, False), (128, 2, True), (128, 6, True),
            (128, 16, True), (64, 2, True), (64, 8, True)]
_KINDS = {                                             # rows of a kv-head, tokens in front
    "few": (20, 70), "few in parts": (20, 1500), "full few": (32, 33), "many": (70, 30), "many in parts": (100, 900), "blocks": (600, 200)}


def _row(q, k, v, sm):
    """One query over the rows it sees: (output, tolerance), NaN where the row is no number."""
    n, D = k.shape
    with np.errstate(all="ignore"):
        products = q * k
        s = products.sum(-1) * sm
    if np.isnan(s).any() or (s == np.inf).any():
        return np.full(D, np.nan), np.full(D, np.inf)
    seen = np.isfinite(s)
    p = np.zeros(n)
    p[seen] = np.exp(s[seen] - s[seen].max())
    p /= p.sum()
    odd = ~np.isfinite(v)
    fine = np.where(odd, 0.0, v)
    size = np.abs(products[seen]).sum(-1).max() * sm * (D + 4) * 2.0 ** -24
    o = p @ fine
    tol = (2.0 ** -11 + 2.0 ** -18 + 2 * size) * (p @ np.abs(fine)) + n * 2.0 ** -29 * np.abs(fine).max()
    with np.errstate(all="ignore"):
        for d in np.nonzero(odd.any(0))[0]:
            o[d] = v[odd[:, d], d].sum()
    return o, tol


def _reference(c, b, g):
    n, first, s, G = c.new[b], c.context[b], c.starts[b], c.G
    sm = float(np.float32(1 / math.sqrt(c.D)))
    q, k, v = (x.astype(np.float64) for x in (c.q[s:s + n, g * G:(g + 1) * G], c.k[b][:, g], c.v[b][:, g]))
    rows = [[_row(q[t, j], k[:first + t + 1], v[:first + t + 1], sm) for j in range(G)] for t in range(n)]
    o, tol = (np.array([[r[i] for r in heads] for heads in rows]) for i in (0, 1))
    with np.errstate(all="ignore"):
        if c.diff:
            lam = c.lam[s:s + n, g * G // 2:(g + 1) * G // 2, None].astype(np.float64)
            o, tol = o[:, 0::2] - lam * o[:, 1::2], tol[:, 0::2] + np.abs(lam) * tol[:, 1::2]
        return o, tol + 2.0 ** -11 * np.abs(o) + 2.0 ** -25


def _check(c, what):
    got, J = c.out.cpu().numpy().astype(np.float64), c.G // (2 if c.diff else 1)
    for b, (n, s) in enumerate(zip(c.new, c.starts)):
        for g in range(c.H if n else 0):
            ref, tol = _reference(c, b, g)
            mine, fine = got[s:s + n, g * J:(g + 1) * J], np.isfinite(ref)
            assert np.isfinite(tol[fine]).all()
            assert np.array_equal(np.isnan(mine), np.isnan(ref)), (what, b, g, np.argwhere(np.isnan(mine) != np.isnan(ref))[:3])
            assert np.array_equal(mine[np.isinf(ref)], ref[np.isinf(ref)]), (what, b, g)
            err = np.abs(mine[fine] - ref[fine]) / tol[fine]
            assert np.all(err <= 1.0), f"{what} sequence {b} head {g}: off by {err.max():.3g} x tolerance"


@pytest.mark.parametrize("own_rows", [True, False])
@pytest.mark.parametrize("kind", _KINDS)
@pytest.mark.parametrize("D,G,diff", _CONFIGS)
def test_they_show_where_they_are_seen(lib, torch_cuda, D, G, diff, kind, own_rows):
    rows, context = _KINDS[kind]
    n = max(1, rows // G)
    c = _Case(lib, torch_cuda, D, G, 2, 16, [n, 1], [context, 40], diff=diff, own_rows=own_rows, seed=rows + G)
    # one in front, one in the middle of the new tokens, the last one; different channels; the second kv-head only
    places = [(context // 3, 5), (context + n // 2, D - 3), (context + n - 1, 40)]
    clean = [x.copy() for x in (c.k[0], c.v[0])]
    for plane in ("k", "v"):
        for value in (np.inf, -np.inf, np.nan):
            what = f"{plane} {value}"
            print(what, flush=True)
            c.k[0][:], c.v[0][:] = clean
            for t, d in places:
                getattr(c, plane)[0][t, 1, d] = value
            c.upload()
            c.call()
            _check(c, what)
    # both infinities in one channel, and next to each other
    c.k[0][:], c.v[0][:] = clean
    for t, d, value in ((context // 3, 5, np.inf), (context // 2, 5, -np.inf), (context // 2, 6, np.inf), (context + n - 1, 6, np.inf)):
        c.v[0][t, 1, d] = value
    c.upload()
    c.call()
    _check(c, "both infinities")
    c.kv.close()


@pytest.mark.parametrize("D,G,new,context", [(128, 4, [3], [200]), (128, 4, [1], [2000]), (128, 4, [40], [30]), (64, 8, [40], [700]), (128, 2, [300], [5])])
@pytest.mark.parametrize("diff", [False, True])
def test_queries_that_are_no_numbers(lib, torch_cuda, D, G, new, context, diff):
    """They show in their own row only (their pair's, of two maps)."""
    c = _Case(lib, torch_cuda, D, G, 2, 16, new, context, diff=diff, seed=3)
    first = c.starts[0]
    c.q[first, 1, 7], c.q[first + new[0] - 1, G, D - 1] = np.nan, np.inf
    c.call()
    _check(c, "queries")
    c.kv.close()


@pytest.mark.parametrize("D,G,new,context", [(128, 4, [1], [0]), (128, 4, [2], [1500]), (64, 4, [40], [0]), (128, 2, [40], [900])])
@pytest.mark.parametrize("diff", [False, True])
def test_rows_that_see_nothing_of_any_weight(lib, torch_cuda, D, G, new, context, diff):
    """All scores infinite downwards: no number; rows behind a key that has a weight are its values."""
    c = _Case(lib, torch_cuda, D, G, 1, 16, new, context, diff=diff, seed=4)
    c.q[:, :, 9] = 1.0
    c.k[0][:, :, 9] = -np.inf
    last = len(c.k[0]) - 1
    if new[0] > 1:
        c.k[0][last, 0, 9] = 0.0
    c.upload()
    c.call()
    got = c.out.cpu().numpy()[c.starts[0]:c.starts[0] + new[0]].astype(np.float64)
    blind = new[0] if new[0] == 1 else new[0] - 1
    assert np.isnan(got[:blind]).all()
    if blind < new[0]:
        v = c.v[0][last, 0].astype(np.float64)
        w = 1.0 - c.lam[c.starts[0] + blind].astype(np.float64)[:, None] if diff else np.ones((G, 1))
        size = 1.0 + (np.abs(c.lam[c.starts[0] + blind])[:, None] if diff else 0.0)
        assert np.all(np.abs(got[blind] - w * v) <= (2.0 ** -11 + 2.0 ** -18) * size * np.abs(v) + 2.0 ** -11 * np.abs(w * v) + 2.0 ** -25)
    c.kv.close()

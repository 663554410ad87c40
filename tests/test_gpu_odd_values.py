"""Keys and values that are no numbers in decode attention, with and without a shared prefix: what a sequence sees of them shows in its
output, whatever the number of splits and wavefronts, and whatever the other sequences see.

  a key that is NaN       its score and with it every probability of the row is NaN: the whole output is
  a value v, |v| = inf    p v = v for every probability p > 0, however small: the output's channel is v, NaN where both infinities meet
  a value that is NaN     the output's channel is NaN"""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_gpu_shared import _Case  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


_FORMS = [(128, 4, 1), (128, 1, 1), (64, 4, 1), (64, 1, 1), (128, 16, 1), (128, 4, 3)]


def _out(c, prefix, q, kn, vn):
    torch = c.torch
    out = torch.zeros(c.B, c.tq, c.H * c.G, c.D, dtype=torch.float16, device="cuda")
    x = [c.on(z) for z in (q, kn, vn)]
    if prefix:
        seen = None if c.seen is None else c.on(np.array(c.seen, np.int32))
        c.kv.attend_shared(0, *x, out, *c.shared, seen=seen)
    elif c.tq > 1:
        c.kv.attend_chunk(0, *x, out)
    else:
        c.kv.attend(0, *x, out)
    got = out.cpu().numpy().astype(np.float64)
    assert c.kv.counters().device_errors == 0
    return got


@pytest.mark.parametrize("splits,two_launch", [(1, False), (3, False), (4, True)])
@pytest.mark.parametrize("prefix,D,G,tq", [(False, 128, 8, 4)] + [(p, *f) for p in (False, True) for f in _FORMS])
def test_own_key_not_a_number(lib, torch_cuda, monkeypatch, prefix, D, G, tq, splits, two_launch):
    """The call's last key is NaN, in a cache of 700 tokens on several splits: nothing but NaN for the token that sees it."""
    c = _Case(lib, torch_cuda, monkeypatch, D, G, 2, 2, 300, 700, -1, tq=tq, splits=splits, two_launch=two_launch, seed=G)
    q, kn, vn = c.inputs()
    kn[0, -1, 1, 5] = math.nan
    got = _out(c, prefix, q, kn, vn)
    hit = np.zeros(got.shape, bool)
    hit[0, -1, G:] = True
    assert np.array_equal(np.isnan(got), hit) and np.isfinite(got[~hit]).all()
    ema = c.kv.export(0, 0, 1)["ema"], c.kv.export(0, 0, 0)["ema"], c.kv.export(0, 1, 1)["ema"]
    assert np.isnan(ema[0]).all() and np.isfinite(ema[1]).all() and np.isfinite(ema[2]).all()
    c.close()


@pytest.mark.parametrize("T0", [0, 1, 8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("prefix,D,G,tq", [(False, 128, 8, 4)] + [(p, *f) for p in (False, True) for f in _FORMS])
def test_own_key_not_a_number_in_a_tile_of_its_own(lib, torch_cuda, monkeypatch, prefix, D, G, tq, T0):
    """The call's first key is NaN and, at some of these lengths, the only one that its wavefront meets, so that the wavefront's
    largest score is that of one that met nothing; the other wavefronts, or the prefix, have numbers."""
    for T in (1, 700) if prefix else (1,):
        c = _Case(lib, torch_cuda, monkeypatch, D, G, 2, 2, T, T0, -1, tq=tq, seed=T0)
        q, kn, vn = c.inputs()
        kn[1, 0, 0, 7] = math.nan
        got = _out(c, prefix, q, kn, vn)
        hit = np.zeros(got.shape, bool)
        hit[1, :, :G] = True
        assert np.array_equal(np.isnan(got), hit) and np.isfinite(got[~hit]).all(), T
        assert np.isnan(c.kv.export(0, 1, 0)["ema"]).all() and np.isfinite(c.kv.export(0, 1, 1)["ema"]).all(), T
        c.close()


_LAUNCHES = [(1, False), (3, False), (3, True)]


def _leading(c, lead, where, at):
    """Queries that score 0 with every key but one, which leads them by `lead`: the prefix's key `at`, or the call's own."""
    q, kn, vn = c.inputs()
    q[:], kn[:], c.pk[:] = 0, 0, 0
    q[..., 0] = 16
    key = np.float16(lead * math.sqrt(c.D) / 16)
    if where == "prefix":
        c.pk[:, at, 0] = key
    else:
        kn[..., 0] = key
    return q, kn, vn


def _share(c):
    c.shared[0].copy_(c.on(c.pk))
    c.shared[1].copy_(c.on(c.pv))


@pytest.mark.parametrize("splits,two_launch", _LAUNCHES)
@pytest.mark.parametrize("row_waves", [1, 2, 4])
@pytest.mark.parametrize("D,G,tq", _FORMS)
def test_prefix_key_not_a_number_behind_larger_scores(lib, torch_cuda, monkeypatch, D, G, tq, row_waves, splits, two_launch):
    """Scores 150 above all others, in the prefix and in the cache, beside which the weight of the part with the NaN vanishes in
    float32; a cache of 200 tokens, and one of which a wavefront has all."""
    for where, T, T0 in (("prefix", 1500, 200), ("own", 1500, 200), ("prefix", 100, 0), ("own", 100, 0)):
        c = _Case(lib, torch_cuda, monkeypatch, D, G, 1, 2, T, T0, -1, tq=tq, splits=splits, two_launch=two_launch, row_waves=row_waves)
        q, kn, vn = _leading(c, 150.0, where, T - 1)
        c.pk[0, 9, 1] = math.nan
        _share(c)
        c.seen = [T, 9]
        got = _out(c, True, q, kn, vn)
        assert np.isnan(got[0]).all() and np.isfinite(got[1]).all(), (where, T)
        c.close()


@pytest.mark.parametrize("splits,two_launch", _LAUNCHES)
@pytest.mark.parametrize("D,G,tq", _FORMS)
def test_own_key_not_a_number_behind_a_larger_prefix(lib, torch_cuda, monkeypatch, D, G, tq, splits, two_launch):
    for T, T0 in ((1500, 200), (100, 1)):
        c = _Case(lib, torch_cuda, monkeypatch, D, G, 1, 2, T, T0, -1, tq=tq, splits=splits, two_launch=two_launch)
        q, kn, vn = _leading(c, 150.0, "prefix", T // 2)
        kn[1, 0, 0, 2] = math.nan
        _share(c)
        got = _out(c, True, q, kn, vn)
        assert np.isnan(got[1]).all() and np.isfinite(got[0]).all(), T
        c.close()


@pytest.mark.parametrize("splits,two_launch", _LAUNCHES)
@pytest.mark.parametrize("row_waves", [1, 2, 4])
@pytest.mark.parametrize("lead", [0.0, 20.0, 40.0, 200.0])
@pytest.mark.parametrize("D,G,tq", _FORMS)
def test_odd_prefix_values_of_any_weight(lib, torch_cuda, monkeypatch, D, G, tq, lead, row_waves, splits, two_launch):
    """Values that are infinite or NaN, with a probability of e^-lead beside one key of the prefix or of the cache: what the
    sequences that see them get is the same whether the others see them or not."""
    B, T, at = 3, 1500, (3, 700, 701, 1499)
    for where in ("prefix", "own"):
        for seen in (None, [T, T, 2], [T, 702, 1490]):
            c = _Case(lib, torch_cuda, monkeypatch, D, G, 1, B, T, 40, -1, tq=tq, splits=splits, two_launch=two_launch, row_waves=row_waves,
                      seen=seen)
            q, kn, vn = _leading(c, lead, where, 1)
            odd = ((at[0], 0, math.inf), (at[1], 9, -math.inf), (at[1], D - 1, math.nan), (at[2], 33, math.inf), (at[2], 9, -math.inf),
                   (at[3], 33, -math.inf), (at[3], 50, math.inf))
            for t, d, x in odd:
                c.pv[0, t, d] = x
            _share(c)
            got = _out(c, True, q, kn, vn)
            for b in range(B):
                ref = [0.0] * D
                for t, d, x in odd:
                    if t < (T if seen is None else seen[b]):
                        ref[d] += x                           # (infinities that meet: NaN)
                ref = np.array(ref)
                fine = ref == 0
                assert np.isfinite(got[b][..., fine]).all(), (where, seen, b)
                shown = np.broadcast_to(ref[~fine], got[b][..., ~fine].shape)
                assert np.array_equal(got[b][..., ~fine], shown, equal_nan=True), (where, seen, b, got[b][0, 0, ~fine], ref[~fine])
            c.close()

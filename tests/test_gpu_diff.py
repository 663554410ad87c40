"""conf_kv_attend_diff against the formulas in 64 bits: the difference of two softmax maps over the mixed cache, and the importance that
follows the size of a value's weight.

Tolerance of the outputs, from the arithmetic: of each map a probability is rounded to fp16 once as an operand (2^-11 of it); the result
is once; a score is a float32 sum of D products, off by at most (D + 4) 2^-24 of sum |q_d K_d| * sm, which moves a probability
by twice that, relative; exponentials, sums and weights of the merges stay under 2^-18 together.  INT8 values meet probabilities times
their scale, rounded once, biased by a constant whose share is taken back in float32: 2^-18 of its size, 1024 + 128 codes.  The second
map's errors count its weight.  An importance is a float64 sum of float32 exponentials: twice the score's error and 2^-21 of each map's
probability."""
import math
import os
import sys

import numpy as np
import pytest

from oracle import confkv_oracle as O

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from harness import Report, compare_unit_state, f32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def _attend(u, q, kn, vn, lam, pos0, sm, decay, gain):
    """Oracle: tokens q [tq][G][D] of one unit with weights lam [tq][G / 2].  (outputs, their tolerance, importance, its tolerance)."""
    tq = q.shape[0]
    a = np.concatenate([u.ema.astype(np.float64), np.zeros(tq)])
    slack, outs, tols, n_old = np.zeros_like(a), [], [], u.n
    for t in range(tq):
        O.append_token(u, kn[t], vn[t], pos0 + t)
        k, v, x = u.stored_k(), u.stored_v(), q[t].astype(np.float64)
        _, p = O.attention_naive(x, k, v, sm)
        score = (np.abs(x) @ np.abs(k).T).max(1, keepdims=True) * sm * (q.shape[-1] + 4) * 2.0 ** -24
        l = lam[t].astype(np.float64)[:, None]
        w = p[0::2] - l * p[1::2]
        out = w @ v
        one = (2.0 ** -11 + 2.0 ** -18 + 2 * score) * (p @ np.abs(v))
        if not u.is16.all():
            one = one + 2.0 ** -18 * 9.1 * (p @ (np.abs(v).max(1, keepdims=True) * ~u.is16[:, None]))
        tols.append(one[0::2] + np.abs(l) * one[1::2] + 2.0 ** -11 * np.abs(out) + 2.0 ** -25)
        outs.append(out)
        n = n_old + t + 1
        near = (2 * score + 2.0 ** -21) * p
        a[:n] = decay * a[:n] + gain * np.abs(w).sum(0)
        slack[:n] = decay * slack[:n] + gain * (near[0::2] + np.abs(l) * near[1::2]).sum(0)
    u.ema = a.astype(np.float32)
    return np.stack(outs), np.stack(tols), a, slack + 2.0 ** -23 * np.abs(a) + 1e-38


class _Case:
    def __init__(self, lib, torch, monkeypatch, D, G, H, B, T0, W, tq=1, splits=0, two_launch=False, scales="token", layout="contiguous",
                 seed=0, budget=None, per_token=True, **kw):
        monkeypatch.setenv("CONF_KV_SPLITS", str(splits))
        monkeypatch.setenv("CONF_KV_TWO_LAUNCH", str(int(two_launch)))
        self.torch, self.D, self.G, self.H, self.B, self.W, self.tq, self.per_token = torch, D, G, H, B, W, tq, per_token
        self.budget = budget or T0 + 40
        page = 16 if layout == "paged" else 0
        self.P, self.page, self.pos = max(8, W) if layout == "paged" else 8, page, T0
        cap = (max(T0, self.budget, self.P + page) + 2 * tq + 2 * page + max(W, 0) + 64 + 63) // 64 * 64
        self.kv = lib.ConfKV(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=100, capacity=cap, fp16_window=W,
                             protected_window=self.P, n_tight=[self.budget], n_loose=[self.budget], scale_mode=scales,
                             max_chunk=tq if tq > 1 else 0, evict_page=page, layout=layout, **kw)
        self.decay, self.gain = f32(0.9), f32(1) - f32(0.9)
        self.rng = np.random.default_rng(seed)
        K, V, e0 = self.normal(B, H, T0, D), self.normal(B, H, T0, D), self.rng.random((B, H, T0)).astype(np.float32)
        if T0:
            self.kv.load_prefill(0, *(self.on(x) for x in (K, V, e0)))
        self.units = {(b, g): O.load_prefill(K[b, g], V[b, g], W, e0[b, g], scale_mode=scales) for b in range(B) for g in range(H)}

    def on(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def normal(self, *shape):
        return self.rng.standard_normal(shape).astype(np.float16)

    def inputs(self):
        B, H, G, D, tq = self.B, self.H, self.G, self.D, self.tq
        lam = self.rng.uniform(-0.5, 1.5, (B, tq, H * G // 2) if self.per_token else (H * G // 2,)).astype(np.float32)
        return self.normal(B, tq, H * G, D), self.normal(B, tq, H, D), self.normal(B, tq, H, D), lam

    def step(self, what="", inputs=None):
        G, J = self.G, self.G // 2
        q, kn, vn, lam = inputs or self.inputs()
        out = self.torch.full((self.B, self.tq, self.H * J, self.D), math.nan, dtype=self.torch.float16, device="cuda")
        self.kv.attend_diff(0, self.on(q), self.on(kn), self.on(vn), out, self.on(lam))
        got, worst = out.cpu().numpy().astype(np.float64), 0.0
        lam = np.broadcast_to(lam, (self.B, self.tq, self.H * J))
        for (b, g), u in self.units.items():
            ref, tol, mass, near = _attend(u, q[b, :, g * G:(g + 1) * G], kn[b, :, g], vn[b, :, g], lam[b, :, g * J:(g + 1) * J], self.pos,
                                           f32(1 / math.sqrt(self.D)), self.decay, self.gain)
            err = np.abs(got[b, :, g * J:(g + 1) * J] - ref) / tol
            assert np.all(err <= 1.0), f"{what} unit {(b, g)}: out off by {np.nanmax(err):.3g} x tolerance"
            worst = max(worst, float(err.max()))
            ema = self.kv.export(0, b, g, planes={"ema"})["ema"]
            assert len(ema) == len(mass)
            off = np.abs(ema - mass) / near
            assert np.all(off <= 1.0), f"{what} unit {(b, g)}: importance off by {off.max():.3g} x tolerance"
            u.ema = ema.copy()                                         # (what decides the eviction is the stored one)
        self.kv.evict_compact()
        rep = Report()
        for (b, g), u in self.units.items():
            O.evict_compact_unit(u, self.budget, self.P, f32(0.65), self.W, page=self.page)
            compare_unit_state(self.kv.export(0, b, g), u, f"{what} unit {(b, g)}", rep)
        self.pos += self.tq
        return worst

    def close(self):
        assert self.kv.counters().device_errors == 0
        self.kv.close()


_SHAPES = [
    # D, G, H, B, T0, W, tq, splits
    (128, 2, 2, 2, 200, 40, 1, 0),
    (128, 4, 1, 1, 0, 4, 1, 0),                # nothing but the token itself
    (128, 4, 2, 2, 777, 40, 1, 5),
    (128, 6, 1, 2, 300, 0, 1, 2),
    (128, 8, 2, 3, 600, 24, 1, 3),
    (128, 8, 1, 1, 3000, -1, 1, 0),
    (128, 16, 1, 2, 200, 64, 1, 3),            # sixteen rows of one token
    (128, 12, 2, 1, 150, 32, 1, 0),
    (128, 10, 1, 2, 900, 32, 1, 7),
    (128, 4, 2, 2, 200, 40, 4, 0),             # several tokens per call
    (128, 2, 2, 3, 200, 16, 8, 2),
    (128, 2, 1, 2, 700, -1, 5, 4),
    (128, 6, 1, 2, 120, -1, 2, 0),
    (128, 8, 8, 1, 64, 8, 2, 1),
    (64, 2, 3, 4, 256, -1, 1, 0),
    (64, 2, 12, 1, 700, 32, 1, 4),
    (64, 4, 2, 3, 130, 100, 1, 2),
    (64, 6, 2, 2, 97, 16, 1, 0),
    (64, 8, 2, 9, 300, 48, 1, 0),
]


@pytest.mark.parametrize("two_launch", [False, True])
@pytest.mark.parametrize("D,G,H,B,T0,W,tq,splits", _SHAPES)
def test_outputs_and_importance(lib, torch_cuda, monkeypatch, D, G, H, B, T0, W, tq, splits, two_launch):
    print(f"diff D={D} G={G} H={H} B={B} T0={T0} W={W} tq={tq} splits={splits} two_launch={two_launch}", flush=True)
    c = _Case(lib, torch_cuda, monkeypatch, D, G, H, B, T0, W, tq=tq, splits=splits, two_launch=two_launch, seed=T0 + B,
              per_token=splits != 2)
    for t in range(2):
        worst = c.step(f"step {t}")
    print(f"  out {worst:.3g} x tolerance", flush=True)
    c.close()


@pytest.mark.parametrize("G,scales,layout,W,splits", [(4, "channel", "contiguous", 24, 0), (12, "channel", "contiguous", 8, 3),
                                                      (4, "token", "paged", 8, 0), (8, "token", "paged", 16, 2), (2, "token", "paged", 16, 3)])
def test_storage_variants(lib, torch_cuda, monkeypatch, G, scales, layout, W, splits):
    c = _Case(lib, torch_cuda, monkeypatch, 128, G, 2, 3, 400, W, scales=scales, layout=layout, seed=G, splits=splits)
    for t in range(3):
        c.step(f"{scales} {layout} step {t}")
    c.close()


@pytest.mark.parametrize("splits", [0, 3])
def test_lockstep_with_eviction(lib, torch_cuda, monkeypatch, splits):
    """Importance decides what goes: 30 steps at a budget below the prompt's length, kept sets as the oracle's."""
    c = _Case(lib, torch_cuda, monkeypatch, 128, 4, 2, 2, 420, 16, budget=400, seed=11, splits=splits)
    for t in range(30):
        c.step(f"step {t}")
    assert c.kv.counters().evicted > 0
    c.close()


@pytest.mark.parametrize("splits", [0, 2])
def test_equal_maps_cancel(lib, torch_cuda, monkeypatch, splits):
    """Two maps alike with weight one leave nothing, to the bit; with weight zero the first map is conf_kv_attend's."""
    torch, D, G, H, B, T0 = torch_cuda, 128, 4, 2, 2, 500
    c = _Case(lib, torch, monkeypatch, D, G, H, B, T0, 40, seed=3, splits=splits)
    q, kn, vn, _ = c.inputs()
    q[:, :, 1::2] = q[:, :, 0::2]
    out = torch.full((B, 1, H * G // 2, D), 7.0, dtype=torch.float16, device="cuda")
    ones = torch.ones(H * G // 2, device="cuda")
    c.kv.attend_diff(0, c.on(q), c.on(kn), c.on(vn), out, ones)
    assert not out.any()
    c.close()
    both = []
    for lam in (None, 0.0):
        c = _Case(lib, torch, monkeypatch, D, G, H, B, T0, 40, seed=3, splits=splits)
        q, kn, vn, _ = c.inputs()
        if lam is None:
            o = torch.empty(B, H * G, D, dtype=torch.float16, device="cuda")
            c.kv.attend(0, c.on(q[:, 0]), c.on(kn[:, 0]), c.on(vn[:, 0]), o)
            both.append(o[:, 0::2])
        else:
            o = torch.empty(B, 1, H * G // 2, D, dtype=torch.float16, device="cuda")
            c.kv.attend_diff(0, c.on(q), c.on(kn), c.on(vn), o, ones * 0)
            both.append(o[:, 0])
        c.close()
    assert torch.equal(*both)


@pytest.mark.parametrize("splits", [0, 3])
def test_strided_weights(lib, torch_cuda, monkeypatch, splits):
    """Weights as a projection leaves them: a slice of wider rows."""
    c = _Case(lib, torch_cuda, monkeypatch, 128, 4, 2, 2, 300, 16, tq=3, seed=9, splits=splits)
    put = c.on
    wide = torch_cuda.full((2, 3, 50), math.nan, device="cuda")

    def on(x):
        if x.dtype != np.float32:
            return put(x)
        wide[:, :, 7:11] = put(x)
        return wide[:, :, 7:11]
    c.on = on
    c.step("strided")
    c.close()


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("plane", ["k", "v"])
def test_values_that_are_no_numbers(lib, torch_cuda, monkeypatch, plane, splits):
    """They show in the outputs of the kv-head that holds them and in no other."""
    torch = torch_cuda
    for bad in (math.inf, math.nan):
        c = _Case(lib, torch, monkeypatch, 128, 4, 2, 1, 600, -1, seed=1, splits=splits)
        q, kn, vn, lam = c.inputs()
        (kn if plane == "k" else vn)[0, 0, 1, 3] = bad
        out = torch.zeros(1, 1, 4, 128, dtype=torch.float16, device="cuda")
        c.kv.attend_diff(0, c.on(q), c.on(kn), c.on(vn), out, c.on(lam))
        ok = torch.isfinite(out[0, 0])
        assert ok[:2].all()
        if plane == "v":
            assert not ok[2:, 3].any() and ok[2:, :3].all() and ok[2:, 4:].all()
        else:                                          # (an infinite score downwards is one of no weight)
            for j in (2, 3):
                shows = math.isnan(bad) or (q[0, 0, 2 * j:2 * j + 2, 3] > 0).any()
                assert (not ok[j].any()) if shows else ok[j].all()
        c.close()


def test_a_recorded_step(lib, torch_cuda, monkeypatch):
    """attend_diff, step and evict_compact recorded once, replayed against an eager twin."""
    torch = torch_cuda
    twins = [_Case(lib, torch, monkeypatch, 128, 4, 2, 2, 300, 16, budget=280, seed=21) for _ in range(2)]
    q, kn, vn, lam = (twins[0].on(x) for x in twins[0].inputs())
    outs = [torch.zeros(2, 1, 4, 128, dtype=torch.float16, device="cuda") for _ in range(2)]

    def step(i):
        twins[i].kv.attend_diff(0, q, kn, vn, outs[i], lam)
        twins[i].kv.evict_compact()
    for i in range(2):
        twins[i].kv.static_plan(True)
        step(i)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(0)
    for t in range(6):
        fresh = twins[0].inputs()
        for dst, src in zip((q, kn, vn, lam), fresh):
            dst.copy_(torch.from_numpy(src))
        g.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(*outs), t
        for b in range(2):
            x, y = (c.kv.export(0, b, 1) for c in twins)
            assert np.array_equal(x["ema"], y["ema"]) and np.array_equal(x["pos"], y["pos"])
    for c in twins:
        c.close()


def test_refusals(lib, torch_cuda, monkeypatch):
    torch, b = torch_cuda, lib.binding
    t = lambda *s, d=torch.float16: torch.zeros(s, dtype=d, device="cuda")
    f32_ = torch.float32
    c = _Case(lib, torch, monkeypatch, 128, 4, 2, 2, 50, 8, tq=8)
    ok = lambda tq: [t(2, tq, 8, 128), t(2, tq, 2, 128), t(2, tq, 2, 128), t(2, tq, 4, 128), t(2, tq, 4, d=f32_)]

    def status(args, layer=0):
        with pytest.raises(lib.ConfKVError) as e:
            c.kv.attend_diff(layer, *args)
        return e.value.status
    assert status(ok(5)) == b.ERR_INVALID_ARG                        # twenty rows
    assert status(ok(9)) == b.ERR_INVALID_ARG
    assert status(ok(1), layer=1) == b.ERR_BAD_LAYER
    for i, bad in ((0, t(2, 1, 7, 128)), (3, t(2, 1, 8, 128)), (4, t(2, 1, 4)), (4, t(2, 1, 8, d=f32_)[..., ::2]), (4, t(3, d=f32_)),
                   (4, t(2, 2, 4, d=f32_))):
        args = ok(1)
        args[i] = bad
        with pytest.raises(ValueError):
            c.kv.attend_diff(0, *args)
    c.kv.attend_diff(0, *ok(2))
    assert status(ok(1)) == b.ERR_BAD_STATE                          # one call per layer and step
    c.kv.evict_compact()
    c.close()
    odd = _Case(lib, torch, monkeypatch, 128, 3, 2, 2, 50, 8)
    with pytest.raises(lib.ConfKVError) as e:
        odd.kv.attend_diff(0, t(2, 1, 6, 128), t(2, 1, 2, 128), t(2, 1, 2, 128), t(2, 1, 3, 128), t(2, 1, 3, d=f32_))
    assert e.value.status == b.ERR_INVALID_ARG
    odd.close()

"""conf_kv_attend_shared against the formulas in 64 bits: one softmax over the prefix a sequence sees and its cache.

Tolerance of the outputs, from the arithmetic: every probability is rounded to fp16 once as an operand (2^-11 of it) and so is
the result; a score is a float32 sum of D products, off by at most (D + 4) 2^-24 of sum |q_d K_d| * sm, which moves a
probability by twice that, relative; exponentials, sums and weights of the merges stay under 2^-18 together.  Stored importance: the
harness's 1e-5 (scores of these inputs are below 10, so that their error is below 2e-6)."""
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


def _attend(u, q, kn, vn, pos0, pk, pv, sm, lam):
    """Oracle: tokens q [tq][G][D] of one unit behind prefix rows pk, pv.  Returns (out, tolerance) [tq][G][D]."""
    tq, T = q.shape[0], pk.shape[0]
    a = np.concatenate([u.ema.astype(np.float64), np.zeros(tq)])
    n_old, outs, tols = u.n, [], []
    for t in range(tq):
        O.append_token(u, kn[t], vn[t], pos0 + t)
        k = np.concatenate([pk.astype(np.float64), u.stored_k()])
        v = np.concatenate([pv.astype(np.float64), u.stored_v()])
        x = q[t].astype(np.float64)
        out, p = O.attention_naive(x, k, v, sm)
        score = (np.abs(x) @ np.abs(k).T).max(1, keepdims=True) * sm * (q.shape[-1] + 4) * 2.0 ** -24
        weight = p @ np.abs(v)
        tols.append(2.0 ** -11 * np.abs(out) + (2.0 ** -11 + 2.0 ** -18 + 2 * score) * weight + 2.0 ** -25)
        outs.append(out)
        n = n_old + t + 1
        a[:n] = lam * a[:n] + (1 - lam) * p[:, T:].sum(0)
    u.ema = a.astype(np.float32)
    return np.stack(outs), np.stack(tols)


class _Case:
    """A handle of one layer, its oracle units and the prefix."""

    def __init__(self, lib, torch, monkeypatch, D, G, H, B, T, T0, W, tq=1, splits=0, two_launch=False, scales="token",
                 layout="contiguous", seen=None, seed=0, budget=None, spread=1.0, row_waves=0):
        monkeypatch.setenv("CONF_KV_SPLITS", str(splits))
        monkeypatch.setenv("CONF_KV_TWO_LAUNCH", str(int(two_launch)))
        monkeypatch.setenv("CONF_KV_SHARED_ROWS", str(row_waves))
        self.torch, self.D, self.G, self.H, self.B, self.T, self.W, self.tq = torch, D, G, H, B, T, W, tq
        self.budget = budget or T0 + 40
        page = 16 if layout == "paged" else 0
        self.P = max(8, W) if layout == "paged" else 8
        self.page = page
        cap = (max(T0, self.budget, self.P + page) + 2 * tq + 2 * page + max(W, 0) + 64 + 63) // 64 * 64
        self.kv = lib.ConfKV(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=100, capacity=cap, fp16_window=W,
                             protected_window=self.P, n_tight=[self.budget], n_loose=[self.budget], scale_mode=scales,
                             max_chunk=tq if tq > 1 else 0, evict_page=page, layout=layout, max_shared=T)
        self.rng = np.random.default_rng(seed)
        self.pk, self.pv = self.normal(H, T, D), self.normal(H, T, D)
        self.pk = (self.pk * spread).astype(np.float16)
        K, V, e0 = self.normal(B, H, T0, D), self.normal(B, H, T0, D), self.rng.random((B, H, T0)).astype(np.float32)
        if T0:
            self.kv.load_prefill(0, *(self.on(x) for x in (K, V, e0)))
        elif scales == "channel":
            raise ValueError("channel scales come from a prompt")
        self.units = {(b, g): O.load_prefill(K[b, g], V[b, g], W, e0[b, g], scale_mode=scales) for b in range(B) for g in range(H)}
        self.seen, self.pos = seen, T0
        # the prefix lives in a longer buffer, full of NaN around it
        room = torch.full((2, H, T + 5, D), math.nan, dtype=torch.float16, device="cuda")
        room[0, :, :T], room[1, :, :T] = self.on(self.pk), self.on(self.pv)
        self.shared = room[0, :, :T], room[1, :, :T]

    def on(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def normal(self, *shape):
        return self.rng.standard_normal(shape).astype(np.float16)

    def inputs(self):
        B, H, G, D, tq = self.B, self.H, self.G, self.D, self.tq
        return self.normal(B, tq, H * G, D), self.normal(B, tq, H, D), self.normal(B, tq, H, D)

    def step(self, what=""):
        torch, G = self.torch, self.G
        q, kn, vn = self.inputs()
        out = torch.full((self.B, self.tq, self.H * G, self.D), math.nan, dtype=torch.float16, device="cuda")
        seen = None if self.seen is None else self.on(np.array(self.seen, np.int32))
        self.kv.attend_shared(0, self.on(q), self.on(kn), self.on(vn), out, *self.shared, seen=seen)
        got = out.cpu().numpy().astype(np.float64)
        worst = 0.0
        for (b, g), u in self.units.items():
            T = self.T if self.seen is None else min(max(self.seen[b], 0), self.T)
            ref, tol = _attend(u, q[b, :, g * G:(g + 1) * G], kn[b, :, g], vn[b, :, g], self.pos, self.pk[g, :T], self.pv[g, :T],
                               f32(1 / math.sqrt(self.D)), f32(0.9))
            err = np.abs(got[b, :, g * G:(g + 1) * G] - ref) / tol
            assert np.all(err <= 1.0), f"{what} unit {(b, g)}: out off by {np.nanmax(err):.3g} x tolerance"
            worst = max(worst, float(err.max()))
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
    # D, G, H, B, T, T0, W, tq, splits
    (128, 4, 2, 2, 300, 200, 40, 1, 0),
    (128, 4, 1, 8, 1, 100, 16, 1, 0),          # one prefix token; 32 rows: one wavefront's
    (128, 4, 1, 9, 31, 100, 16, 1, 0),         # 36 rows: two wavefronts along the rows
    (128, 4, 1, 17, 33, 60, 16, 1, 0),         # 68: four
    (128, 8, 1, 17, 257, 60, 16, 1, 0),        # 136: a second workgroup along the rows
    (128, 4, 2, 2, 128, 200, 40, 1, 3),
    (128, 4, 2, 2, 129, 777, 40, 1, 5),
    (128, 1, 3, 2, 500, 200, -1, 1, 0),        # the vector-ALU body
    (128, 1, 1, 1, 700, 0, 4, 1, 0),           # nothing cached: prefix and the token itself
    (64, 1, 3, 4, 513, 256, -1, 1, 0),
    (64, 1, 2, 2, 513, 700, -1, 1, 4),
    (64, 4, 2, 3, 127, 130, 100, 1, 2),
    (64, 8, 2, 9, 640, 300, 48, 1, 0),
    (64, 7, 1, 2, 65, 97, -1, 1, 0),
    (128, 5, 2, 3, 1001, 300, 24, 1, 0),
    (128, 2, 1, 1, 64, 300, 0, 1, 2),
    (128, 16, 1, 2, 300, 200, 64, 1, 3),       # sixteen rows of one token
    (128, 12, 2, 1, 95, 150, 32, 1, 0),
    (128, 9, 1, 3, 200, 100, -1, 1, 0),
    (128, 4, 2, 2, 300, 200, 40, 4, 0),        # several tokens per call
    (128, 1, 2, 3, 77, 200, 16, 13, 2),
    (128, 5, 1, 2, 160, 120, -1, 3, 0),
    (128, 8, 1, 5, 2000, 64, 8, 2, 1),
    (128, 4, 1, 1, 9000, 300, 40, 1, 2),       # more parts than wavefronts
    (64, 8, 24, 5, 5003, 60, 16, 1, 0),        # several turns of a workgroup
    (128, 4, 32, 9, 1801, 40, 16, 1, 0),
]


@pytest.mark.parametrize("D,G,H,B,T,T0,W,tq,splits", _SHAPES)
@pytest.mark.parametrize("two_launch,row_waves", [(False, 1), (False, 2), (False, 4), (True, 0)])
def test_outputs_and_importance(lib, torch_cuda, monkeypatch, D, G, H, B, T, T0, W, tq, splits, two_launch, row_waves):
    print(f"shared D={D} G={G} H={H} B={B} T={T} T0={T0} W={W} tq={tq} splits={splits} two_launch={two_launch} rows {row_waves}", flush=True)
    c = _Case(lib, torch_cuda, monkeypatch, D, G, H, B, T, T0, W, tq=tq, splits=splits, two_launch=two_launch, seed=T + B,
              row_waves=row_waves)
    for t in range(2):
        worst = c.step(f"step {t}")
    print(f"  out {worst:.3g} x tolerance", flush=True)
    c.close()


@pytest.mark.parametrize("G,scales,layout,W", [(4, "channel", "contiguous", 24), (12, "channel", "contiguous", 8), (4, "token", "paged", 8),
                                               (5, "token", "paged", 16)])
def test_storage_variants(lib, torch_cuda, monkeypatch, G, scales, layout, W):
    c = _Case(lib, torch_cuda, monkeypatch, 128, G, 2, 3, 333, 200, W, scales=scales, layout=layout, seed=G)
    for t in range(3):
        c.step(f"{scales} {layout} step {t}")
    c.close()


@pytest.mark.parametrize("row_waves", [1, 2, 4])
@pytest.mark.parametrize("G,B,T", [(4, 7, 400), (1, 33, 300), (8, 20, 130), (4, 40, 1500)])
def test_sequences_that_see_part_of_the_prefix(lib, torch_cuda, monkeypatch, G, B, T, row_waves):
    """All of it, some, none; counts outside 0 .. T are held within."""
    seen = [(T, T // 2 + 1, 0, -7, T - 1, 2 ** 31 - 1, 1)[b % 7] for b in range(B)]
    c = _Case(lib, torch_cuda, monkeypatch, 128, G, 1, B, T, 70, 16, seen=seen, seed=B, row_waves=row_waves)
    c.step("part")
    c.seen = [0] * B
    c.step("nobody sees it")
    c.seen = None
    c.step("everybody")
    c.close()


def test_lockstep_with_eviction(lib, torch_cuda, monkeypatch):
    """Importance decides what goes: 30 steps at a budget below the prompt's length, kept sets as the oracle's."""
    c = _Case(lib, torch_cuda, monkeypatch, 128, 4, 2, 2, 250, 120, 16, budget=90, seen=[250, 100], seed=11)
    for t in range(30):
        c.step(f"step {t}")
    assert c.kv.counters().evicted > 0
    c.close()


def test_sharp_scores(lib, torch_cuda, monkeypatch):
    """Keys many times as long: the largest score moves from tile to tile, and one side's weight vanishes beside the other's."""
    for spread in (4.0, 0.0):
        c = _Case(lib, torch_cuda, monkeypatch, 128, 4, 1, 3, 700, 80, 16, spread=spread, seed=5)
        q = c.inputs
        c.inputs = lambda: tuple((x.astype(np.float32) * f).astype(np.float16) for x, f in zip(q(), (2.0, 1.0, 1.0)))
        torch = torch_cuda
        qq, kn, vn = c.inputs()
        out = torch.empty(3, 1, 4, 128, dtype=torch.float16, device="cuda")
        c.kv.attend_shared(0, c.on(qq), c.on(kn), c.on(vn), out, *c.shared)
        got = out.cpu().numpy().astype(np.float64)
        for (b, g), u in c.units.items():
            ref, tol = _attend(u, qq[b], kn[b, :, 0], vn[b, :, 0], 80, c.pk[0], c.pv[0], f32(1 / math.sqrt(128)), f32(0.9))
            assert np.all(np.abs(got[b] - ref) <= tol)
        c.close()


@pytest.mark.parametrize("row_waves", [1, 4])
@pytest.mark.parametrize("lead", [11.0, 14.0])
def test_long_tails_of_small_probabilities(lib, torch_cuda, monkeypatch, row_waves, lead):
    """One key leads all others by `lead`: 20000 equal probabilities of e^-lead (1.7e-5 and 8e-7) hold a quarter or a sixtieth of
    the weight, and their rounding as operands has the same sign for all of them."""
    torch, T, D = torch_cuda, 20000, 128
    c = _Case(lib, torch, monkeypatch, D, 4, 1, 2, T, 20, 16, seed=2, row_waves=row_waves)
    c.pk[:], c.pv[:] = 0, 1
    c.pk[0, 77, 0], c.pv[0, 77] = 4.0, -1
    c.shared[0].copy_(c.on(c.pk))
    c.shared[1].copy_(c.on(c.pv))
    q, kn, vn = c.inputs()
    q[:], kn[:] = 0, 0
    q[..., 0] = lead * math.sqrt(D) / 4.0
    out = torch.empty(2, 1, 4, D, dtype=torch.float16, device="cuda")
    c.kv.attend_shared(0, c.on(q), c.on(kn), c.on(vn), out, *c.shared)
    got = out.cpu().numpy().astype(np.float64)
    for (b, g), u in c.units.items():
        ref, tol = _attend(u, q[b], kn[b, :, 0], vn[b, :, 0], 20, c.pk[0], c.pv[0], f32(1 / math.sqrt(D)), f32(0.9))
        err = np.abs(got[b] - ref) / tol
        assert np.all(err <= 1.0), f"{err.max():.3g} x tolerance"
    c.close()


@pytest.mark.parametrize("row_waves", [1, 2, 4])
@pytest.mark.parametrize("kind", ["inf value", "nan value", "nan key", "inf key"])
def test_odd_values_reach_only_those_who_see_them(lib, torch_cuda, monkeypatch, kind, row_waves):
    """A value or key that is no number shows in the sequences that see its token and in no other, also where their rows share
    tiles with rows that do see it."""
    torch = torch_cuda
    G, B, T, T0, D = 4, 9, 200, 50, 128
    at = 150
    seen = [T, at, at + 1, 0, 10, T, at, 100, 151]
    c = _Case(lib, torch, monkeypatch, D, G, 1, B, T, T0, 16, seen=seen, seed=3, row_waves=row_waves)
    plane = c.shared[1] if "value" in kind else c.shared[0]
    plane[0, at, 3] = math.nan if "nan" in kind else math.inf
    q, kn, vn = c.inputs()
    q[:, :, :, 3] = np.abs(q[:, :, :, 3]) + np.float16(0.1)      # (an infinite key scores +inf: no number)
    out = torch.zeros(B, 1, G, D, dtype=torch.float16, device="cuda")
    c.kv.attend_shared(0, c.on(q), c.on(kn), c.on(vn), out, *c.shared, seen=c.on(np.array(seen, np.int32)))
    got = out.cpu().numpy()[:, 0]
    for b in range(B):
        hit = seen[b] > at
        if not hit:
            assert np.isfinite(got[b]).all(), (b, kind)
        elif "value" in kind:
            odd = np.isnan(got[b]) if "nan" in kind else np.isposinf(got[b])
            assert odd[:, 3].all() and np.isfinite(np.delete(got[b], 3, axis=1)).all(), (b, kind)
        else:
            assert np.isnan(got[b]).all(), (b, kind)
    c.close()


def test_every_score_of_a_part_not_a_number(lib, torch_cuda, monkeypatch):
    """A prefix of one token whose key is NaN: nothing but NaN comes out, importance included."""
    torch = torch_cuda
    for G, D in ((4, 128), (1, 64)):
        c = _Case(lib, torch, monkeypatch, D, G, 1, 1, 1, 50, 16 if G > 1 else -1, seed=3)
        c.shared[0][0, 0, 0] = math.nan
        q, kn, vn = c.inputs()
        out = torch.zeros(1, 1, G, D, dtype=torch.float16, device="cuda")
        c.kv.attend_shared(0, c.on(q), c.on(kn), c.on(vn), out, *c.shared)
        assert bool(out.isnan().all())
        assert np.isnan(c.kv.export(0, 0, 0)["ema"]).all()
        c.close()


def test_no_prefix_is_the_ordinary_call(lib, torch_cuda, monkeypatch):
    torch = torch_cuda
    outs = []
    for shared in (False, True):
        c = _Case(lib, torch, monkeypatch, 128, 4, 2, 2, 64, 300, 40, tq=2, seed=9)
        q, kn, vn = (c.on(x) for x in c.inputs())
        out = torch.zeros(2, 2, 8, 128, dtype=torch.float16, device="cuda")
        if shared:
            c.kv.attend_shared(0, q, kn, vn, out, c.shared[0][:, :0], c.shared[1][:, :0])
        else:
            c.kv.attend_chunk(0, q, kn, vn, out)
        outs.append((out.cpu(), c.kv.export(0, 1, 1)["ema"]))
        c.close()
    assert torch.equal(outs[0][0], outs[1][0]) and np.array_equal(outs[0][1], outs[1][1])


def test_replayed_steps(lib, torch_cuda, monkeypatch):
    """A step recorded once and replayed, with eager work and changed inputs (what is seen included) in between, against the
    oracle at every replay."""
    torch = torch_cuda
    B, G, H, D, T = 3, 4, 2, 128, 700
    c = _Case(lib, torch, monkeypatch, D, G, H, B, T, 200, 24, budget=210, seed=21)
    c.kv.static_plan(True)
    c.seen = [T, 300, 0]
    c.step("eager")
    bufs = [c.on(x) for x in c.inputs()]
    seen = c.on(np.array(c.seen, np.int32))
    out = torch.zeros(B, 1, G * H, D, dtype=torch.float16, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.kv.attend_shared(0, *bufs, out, *c.shared, seen=seen)
        c.kv.evict_compact()
    # (the recording ran nothing; the handle's own count of a pending append is as after a step)
    for t in range(6):
        c.seen = [T - 10 * t, 300 + t, 0 if t % 2 else 5]
        x = c.inputs()
        for buf, host in zip(bufs, x):
            buf.copy_(c.on(host))
        seen.copy_(c.on(np.array(c.seen, np.int32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy().astype(np.float64)
        for (b, g), u in c.units.items():
            n = min(max(c.seen[b], 0), T)
            ref, tol = _attend(u, x[0][b, :, g * G:(g + 1) * G], x[1][b, :, g], x[2][b, :, g], c.pos, c.pk[g, :n], c.pv[g, :n],
                               f32(1 / math.sqrt(D)), f32(0.9))
            assert np.all(np.abs(got[b, :, g * G:(g + 1) * G] - ref) <= tol), f"replay {t} unit {(b, g)}"
            O.evict_compact_unit(u, c.budget, c.P, f32(0.65), c.W)
            compare_unit_state(c.kv.export(0, b, g), u, f"replay {t} unit {(b, g)}", Report())
        c.pos += 1
    c.close()


def test_two_handles_on_two_streams(lib, torch_cuda, monkeypatch):
    """Calls of two handles that share one prefix tensor, each on a stream of its own, give what they give one after the other."""
    torch = torch_cuda
    runs = []
    for together in (False, True):
        cs = [_Case(lib, torch, monkeypatch, 128, 4, 2, 2, 2000, 300, 24, seed=31 + i) for i in range(2)]
        streams = [torch.cuda.Stream() for _ in cs]
        xs = [[c.on(x) for x in c.inputs()] for c in cs]
        outs = [torch.zeros(2, 1, 8, 128, dtype=torch.float16, device="cuda") for _ in cs]
        torch.cuda.synchronize()
        for c, s, x, o in zip(cs, streams, xs, outs):
            with torch.cuda.stream(s):
                c.kv.attend_shared(0, *x, o, *cs[0].shared)
                c.kv.evict_compact()
            if not together:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        runs.append([o.cpu() for o in outs])
        for c in cs:
            c.close()
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_refusals(lib, torch_cuda, monkeypatch):
    torch = torch_cuda
    from paper_2605_24786_amd import binding as b
    c = _Case(lib, torch, monkeypatch, 128, 4, 2, 2, 64, 100, 16, tq=8, seed=1)
    kv, (pk, pv) = c.kv, c.shared
    room = torch.zeros(2, 100, 128, dtype=torch.float16, device="cuda")
    z = lambda tq, h: torch.zeros(2, tq, h, 128, dtype=torch.float16, device="cuda")
    call = lambda tq=1, k=pk, v=pv, **kw: kv.attend_shared(0, z(tq, 8), z(tq, 2), z(tq, 2), z(tq, 8), k, v, **kw)

    def status(*args, **kw):
        with pytest.raises(lib.ConfKVError) as e:
            call(*args, **kw)
        return e.value.status

    assert status(5) == b.ERR_INVALID_ARG                       # 20 rows per kv-head
    assert status(9) == b.ERR_INVALID_ARG                       # more than max_chunk
    assert status(k=room[:, :65], v=room[:, :65]) == b.ERR_INVALID_ARG     # more than max_shared
    off = torch.zeros(2 * 70 * 128 + 8, dtype=torch.float16, device="cuda")[4:4 + 2 * 70 * 128].view(2, 70, 128)[:, :64]
    assert status(k=off, v=off) == b.ERR_INVALID_ARG            # 8-byte alignment
    odd = torch.as_strided(room, (2, 50, 128), (50 * 128 + 4, 128, 1))
    assert status(k=odd, v=odd) == b.ERR_INVALID_ARG            # kv-heads 8 bytes off a 16-byte boundary
    close = torch.as_strided(room, (2, 50, 128), (49 * 128, 128, 1))
    assert status(k=close, v=close) == b.ERR_INVALID_ARG        # kv-heads that overlap
    for kw in (dict(k=pk.float()), dict(k=pk[:1]), dict(v=pv[:, :32]), dict(k=pk[:, ::2], v=pv[:, ::2]), dict(v=pv.contiguous()),
               dict(seen=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(seen=torch.zeros(2, device="cuda")), dict(k=pk.cpu())):
        with pytest.raises(ValueError):
            call(**kw)
    assert kv.lib.conf_kv_attend_shared(kv.h, 0, 1, None, *(x.data_ptr() for x in (z(1, 8), z(1, 2), z(1, 2), z(1, 8))), None) == b.ERR_INVALID_ARG
    call(4)                                                     # (nothing was appended by the refused calls)
    with pytest.raises(lib.ConfKVError) as e:
        call()
    assert e.value.status == b.ERR_BAD_STATE
    kv.close()
    none = _Case(lib, torch, monkeypatch, 128, 4, 2, 2, 0, 100, 16, seed=1).kv     # made without room for prefixes
    with pytest.raises(lib.ConfKVError):
        none.attend_shared(0, z(1, 8), z(1, 2), z(1, 2), z(1, 8), pk, pv)
    none.close()


@pytest.mark.parametrize("row_waves", [1, 2, 4])
@pytest.mark.parametrize("D,G,tq", [(128, 4, 1), (64, 1, 1), (128, 4, 3)])
@pytest.mark.parametrize("size", [1000.0, 9000.0, 60000.0])
def test_largest_scores(lib, torch_cuda, monkeypatch, size, D, G, tq, row_waves):
    """Queries and keys as large as FP16 holds: scores of 5e6 to 4e10, of which one key has the largest by more than any rounding.
    What it leaves to the others is nothing, and its probability is one."""
    torch = torch_cuda
    T = 1300
    c = _Case(lib, torch, monkeypatch, D, G, 1, 4, T, 40, -1, tq=tq, seed=int(size), row_waves=row_waves)
    for win in (0, 31, 700, T - 1):
        q, kn, vn = c.inputs()
        q[:] = size
        c.pk[:] = (c.rng.random((1, T, D)) * 0.5 * size).astype(np.float16)      # a quarter of the largest score, more or less
        c.pk[0, win] = size * (0.9 + 0.1 * c.rng.random())
        c.shared[0].copy_(c.on(c.pk))
        out = torch.full((4, tq, G, D), math.nan, dtype=torch.float16, device="cuda")
        c.kv.attend_shared(0, c.on(q), c.on(kn), c.on(vn), out, *c.shared)
        got = out.cpu().numpy()
        assert np.array_equal(got, np.broadcast_to(c.pv[0, win], got.shape)), win
        c.kv.evict_compact()
        assert all(np.isfinite(c.kv.export(0, b, 0)["ema"]).all() for b in range(4))
    c.close()

"""A serving program's decode step with all of its calls: conf_kv_prepare_qkv, conf_kv_attend_shared per layer, then
conf_kv_constrain, conf_kv_step and conf_kv_evict_compact, against the formulas in 64 bits at every step -- called one by one, and
recorded once into a HIP graph and replayed with eager work in between.

The model between the calls is random rows and logits.  Prepared rows are checked against the rotation's formulas and then
given to the oracle as they are (an fp16 rounding that differs must not be carried on); constrained logits likewise.
Tolerances: test_gpu_prepare.py's, test_gpu_shared.py's, test_gpu_constrain.py's, the harness's for confidence and cache."""
import math
import os
import sys

import numpy as np
import pytest

from oracle import confkv_oracle as O

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from harness import CONF_ATOL, Report, compare_unit_state, f32  # noqa: E402
from test_gpu_constrain import _check, _expected  # noqa: E402
from test_gpu_prepare import _close, _reference  # noqa: E402
from test_gpu_shared import _attend  # noqa: E402

pytestmark = pytest.mark.gpu

L, B, H, G, D, V, T, T0, W, P = 2, 3, 2, 4, 128, 5003, 333, 90, 16, 12
TIGHT, LOOSE = 60, 84
TAU = 0.45


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


class _Program:
    """Everything a serving program holds: the handle, the shared prefix, the histories, and buffers of fixed place."""

    def __init__(self, lib, torch, seed):
        self.torch, self.rng = torch, np.random.default_rng(seed)
        normal = lambda *s: self.rng.standard_normal(s).astype(np.float16)
        self.on = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.kv = lib.ConfKV(n_layers=L, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=V, capacity=128, fp16_window=W,
                             protected_window=P, n_tight=[TIGHT] * L, n_loose=[LOOSE] * L, tau=TAU, max_shared=T)
        self.pk, self.pv = normal(L, H, T, D), normal(L, H, T, D)
        self.units, self.shared = {}, []
        for l in range(L):
            K, Vv = normal(B, H, T0, D), normal(B, H, T0, D)
            self.kv.load_prefill(l, self.on(K), self.on(Vv))
            self.shared.append((self.on(self.pk[l]), self.on(self.pv[l])))
            for b in range(B):
                for g in range(H):
                    self.units[l, b, g] = O.load_prefill(K[b, g], Vv[b, g], W)
        self.seen = [T, 200, 0]
        self.pos = T0
        self.rows = torch.zeros(L, B, 1, H * (G + 2), D, dtype=torch.bfloat16, device="cuda")
        half = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")
        self.q16, self.out = half(L, B, 1, G * H, D), half(L, B, 1, G * H, D)
        self.k16, self.v16 = half(L, B, 1, H, D), half(L, B, 1, H, D)
        self.freq = (10000.0 ** (-torch.arange(48).double() / 48)).float().cuda()
        self.wq, self.wk = (1 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(seed + i)) for i in range(2))
        self.wq, self.wk = self.wq.cuda(), self.wk.cuda()
        self.seen_dev = self.on(np.array(self.seen, np.int32))
        self.logits = torch.zeros(B, V, dtype=torch.bfloat16, device="cuda")
        self.shaped = torch.zeros(B, V, device="cuda")
        self.conf, self.sel = torch.zeros(B, device="cuda"), torch.zeros(B, dtype=torch.uint8, device="cuda")
        n = 64
        c = dict(tokens=self.rng.integers(0, V, (B, n)).astype(np.int32), lengths=np.array([20, 1, 0], np.int32),
                 prompt_lengths=np.array([12, 1, 0], np.int32))
        for name, lo, hi in (("repetition", 1.0, 1.5), ("presence", -0.5, 0.5), ("frequency", 0.0, 0.3)):
            c[name] = (lo + (hi - lo) * self.rng.random(B)).astype(np.float32)
        c["bias_offsets"] = np.array([0, 3, 3, 9], np.int32)
        c["bias_tokens"] = self.rng.integers(0, V, 9).astype(np.int32)
        c["bias_values"] = self.rng.standard_normal(9).astype(np.float32)
        c["bits"] = self.rng.random((B, V)) < 0.7
        c["allowed"] = np.packbits(np.pad(c["bits"], ((0, 0), (0, -V % 32))), axis=1, bitorder="little").view(np.int32)
        self.c = c
        self.dev = {k: self.on(c[k]) for k in c if k != "bits"}

    def calls(self):
        for l in range(L):
            r = self.rows[l]
            self.kv.prepare_qkv(l, r[:, :, :G * H], r[:, :, G * H:G * H + H], r[:, :, G * H + H:], self.q16[l], self.k16[l], self.v16[l],
                                freq=self.freq, first=T, q_weight=self.wq, k_weight=self.wk, eps=1e-6)
            self.kv.attend_shared(l, self.q16[l], self.k16[l], self.v16[l], self.out[l], *self.shared[l], seen=self.seen_dev)
        self.kv.constrain(self.logits, self.shaped, **self.dev)
        self.kv.step(self.shaped, self.conf, self.sel)
        self.kv.evict_compact()

    def new_inputs(self, t):
        """The model's rows and logits of step t; the tokens it chose so far enter the histories."""
        torch = self.torch
        self.rows.copy_(self.on(self.rng.standard_normal(self.rows.shape).astype(np.float32)))
        self.logits.copy_(self.on((self.rng.standard_normal((B, V)) * (0.5, 8.0)[t // 3 % 2]).astype(np.float32)))
        ln = self.c["lengths"]
        for b in range(B):
            self.c["tokens"][b, ln[b]] = self.rng.integers(0, 50)
            ln[b] += 1
        self.dev["tokens"].copy_(self.on(self.c["tokens"]))
        self.dev["lengths"].copy_(self.on(ln))
        torch.cuda.synchronize()

    def check(self, what):
        torch = self.torch
        torch.cuda.synchronize()
        pos = torch.full((B, 1), self.pos + T, dtype=torch.int32)
        x, y = self.logits.float().cpu().numpy(), self.shaped.cpu().numpy()
        _check(y, *_expected(self.c, x), what)
        ref = np.array([O.confidence(r, (f32(0.4), f32(0.3), f32(0.3))) for r in y])
        assert np.max(np.abs(self.conf.cpu().numpy() - ref)) <= CONF_ATOL, what
        sel = self.sel.cpu().numpy().astype(bool)
        far = np.abs(ref - f32(TAU)) > 1e-5
        assert np.array_equal(sel[far], (ref >= f32(TAU))[far]), what
        for l in range(L):
            r = self.rows[l]
            _close(torch, self.q16[l], *_reference(torch, r[:, :, :G * H], self.wq, self.freq, pos, False, 1e-6), f"{what} queries")
            _close(torch, self.k16[l], *_reference(torch, r[:, :, G * H:G * H + H], self.wk, self.freq, pos, False, 1e-6), f"{what} keys")
            q, k, v, out = (z[l].cpu().numpy() for z in (self.q16, self.k16, self.v16, self.out))
            for b in range(B):
                for g in range(H):
                    u, n = self.units[l, b, g], self.seen[b]
                    ref, tol = _attend(u, q[b, :, g * G:(g + 1) * G], k[b, :, g], v[b, :, g], self.pos, self.pk[l, g, :n],
                                       self.pv[l, g, :n], f32(1 / math.sqrt(D)), f32(0.9))
                    err = np.abs(out[b, :, g * G:(g + 1) * G].astype(np.float64) - ref)
                    assert np.all(err <= tol), f"{what} unit {(l, b, g)}"
                    O.evict_compact_unit(u, TIGHT if sel[b] else LOOSE, P, f32(0.65), W)
                    compare_unit_state(self.kv.export(l, b, g), u, f"{what} unit {(l, b, g)}", Report())
        self.pos += 1
        return sel


@pytest.mark.parametrize("recorded", [False, True])
def test_decode_steps(lib, torch_cuda, recorded):
    torch = torch_cuda
    p = _Program(lib, torch, seed=17)
    p.kv.static_plan(True)
    graph, tight = None, 0
    for t in range(14):
        p.new_inputs(t)
        if graph is not None:
            graph.replay()
        else:
            p.calls()
        tight += int(p.check(f"step {t}").sum())
        if recorded and t == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                p.calls()
    st = p.kv.counters()
    assert st.device_errors == 0 and st.evicted > 0 and 0 < tight < 14 * B
    print(f"recorded={recorded}: {st.evicted} evicted, {tight} tight choices of {14 * B}", flush=True)
    p.kv.close()


def test_prompt_hand_over(lib, torch_cuda):
    """conf_kv_prepare_qkv in the prompt layout, conf_kv_load_prefill of what it wrote, and the first token behind a prefix: the
    cache holds the prepared keys bit for bit."""
    torch = torch_cuda
    n = 70
    kv = lib.ConfKV(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=V, capacity=128, fp16_window=n,
                    protected_window=P, n_tight=[100], n_loose=[100], max_shared=T)
    g = torch.Generator().manual_seed(4)
    rows = torch.randn(B, n, H * (G + 2), D, generator=g).bfloat16().cuda()
    q, k, v = rows[:, :, :G * H], rows[:, :, G * H:G * H + H], rows[:, :, G * H + H:]
    freq = (10000.0 ** (-torch.arange(64).double() / 64)).float().cuda()
    pos = (T + torch.arange(n, dtype=torch.int32)).repeat(B, 1).cuda()
    q16 = torch.empty(B, n, G * H, D, dtype=torch.float16, device="cuda")
    k16, v16 = (torch.empty(B, H, n, D, dtype=torch.float16, device="cuda") for _ in range(2))
    kv.prepare_qkv(0, q, k, v, q16, k16, v16, freq=freq, pos=pos, prompt=True)
    kv.load_prefill(0, k16, v16)
    _close(torch, k16.transpose(1, 2), *_reference(torch, k, None, freq, pos, False, 0.0), "keys")
    for b in range(B):
        for h in range(H):
            ex = kv.export(0, b, h)
            assert np.array_equal(ex["k16"].view(np.uint16), k16[b, h].cpu().numpy().view(np.uint16))
            assert np.array_equal(ex["v16"].view(np.uint16), v16[b, h].cpu().numpy().view(np.uint16))
    new = [torch.empty(B, 1, x, D, dtype=torch.float16, device="cuda") for x in (G * H, H, H)]
    kv.prepare_qkv(0, q[:, :1], k[:, :1], v[:, :1], *new, freq=freq, first=T)          # the layer's next place is n
    at = torch.full((B, 1), T + n, dtype=torch.int32)
    _close(torch, new[0], *_reference(torch, q[:, :1], None, freq, at, False, 0.0), "the next token's queries")
    kv.close()

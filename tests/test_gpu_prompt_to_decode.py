"""From projection rows to decoding, with the calls in their order: a prompt in chunks over pages (conf_kv_prepare_qkv,
conf_kv_attend_pages), its pages into the mixed cache (conf_kv_load_pages), the importance of its last queries (conf_kv_observe),
differential decode steps with budgets and evictions (conf_kv_attend_diff, conf_kv_step, conf_kv_evict_compact), against the formulas
in 64 bits and the oracle's cache.  Tolerances are those of the calls' own tests."""
import math
import os
import sys

import numpy as np
import pytest

from oracle import confkv_oracle as O

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from harness import Report, compare_unit_state, f32  # noqa: E402
from test_gpu_diff import _attend  # noqa: E402
from test_gpu_pages import _reference  # noqa: E402

pytestmark = pytest.mark.gpu

L, B, H, G, D, V = 2, 2, 2, 4, 128, 1000
PAGE, W, P, LOOSE, TIGHT = 16, 24, 8, 140, 120


@pytest.mark.parametrize("chunks", [(64, 64, 22), (1, 1, 5, 9, 134), (150,)])
def test_a_prompt_and_the_steps_behind_it(lib, chunks):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    T0 = sum(chunks)
    rng = np.random.default_rng(T0 + len(chunks))
    on = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    wide = -(-T0 // PAGE)
    kv = lib.ConfKV(n_layers=L, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=V, capacity=256, fp16_window=W,
                    protected_window=P, n_tight=[TIGHT] * L, n_loose=[LOOSE] * L, max_chunk=4, max_paged=wide * PAGE)
    freq = on((10000.0 ** (-np.arange(D // 2) / (D // 2))).astype(np.float32))
    weight = on(rng.uniform(0.5, 1.5, D).astype(np.float32))
    table = on(rng.permutation(B * wide).astype(np.int32).reshape(B, wide))
    pages = [[torch.full((B * wide, PAGE, H, D), math.nan, dtype=torch.float16, device="cuda") for _ in range(2)] for _ in range(L)]
    lam = rng.uniform(0.2, 0.9, (L, H * G // 2)).astype(np.float32)
    context = torch.zeros(B, dtype=torch.int32, device="cuda")
    half = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda")
    sm = f32(1 / math.sqrt(D))

    def projected(l, T, **kw):
        fused = on(rng.standard_normal((B, T, (G + 2) * H, D)).astype(np.float32))
        q, k, v = half(B, T, G * H, D), half(B, T, H, D), half(B, T, H, D)
        kv.prepare_qkv(l, fused[:, :, :G * H], fused[:, :, G * H:(G + 1) * H], fused[:, :, (G + 1) * H:], q, k, v, freq=freq, q_weight=weight,
                       k_weight=weight, **kw)
        return q, k, v

    qs, ks, vs = ([[] for _ in range(L)] for _ in range(3))
    at = 0
    for T in chunks:
        for l in range(L):
            pos = (context[:, None] + torch.arange(T, device="cuda", dtype=torch.int32)).contiguous()
            q, k, v = projected(l, T, pos=pos)
            out = half(B, T, G * H // 2, D)
            kv.attend_pages(q, k, v, out, *pages[l], table, context, lam=on(lam[l]))
            for rows, x in ((qs, q), (ks, k), (vs, v)):
                rows[l].append(x.cpu().numpy())
            keys, values = np.concatenate(ks[l], 1), np.concatenate(vs[l], 1)
            got = out.cpu().numpy().astype(np.float64)
            for b in range(B):
                for g in range(H):
                    ref, tol = _reference(qs[l][-1][b, :, g * G:(g + 1) * G], keys[b, :, g], values[b, :, g], at, sm,
                                          np.broadcast_to(lam[l, g * G // 2:(g + 1) * G // 2], (T, G // 2)))
                    assert np.all(np.abs(got[b, :, g * G // 2:(g + 1) * G // 2] - ref) <= tol), (T, l, b, g)
        context += T
        at += T
    units = {}
    for l in range(L):
        kv.load_pages(l, *pages[l], table, T0)
        q, k, v = (np.concatenate(x[l], 1) for x in (qs, ks, vs))
        last = on(q[:, T0 - 4:])
        kv.observe(l, T0 - 4, last)
        for b in range(B):
            for g in range(H):
                u = O.load_prefill(k[b, :, g], v[b, :, g], W, None)
                O.observe_unit(u, q[b, T0 - 4:, g * G:(g + 1) * G], T0 - 4, sm, f32(0.9), mass_gain=f32(1) - f32(0.9))
                compare_unit_state(kv.export(l, b, g), u, f"prompt unit {(l, b, g)}", Report())
                units[l, b, g] = u
    for t in range(4):
        for l in range(L):
            q, k, v = projected(l, 1)
            out = half(B, 1, G * H // 2, D)
            kv.attend_diff(l, q, k, v, out, on(lam[l]))
            got, (qn, kn, vn) = out.cpu().numpy().astype(np.float64), (x.cpu().numpy() for x in (q, k, v))
            for b in range(B):
                for g in range(H):
                    u, weights = units[l, b, g], lam[l, None, g * G // 2:(g + 1) * G // 2]
                    ref, tol, mass, near = _attend(u, qn[b, :, g * G:(g + 1) * G], kn[b, :, g], vn[b, :, g], weights, T0 + t, sm, f32(0.9),
                                                   f32(1) - f32(0.9))
                    assert np.all(np.abs(got[b, :, g * G // 2:(g + 1) * G // 2] - ref) <= tol)
                    ema = kv.export(l, b, g, planes={"ema"})["ema"]
                    assert np.all(np.abs(ema - mass) <= near)
                    u.ema = ema.copy()
        logits = rng.standard_normal((B, V)).astype(np.float32)
        sel = torch.zeros(B, dtype=torch.uint8, device="cuda")
        kv.step(on(logits), None, sel)
        kv.evict_compact()
        for (l, b, g), u in units.items():
            O.evict_compact_unit(u, TIGHT if int(sel[b]) else LOOSE, P, f32(0.65), W)
            compare_unit_state(kv.export(l, b, g), u, f"step {t} unit {(l, b, g)}", Report())
    assert kv.counters().device_errors == 0 and kv.counters().evicted > 0
    kv.close()

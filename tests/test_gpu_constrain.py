"""conf_kv_constrain against the formulas in 64 bits.

Tolerance per value: at most five float32 operations, each off by at most 2^-24 of what it gives, and what they give is
bounded by |x| max(r, 1/r) + frequency * count + |presence| + |bias|."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def _kv(lib, B, V):
    return lib.ConfKV(n_layers=1, batch=B, n_q_heads=1, n_kv_heads=1, head_dim=64, vocab=V, capacity=64, fp16_window=16,
                      protected_window=8, n_tight=[16], n_loose=[32])


def _case(B, V, n, m, seed, masks=None):
    """Host inputs: logits, histories with repeats and ids that do not exist, biases with repeats, masks."""
    rng = np.random.default_rng(seed)
    c = dict(logits=(3 * rng.standard_normal((B, V))).astype(np.float32))
    c["tokens"] = np.floor(V ** rng.random((B, n))).astype(np.int32) - 1
    if n > 3:
        c["tokens"][:, 1], c["tokens"][:, 2], c["tokens"][:, 3] = -1, V, 2 ** 31 - 1
    c["lengths"] = rng.integers(0, n + 1, B).astype(np.int32)
    c["lengths"][0] = n
    c["prompt_lengths"] = (c["lengths"] // 2).astype(np.int32)
    c["repetition"] = (0.7 + rng.random(B)).astype(np.float32)
    c["presence"] = rng.standard_normal(B).astype(np.float32)
    c["frequency"] = rng.standard_normal(B).astype(np.float32)
    cuts = np.sort(rng.integers(0, m + 1, B - 1)) if B > 1 else np.zeros(0)
    c["bias_offsets"] = np.concatenate([[0], cuts, [m]]).astype(np.int32)
    c["bias_tokens"] = rng.integers(-2, V + 2, m).astype(np.int32)
    if m > 4:
        c["bias_tokens"][m // 2:] = c["bias_tokens"][rng.integers(0, m // 2, m - m // 2)]       # tokens listed twice and more
    c["bias_values"] = rng.standard_normal(m).astype(np.float32)
    c["bias_values"][::7] = -np.inf
    if masks:
        c["bits"] = rng.random((masks, V)) < rng.random((masks, 1)) ** 2
        c["bits"][0] = False                                                          # a row that forbids everything
        words = (V + 31) // 32
        c["allowed"] = np.packbits(np.pad(c["bits"], ((0, 0), (0, words * 32 - V))), axis=1, bitorder="little").view(np.uint32)
    return c


def _expected(c, x, rows=None):
    """(values, bound of the magnitudes) in float64."""
    B, V = x.shape
    y, size = np.empty((B, V)), np.empty((B, V))
    for b in range(B):
        z, ln = x[b].astype(np.float64), (c["lengths"][b] if c.get("lengths") is not None else 0)
        hist = c["tokens"][b, :ln] if c.get("tokens") is not None else np.zeros(0, np.int64)
        pl = c["prompt_lengths"][b] if c.get("prompt_lengths") is not None else 0
        ok = lambda t: t[(t >= 0) & (t < V)]
        said = np.bincount(ok(hist[pl:]), minlength=V)
        seen = np.bincount(ok(hist), minlength=V) > 0
        get = lambda k, d: float(c[k][b]) if c.get(k) is not None else d
        r, p, f = get("repetition", 1.0), get("presence", 0.0), get("frequency", 0.0)
        z = np.where(seen, np.where(z > 0, z / r, z * r), z)
        size[b] = np.abs(z) * max(r, 1 / r) + abs(f) * said + abs(p)
        z = z - f * said - p * (said > 0)
        if c.get("bias_offsets") is not None:
            last = {}
            for i in range(c["bias_offsets"][b], c["bias_offsets"][b + 1]):
                if 0 <= c["bias_tokens"][i] < V:
                    last[int(c["bias_tokens"][i])] = float(c["bias_values"][i])
            for t, val in last.items():
                z[t] += val
                size[b, t] += abs(val) if math.isfinite(val) else 0.0
        if c.get("bits") is not None:
            m = b if rows is None else rows[b]
            if 0 <= m < len(c["bits"]):
                z[~c["bits"][m]] = -np.inf
        y[b] = z
    return y, size


def _check(got, ref, size, what):
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), what
    fine = np.isfinite(ref)
    err, tol = np.abs(got[fine] - ref[fine]), 5 * 2.0 ** -24 * size[fine] + 1e-38
    assert np.all(err <= tol), f"{what}: {np.max(err / tol):.3g} x tolerance"


_NAMES = ("tokens", "lengths", "prompt_lengths", "repetition", "presence", "frequency", "bias_offsets", "bias_tokens",
          "bias_values")


def _device(torch, c):
    kw = {k: torch.from_numpy(c[k]).cuda() for k in _NAMES if c.get(k) is not None}
    if c.get("allowed") is not None:
        kw["allowed"] = torch.from_numpy(c["allowed"].view(np.int32)).cuda()
    return kw


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("B,V,n,m,masks", [
    (1, 2, 1, 0, None), (1, 33, 0, 0, 1), (2, 31, 5, 3, 2), (3, 4096, 100, 40, 3), (2, 4097, 1000, 0, None),
    (1, 50257, 300, 17, 1), (5, 12007, 2, 1, 5), (2, 128256, 9000, 300, 2), (33, 1001, 64, 64, 33), (1, 152064, 40000, 1000, 1),
    (32, 50257, 3000, 64, 32), (64, 50256, 500, 10, None), (85, 50257, 100, 90, 85), (85, 50256, 30, 0, None),   # two, four, five quads per thread
])
def test_rows_match_the_formulas(lib, torch_cuda, dtype, B, V, n, m, masks):
    torch = torch_cuda
    print(f"constrain {dtype} B={B} V={V} history {n} biases {m} masks {masks}", flush=True)
    c = _case(B, V, n, m, seed=B + V + n, masks=masks)
    x = torch.from_numpy(c["logits"]).to(getattr(torch, dtype)).cuda()
    ref, size = _expected(c, x.float().cpu().numpy())
    kv = _kv(lib, B, V)
    out = torch.full((B, V), 9.0, device="cuda")
    kw = _device(torch, c)
    kv.constrain(x, out, **kw)
    torch.cuda.synchronize()
    _check(out.cpu().numpy(), ref, size, "dense rows")
    # rows of a wider tensor, at an odd place of it
    wide = torch.zeros(B, V + 13, dtype=x.dtype, device="cuda")
    wide[:, 5:5 + V] = x
    again = torch.full((B * V + 1,), 9.0, device="cuda")[1:].view(B, V)
    kv.constrain(wide[:, 5:5 + V], again, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    if dtype == "float32":                                                            # in place
        kv.constrain(x, x, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, x)
    kv.close()


def test_parts_alone(lib, torch_cuda):
    """Each part without the others, and nothing at all: a conversion to float32."""
    torch = torch_cuda
    B, V = 3, 5003
    full = _case(B, V, 400, 60, seed=8, masks=4)
    kv = _kv(lib, B, V)
    x = torch.from_numpy(full["logits"]).bfloat16().cuda()
    host = x.float().cpu().numpy()
    out = torch.empty(B, V, device="cuda")
    history = ("tokens", "lengths")
    for names in ((), history, history + ("repetition",), history + ("presence",), history + ("frequency", "prompt_lengths"),
                  history + ("repetition", "prompt_lengths"), ("bias_offsets", "bias_tokens", "bias_values"), ("bits", "allowed")):
        c = {k: full[k] for k in names}
        kv.constrain(x, out, **_device(torch, c))
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), *_expected(c, host), str(names))
    for rows in ([3, -1, 1], [0, 4, 2], [2 ** 31 - 1, -2 ** 31, 3]):                  # which mask row; outside: none
        c = {k: full[k] for k in ("bits", "allowed")}
        kv.constrain(x, out, allowed_rows=torch.tensor(rows, dtype=torch.int32, device="cuda"), **_device(torch, c))
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), *_expected(c, host, rows), str(rows))
    kv.close()


def test_masked_places_and_rows_that_allow_nothing(lib, torch_cuda):
    """NaN, infinities and the type's lowest value where the mask forbids become -inf; where it allows they stay.  A row that
    allows nothing goes through conf_kv_step: NaN, the loose budget, the other rows as ever."""
    torch = torch_cuda
    B, V = 3, 4100
    x = torch.randn(B, V, generator=torch.Generator().manual_seed(2)).cuda()
    odd = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(torch.float32).min, torch.finfo(torch.float32).max])
    x[:, :5] = odd.cuda()
    x[:, 4095:4100] = odd.cuda()
    bits = np.ones((B, V), bool)
    bits[0, :5], bits[1], bits[2, 4095:], bits[2, :5] = False, False, False, False
    words = np.packbits(np.pad(bits, ((0, 0), (0, 28))), axis=1, bitorder="little").view(np.int32)
    kv = _kv(lib, B, V)
    out, conf, sel = torch.empty(B, V, device="cuda"), torch.zeros(B, device="cuda"), torch.ones(B, dtype=torch.uint8, device="cuda")
    kv.constrain(x, out, allowed=torch.from_numpy(words).cuda())
    kv.step(out, conf, sel)
    torch.cuda.synchronize()
    o = out.cpu().numpy()
    ref = np.where(bits, x.cpu().numpy(), -np.inf)
    assert np.array_equal(o, ref, equal_nan=True)
    from oracle import confkv_oracle as O
    assert math.isnan(conf[1].item()) and sel[1].item() == 0
    assert abs(conf[2].item() - O.confidence(ref[2], tuple(float(np.float32(w)) for w in (0.4, 0.3, 0.3)))) < 1e-5
    kv.close()


def test_lengths_and_offsets_are_held_within_the_arrays(lib, torch_cuda):
    """Lengths beyond the row, negative ones, offsets that run backwards or out of the list: no entry outside is read."""
    torch = torch_cuda
    B, V, n = 4, 500, 12
    c = _case(B, V, n, 20, seed=4)
    kv = _kv(lib, B, V)
    x = torch.from_numpy(c["logits"]).cuda()
    out = torch.empty(B, V, device="cuda")
    c["lengths"] = np.array([-3, 2 ** 31 - 1, n + 1, 5], np.int32)
    c["prompt_lengths"] = np.array([4, -7, 2 ** 31 - 1, 9], np.int32)
    c["bias_offsets"] = np.array([-5, 6, 3, 2 ** 31 - 1, 2 ** 31 - 1], np.int32)
    kv.constrain(x, out, **_device(torch, c))
    torch.cuda.synchronize()
    held = dict(c, lengths=np.clip(c["lengths"], 0, n), prompt_lengths=np.clip(c["prompt_lengths"], 0, n))
    held["bias_offsets"] = np.array([0, 6, 3, 20, 20], np.int32)
    _check(out.cpu().numpy(), *_expected(held, c["logits"]), "held")
    kv.close()


def test_refusals(lib, torch_cuda):
    torch = torch_cuda
    B, V = 2, 100
    kv = _kv(lib, B, V)
    x, out = torch.zeros(B, V, device="cuda"), torch.zeros(B, V, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    f = torch.ones(B, device="cuda")
    from paper_2605_24786_amd import binding as b
    room = torch.zeros(B * V + 4, device="cuda")
    for args, kw in (((room[:B * V].view(B, V), room[4:].view(B, V)), {}),            # overlapping, not the same
                     ((x.half(), out), dict(tokens=torch.zeros(B, 3, dtype=torch.int32, device="cuda"), repetition=f)),  # no lengths
                     ((x, out), dict(allowed=torch.zeros(1, 4, dtype=torch.int32, device="cuda"))),                      # too few masks
                     ((x, out), dict(bias_offsets=i32(0, 1, 2), bias_tokens=i32(1, 2)))):                                # no values
        with pytest.raises(lib.ConfKVError) as e:
            kv.constrain(*args, **kw)
        assert e.value.status == b.ERR_INVALID_ARG
    for args, kw in (((x[:, :50], out), {}), ((x.double(), out), {}), ((x, out.half()), {}), ((x, out[:1]), {}), ((x.cpu(), out), {}),
                     ((x.t().contiguous().t(), out), {}), ((x, out), dict(repetition=f)), ((x, out), dict(tokens=i32(1, 2))),
                     ((x, out), dict(tokens=i32(1, 2).view(2, 1), lengths=i32(1), repetition=f)),
                     ((x, out), dict(allowed=torch.zeros(2, 3, dtype=torch.int32, device="cuda"))),
                     ((x, out), dict(bias_offsets=i32(0, 1)))):
        with pytest.raises(ValueError):
            kv.constrain(*args, **kw)
    kv.close()


def test_parts_that_would_do_nothing_are_refused(lib, torch_cuda):
    """Half a list of biases, a choice among no masks, more biases than indexes are made for."""
    torch = torch_cuda
    B, V = 2, 100
    kv = _kv(lib, B, V)
    x, out = torch.zeros(B, V, device="cuda"), torch.zeros(B, V, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    offsets, ids, values = i32(0, 1, 2), i32(1, 2), torch.ones(2, device="cuda")
    for kw in (dict(bias_tokens=ids, bias_values=values), dict(bias_offsets=offsets), dict(bias_values=values),
               dict(bias_offsets=offsets, bias_values=values), dict(allowed_rows=i32(0, 1))):
        with pytest.raises(ValueError):
            kv.constrain(x, out, **kw)
    from paper_2605_24786_amd import binding as b
    args = b._CONSTRAINTS.pack(b.TYPE_FP32, 0, x.data_ptr(), V, out.data_ptr(), 0, 0, 0, 0, 0, 0, 0, offsets.data_ptr(), ids.data_ptr(),
                               values.data_ptr(), 2 ** 30 + 1, 0, 0, 0)
    assert kv.lib.conf_kv_constrain(kv.h, args, kv._stream()) == b.ERR_INVALID_ARG
    kv.close()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("B,V", [(1, 4094), (1, 4095), (3, 4094), (5, 4095), (2, 8190), (1, 8191), (3, 8191), (1, 32767), (2, 32768),
                                 (40, 32766), (1, 131072), (33, 122879), (256, 20479)])
def test_vocabularies_that_end_at_a_range(lib, torch_cuda, dtype, B, V):
    """Rows that end where a workgroup's range does or one to three logits ahead of it, the result on a 16-byte boundary and one,
    two and three places behind it; histories and biases that name the first and the last tokens."""
    torch = torch_cuda
    print(f"constrain {dtype} B={B} V={V}", flush=True)
    c = _case(B, V, 60, 3 * B, seed=V + B, masks=2 if B == 2 else None)
    c["tokens"][:, 10:14], c["tokens"][:, 14:18] = np.arange(4), V - 1 - np.arange(4)
    c["lengths"][:] = 60
    c["prompt_lengths"] = np.full(B, 12, np.int32)
    c["bias_offsets"] = 3 * np.arange(B + 1, dtype=np.int32)
    c["bias_tokens"][0::3], c["bias_tokens"][1::3] = 0, V - 1
    x = torch.from_numpy(c["logits"]).to(getattr(torch, dtype)).cuda()
    ref, size = _expected(c, x.float().cpu().numpy())
    kv = _kv(lib, B, V)
    kw = _device(torch, c)
    for places in range(4):
        room = torch.full((B * V + 8,), 9.0, device="cuda")
        out = room[places:places + B * V].view(B, V)
        kv.constrain(x, out, **kw)
        torch.cuda.synchronize()
        _check(out.cpu().numpy(), ref, size, f"{places} places behind a boundary")
        assert bool((room[:places] == 9).all()) and bool((room[places + B * V:] == 9).all())
    kv.close()

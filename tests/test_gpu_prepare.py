"""conf_kv_prepare_qkv against the formulas in 64 bits.

Tolerance per value, from the arithmetic: the rounding to fp16 is off by at most 2^-11 of the value (2^-25 below fp16's normal
range); ahead of it stand the norm (the sum of up to 128 squares, a square root, a division and two products: under 2^-20
relative), the angle (formed in float64; as a fraction of a turn held in float32, off by 2^-26 turns = 9.4e-8 rad), sine and
cosine (2 ulp) and three float32 operations, all together under 2^-19 of |a| + |b| for a pair (a, b)."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch_cuda():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


def _kv(lib, B=1, Hq=8, Hkv=2, D=128, **kw):
    base = dict(n_layers=2, batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, vocab=100, capacity=64, fp16_window=16,
                protected_window=8, n_tight=[16, 16], n_loose=[32, 32])
    return lib.ConfKV(**dict(base, **kw))


def _reference(torch, x, w, freq, pos, interleaved, eps):
    """(values, |a| + |b| of each value's pair) in float64 on the CPU."""
    x = x.detach().cpu().double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.cpu().double()
    y, size = x.clone(), x.abs()
    if freq is not None and freq.numel():
        n = freq.numel()
        t = (pos.cpu().double()[..., None] * freq.cpu().double())[:, :, None]
        ia = torch.arange(0, 2 * n, 2) if interleaved else torch.arange(n)
        ib = ia + 1 if interleaved else ia + n
        a, b = x[..., ia], x[..., ib]
        y[..., ia] = a * t.cos() - b * t.sin()
        y[..., ib] = b * t.cos() + a * t.sin()
        size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return y, size


def _close(torch, got, ref, size, what):
    got = got.cpu().double()
    err, tol = (got - ref).abs(), ref.abs() * 2.0 ** -11 + 2.0 ** -25 + size * 2.0 ** -19
    assert bool((err <= tol).all()), f"{what}: {(err / tol).max().item():.3g} x tolerance"


def _run(torch, lib, B, T, Hq, Hkv, D, dtype, rotated, interleaved, prompt, norm, fused=True, far=1000, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    rows = (scale * torch.randn(B, T, Hq + 2 * Hkv, D, generator=g)).to(dtype).cuda()
    q, k, v = rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    wq = (1 + 0.3 * torch.randn(D, generator=g)).cuda() if norm in ("q", "both") else None
    wk = (1 + 0.3 * torch.randn(D, generator=g)).cuda() if norm in ("k", "both") else None
    freq = (10000.0 ** (-torch.arange(rotated // 2).double() / max(1, rotated // 2))).float().cuda() if rotated else None
    pos = torch.randint(-5, far, (B, T), generator=g, dtype=torch.int32).cuda()
    kv = _kv(lib, B, Hq, Hkv, D)
    q16 = torch.full((B, T, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    shape = (B, Hkv, T, D) if prompt else (B, T, Hkv, D)
    k16, v16 = (torch.full(shape, 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    eps = 1e-5
    kv.prepare_qkv(1, q, k, v, q16, k16, v16, freq=freq, pos=pos, q_weight=wq, k_weight=wk, eps=eps, interleaved=interleaved,
                   prompt=prompt)
    torch.cuda.synchronize()
    back = (lambda x: x.transpose(1, 2)) if prompt else (lambda x: x)
    _close(torch, q16, *_reference(torch, q, wq, freq, pos, interleaved, eps), "queries")
    _close(torch, back(k16), *_reference(torch, k, wk, freq, pos, interleaved, eps), "keys")
    assert torch.equal(back(v16), v.float().half()), "values"
    kv.close()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,rotated,interleaved,prompt,norm", [
    (1, 1, 8, 2, 128, 128, False, False, None),
    (1, 1, 8, 2, 128, 128, True, False, "both"),
    (3, 1, 10, 2, 128, 64, False, False, "q"),          # rows that fill no pass of a wavefront
    (2, 5, 3, 3, 64, 64, False, True, "both"),
    (2, 33, 12, 12, 64, 16, True, True, "k"),
    (1, 17, 16, 1, 128, 112, False, True, "both"),      # one kv-head, sixteen query heads
    (1, 70, 7, 7, 64, 48, False, False, None),
    (2, 3, 8, 8, 128, 0, False, True, "both"),          # nothing turns
    (2, 3, 8, 8, 128, 16, True, False, None),
    (1, 4099, 4, 2, 64, 32, False, True, "both"),       # enough wavefronts for one per token
    (2, 2050, 4, 2, 128, 128, False, True, "both"),     # streaming accesses of whole lines
    (3, 1400, 9, 3, 128, 64, True, False, "q"),
])
def test_rows_match_the_formulas(lib, torch_cuda, dtype, B, T, Hq, Hkv, D, rotated, interleaved, prompt, norm):
    torch = torch_cuda
    print(f"prepare {dtype} B={B} T={T} heads {Hq}/{Hkv} D={D} rotated={rotated} {norm}", flush=True)
    _run(torch, lib, B, T, Hq, Hkv, D, getattr(torch, dtype), rotated, interleaved, prompt, norm, seed=T + D)
    _run(torch, lib, B, T, Hq, Hkv, D, getattr(torch, dtype), rotated, interleaved, prompt, norm, fused=False, seed=T)


def test_far_positions(lib, torch_cuda):
    """Angles of positions up to 2^31 - 6: their product with a frequency of 1 is exact in float64 and reduced there."""
    torch = torch_cuda
    _run(torch, lib, 2, 9, 8, 2, 128, torch.float32, 128, False, False, "both", far=2 ** 31 - 6, seed=3)


def test_positions_of_the_handle(lib, torch_cuda):
    """Without positions, token t has the place the layer's next appended token gets, plus t, plus `first`."""
    torch = torch_cuda
    B, Hq, Hkv, D, T, T0 = 2, 8, 2, 128, 3, 11
    g = torch.Generator().manual_seed(5)
    kv = _kv(lib, B, Hq, Hkv, D)
    kv.load_prefill(1, *(torch.randn(B, Hkv, T0, D, generator=g).half().cuda() for _ in range(2)))
    q = torch.randn(B, T, Hq, D, generator=g).half().cuda()
    freq = (100.0 ** (-torch.arange(64) / 64.0)).float().cuda()
    outs = [torch.empty_like(q) for _ in range(2)]
    for layer, first, start in ((1, 0, T0), (1, 4096, T0 + 4096), (0, -2, -2)):
        kv.prepare_qkv(layer, q, None, None, outs[0], freq=freq, first=first)
        pos = (start + torch.arange(T, dtype=torch.int32)).repeat(B, 1).cuda()
        kv.prepare_qkv(layer, q, None, None, outs[1], freq=freq, pos=pos)
        torch.cuda.synchronize()
        assert torch.equal(*outs)
        _close(torch, outs[0], *_reference(torch, q, None, freq, pos, False, 0.0), f"layer {layer}")
    kv.close()


def test_values_at_the_edges(lib, torch_cuda):
    """Beyond fp16's range: infinite, as a conversion gives; a row of zeros stays zero under the norm; a NaN stays in its row,
    and in its pair where there is no norm."""
    torch = torch_cuda
    B, T, Hq, Hkv, D = 1, 2, 4, 2, 128
    kv = _kv(lib, B, Hq, Hkv, D)
    x = torch.randn(B, T, Hq, D, generator=torch.Generator().manual_seed(1)).cuda()
    x[0, 0, 0, 3], x[0, 0, 1], x[0, 1, 2, 5], x[0, 1, 3, 100] = 1e6, 0.0, math.nan, math.inf
    pos, freq = torch.zeros(B, T, dtype=torch.int32, device="cuda"), torch.ones(16, device="cuda")
    out = torch.empty(B, T, Hq, D, dtype=torch.float16, device="cuda")
    kv.prepare_qkv(0, x, None, None, out, freq=freq, pos=pos)
    torch.cuda.synchronize()
    o = out.cpu()
    bad = torch.zeros(B, T, Hq, D, dtype=torch.bool)
    bad[0, 1, 2, 5] = bad[0, 1, 2, 21] = True
    assert torch.equal(o.isnan(), bad)
    assert torch.equal(o.isinf().nonzero(), torch.tensor([[0, 0, 0, 3], [0, 1, 3, 100]]))
    kv.prepare_qkv(0, x, None, None, out, freq=freq, pos=pos, q_weight=torch.ones(D, device="cuda"))
    torch.cuda.synchronize()
    o = out.cpu()
    assert bool((o[0, 0, 1] == 0).all()) and bool(o[0, 1, 2].isnan().all()) and o[0, 1, 3].isnan().sum() == 1
    assert bool(o[0, 0].isfinite().all())
    kv.close()


def test_parts_can_be_left_out_and_nothing_else_is_written(lib, torch_cuda):
    torch = torch_cuda
    B, T, Hq, Hkv, D = 2, 3, 8, 2, 64
    kv = _kv(lib, B, Hq, Hkv, D)
    k = torch.randn(B, T, Hkv, D, device="cuda").bfloat16()
    room = torch.full((4, B, Hkv, T, D), 3.0, dtype=torch.float16, device="cuda")
    kv.prepare_qkv(0, None, k, None, k16=room[1], prompt=True)
    kv.prepare_qkv(0, None, None, k, v16=room[2].view(B, T, Hkv, D))
    torch.cuda.synchronize()
    assert torch.equal(room[1], k.half().transpose(1, 2)) and torch.equal(room[2].view(B, T, Hkv, D), k.half())
    assert bool((room[0] == 3).all()) and bool((room[3] == 3).all())
    empty = k[:, :0]
    kv.prepare_qkv(0, None, empty, None, k16=room[3, :, :, :0], prompt=True)
    kv.close()


def test_refusals(lib, torch_cuda):
    torch = torch_cuda
    B, T, Hq, Hkv, D = 2, 3, 8, 2, 64
    kv = _kv(lib, B, Hq, Hkv, D)
    q = torch.randn(B, T, Hq, D, device="cuda").half()
    out = torch.empty_like(q)
    f = torch.ones(D // 2, device="cuda")

    def status(layer=0, **kw):
        with pytest.raises(lib.ConfKVError) as e:
            kv.prepare_qkv(layer, q, None, None, kw.pop("q16", out), **kw)
        return e.value.status

    from paper_2605_24786_amd import binding as b
    assert status(layer=2) == b.ERR_BAD_LAYER and status(layer=-1) == b.ERR_BAD_LAYER
    assert status(freq=f[:4]) == b.ERR_INVALID_ARG                              # 8 channels
    assert status(freq=torch.ones(D, device="cuda")) == b.ERR_INVALID_ARG       # more than the head has
    w = torch.ones(D, device="cuda")
    for eps in (-1.0, math.nan, math.inf):
        assert status(q_weight=w, eps=eps) == b.ERR_INVALID_ARG
    assert status(q16=q) == b.ERR_INVALID_ARG                                   # in place
    room = torch.empty(2 * q.numel() + 8, dtype=torch.float16, device="cuda")
    at = room[4:4 + q.numel()].view_as(q)
    assert status(q16=at) == b.ERR_INVALID_ARG                                  # 8-byte alignment
    with pytest.raises(lib.ConfKVError):
        kv.prepare_qkv(0, q, None, None)                                        # a source without a destination
    with pytest.raises(lib.ConfKVError):
        kv.prepare_qkv(0, torch.as_strided(room, q.shape, (T * Hq * D + 4, Hq * D, D, 1)), None, None, out)
    for bad in (dict(q16=out.float()), dict(q16=out[:, :2]), dict(pos=torch.zeros(B, T, device="cuda")), dict(freq=f.double()),
                dict(q_weight=w[:8]), dict(q16=out.cpu())):
        with pytest.raises(ValueError):
            kv.prepare_qkv(0, q, None, None, **dict(dict(q16=out), **bad))
    for bad in (q.double(), q[:, :, :4], q.transpose(2, 3), q.cpu(), q[0]):
        with pytest.raises(ValueError):
            kv.prepare_qkv(0, bad, None, None, out)
    with pytest.raises(ValueError):
        kv.prepare_qkv(0, None, None, None)
    kv.close()


def test_destinations_that_overlap_are_refused(lib, torch_cuda):
    torch = torch_cuda
    B, T, H, D = 2, 3, 2, 64
    kv = _kv(lib, B, H, H, D)
    q, k, v = torch.randn(3, B, T, H, D, device="cuda").half()
    n = q.numel()
    room = torch.empty(3 * n, dtype=torch.float16, device="cuda")
    at = lambda i: room[i:i + n].view(B, T, H, D)
    from paper_2605_24786_amd import binding as b
    for places in ((0, 0, n), (0, n, n), (0, n, 2 * n - 8), (8, 0, 2 * n)):
        with pytest.raises(lib.ConfKVError) as e:
            kv.prepare_qkv(0, q, k, v, *(at(i) for i in places))
        assert e.value.status == b.ERR_INVALID_ARG
    kv.prepare_qkv(0, q, k, v, at(2 * n), at(0), at(n))                         # side by side
    for i, x in ((2 * n, q), (0, k), (n, v)):
        assert torch.equal(at(i), x)
    kv.close()


def test_more_tokens_than_a_grid_dimension(lib, torch_cuda):
    """2^26 + 13 tokens, one wavefront each: more threads than one dimension of a launch has.  Every token reads the same row; keys at
    the handle's positions, sampled, and all values."""
    torch = torch_cuda
    T, D = 2 ** 26 + 13, 64
    kv = _kv(lib, 1, 1, 1, D)
    row = torch.randn(2, D, generator=torch.Generator().manual_seed(6)).half().cuda()
    k, v = (r.view(1, 1, 1, D).expand(1, T, 1, D) for r in row)
    freq = (100.0 ** (-torch.arange(32) / 32.0)).float().cuda()
    k16, v16 = (torch.zeros(1, T, 1, D, dtype=torch.float16, device="cuda") for _ in range(2))
    kv.prepare_qkv(0, None, k, v, k16=k16, v16=v16, freq=freq)
    torch.cuda.synchronize()
    for part in v16.view(T, D).split(2 ** 23):
        assert bool((part == row[1]).all())
    at = torch.tensor([0, 1, 2 ** 23 * 4 - 1, 2 ** 23 * 4, 2 ** 25 + 5, 2 ** 26 - 1, 2 ** 26, T - 2, T - 1])
    _close(torch, k16[:, at.cuda()], *_reference(torch, k[:, at.cuda()], None, freq, at[None].int(), False, 0.0), "keys")
    kv.close()


@pytest.mark.parametrize("c", [1, 3])
def test_positions_of_the_handle_behind_an_append(lib, torch_cuda, c):
    """Between the attention, which appends, and conf_kv_evict_compact, which ends the step, the next appended token is the one behind
    the call's own -- recorded as well."""
    torch = torch_cuda
    B, Hq, Hkv, D, T, T0 = 2, 8, 2, 128, 2, 11
    g = torch.Generator().manual_seed(5)
    kv = _kv(lib, B, Hq, Hkv, D, max_chunk=4)
    for layer in (0, 1):
        kv.load_prefill(layer, *(torch.randn(B, Hkv, T0, D, generator=g).half().cuda() for _ in range(2)))
    q = torch.randn(B, T, Hq, D, generator=g).half().cuda()
    freq = (100.0 ** (-torch.arange(64) / 64.0)).float().cuda()
    q16, before, behind, other, ref = (torch.zeros_like(q) for _ in range(5))
    new = [torch.randn(B, c, h, D, generator=g).half().cuda() for h in (Hq, Hkv, Hkv)]
    out = torch.empty_like(new[0])

    def calls():
        kv.prepare_qkv(0, q, None, None, before, freq=freq, first=7)
        kv.attend_chunk(0, *new, out)
        kv.prepare_qkv(0, q, None, None, behind, freq=freq, first=7)
        kv.prepare_qkv(1, q, None, None, other, freq=freq, first=7)
        kv.attend_chunk(1, *new, out)
        kv.evict_compact()

    def check(steps):
        torch.cuda.synchronize()
        at = T0 + c * steps
        for got, start in ((before, at), (behind, at + c), (other, at)):
            pos = (start + 7 + torch.arange(T, dtype=torch.int32)).repeat(B, 1).cuda()
            kv.prepare_qkv(0, q, None, None, ref, freq=freq, pos=pos)
            torch.cuda.synchronize()
            assert torch.equal(got, ref), steps

    kv.static_plan(True)
    calls()
    check(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(1, 5):
        graph.replay()
        check(i)
    kv.close()


@pytest.mark.parametrize("D,interleaved", [(128, False), (64, True)])
@pytest.mark.parametrize("dtype,scale", [("float32", 1e25), ("float32", 3e37), ("float32", 1e-30), ("float32", 1e-38), ("bfloat16", 1e30),
                                         ("bfloat16", 1e-25), ("float16", 2e-7), ("float16", 1.2e4)])
def test_norm_of_rows_whose_squares_leave_float32(lib, torch_cuda, dtype, scale, D, interleaved):
    """Rows so large or small that the sum of their squares is no float32 number, beside ordinary ones and one of zeros: what the norm
    makes of them is of the size of its weight (eps: 0 for the small ones, which it would drown)."""
    torch = torch_cuda
    B, T, Hq, Hkv = 1, 3, 6, 2
    g = torch.Generator().manual_seed(9)
    size = torch.tensor([scale, 1.0, 1.0, scale, 1.0, scale])[:, None]
    q = (torch.randn(B, T, Hq, D, generator=g).clamp(-5, 5) * size).to(getattr(torch, dtype)).cuda()
    k = (torch.randn(B, T, Hkv, D, generator=g).clamp(-5, 5) * scale).to(getattr(torch, dtype)).cuda()
    eps = 1e-5 if scale > 1 else 0.0
    if eps:
        q[0, 1, 4] = 0
    w = (1 + 0.3 * torch.randn(2, D, generator=g)).cuda()
    freq = (100.0 ** (-torch.arange(D // 2) / (D / 2))).float().cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    kv = _kv(lib, B, Hq, Hkv, D)
    q16 = torch.empty(B, T, Hq, D, dtype=torch.float16, device="cuda")
    k16 = torch.empty(B, T, Hkv, D, dtype=torch.float16, device="cuda")
    kv.prepare_qkv(0, q, k, None, q16, k16, freq=freq, pos=pos, q_weight=w[0], k_weight=w[1], eps=eps, interleaved=interleaved)
    torch.cuda.synchronize()
    _close(torch, q16, *_reference(torch, q, w[0], freq, pos, interleaved, eps), "queries")
    _close(torch, k16, *_reference(torch, k, w[1], freq, pos, interleaved, eps), "keys")
    kv.close()

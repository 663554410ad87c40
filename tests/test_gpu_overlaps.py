"""Tensors that a call writes and that share memory with what it reads or writes elsewhere are refused, whatever small part they share;
neighbours in one allocation are not."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return torch


@pytest.mark.parametrize("tq", [1, 2])
def test_output_of_differences_inside_its_inputs(lib, torch, tq):
    B, H, G, D = 3, 2, 4, 128
    kv = lib.ConfKV(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=100, capacity=64, fp16_window=16,
                    protected_window=16, n_tight=[32], n_loose=[32], max_chunk=tq if tq > 1 else 0)
    sizes = dict(q=B * tq * G * H * D, k=B * tq * H * D, v=B * tq * H * D, lam=2 * B * tq * G * H // 2)
    shapes = dict(q=(B, tq, G * H, D), k=(B, tq, H, D), v=(B, tq, H, D), lam=(B, tq, G * H // 2))
    n_out = B * tq * G * H // 2 * D

    def call(name, shift):
        """The output `shift` values behind the first value of the input (negative: in front of it)."""
        room = torch.zeros(sizes[name] + 2 * n_out, dtype=torch.float16, device="cuda")
        at = {n: torch.zeros(s, dtype=torch.float16, device="cuda") for n, s in sizes.items()}
        at[name] = room[n_out:n_out + sizes[name]]
        out = room[n_out + shift:][:n_out].view(B, tq, G * H // 2, D)
        t = {n: (x.view(torch.float32) if n == "lam" else x).view(shapes[n]) for n, x in at.items()}
        kv.attend_diff(0, t["q"], t["k"], t["v"], out, t["lam"])
    for name, size in sizes.items():
        for shift in (0, size - 8, 8 - n_out, (8 - n_out) // 16 * 8):
            with pytest.raises(lib.ConfKVError) as e:
                call(name, shift)
            assert e.value.status == lib.binding.ERR_INVALID_ARG, (name, shift)
        for shift in (size, -n_out):
            call(name, shift)
            kv.evict_compact()
    # weights that all tokens share, and weights far apart
    out = torch.zeros(B, tq, G * H // 2, D, dtype=torch.float16, device="cuda")
    q, k, v = (torch.zeros(shapes[n], dtype=torch.float16, device="cuda") for n in "qkv")
    far = torch.zeros(B * tq, 4096, device="cuda")
    for lam in (torch.zeros(G * H // 2, device="cuda"), far.view(B, tq, 4096)[:, :, 1:1 + G * H // 2]):
        kv.attend_diff(0, q, k, v, out, lam)
        kv.evict_compact()
    with pytest.raises(lib.ConfKVError):
        kv.attend_diff(0, q, k, v, out, out.view(torch.float32).reshape(-1)[64:64 + G * H // 2])
    assert kv.counters().device_errors == 0
    kv.close()


def test_planes_of_pages_that_share_some_values(lib, torch):
    """Keys and values may take turns in one tensor; where a row of one reaches into a row of the other they are refused, unless
    nothing is written."""
    B, H, G, D, page, n = 2, 2, 2, 128, 16, 6
    kv = lib.ConfKV(n_layers=1, batch=B, n_q_heads=G * H, n_kv_heads=H, head_dim=D, vocab=100, capacity=64, fp16_window=16,
                    protected_window=16, n_tight=[32], n_loose=[32], max_paged=4 * page)
    t = lambda *s, d=torch.float16: torch.zeros(s, dtype=d, device="cuda")
    q, k, v, out = t(B, 2, G * H, D), t(B, 2, H, D), t(B, 2, H, D), t(B, 2, G * H, D)
    table, context = t(B, 4, d=torch.int32), t(B, d=torch.int32)
    table[1] = 4
    plane = page * H * D
    room = t(4 * n * plane)
    for strides, turn in (((2 * plane, H * D, D), plane), ((2 * plane, 2 * H * D, D), H * D), ((2 * plane, 2 * H * D, 2 * D), D),
                          ((plane, H * D, D), n * plane)):
        view = lambda at: room[at:].as_strided((n, page, H, D), strides + (1,), room.storage_offset() + at)
        kv.attend_pages(q, k, v, out, view(0), view(turn), table, context)
        kv.attend_pages(q, k, v, out, view(turn), view(0), table, context)
        for off in (0, 8, turn - 8, turn - D + 8):
            for pair in ((0, off), (off, 0)):
                with pytest.raises(lib.ConfKVError) as e:
                    kv.attend_pages(q, k, v, out, *(view(x) for x in pair), table, context)
                assert e.value.status == lib.binding.ERR_INVALID_ARG
                kv.attend_pages(q, None, None, out, *(view(x) for x in pair), table, context)
    kv.close()

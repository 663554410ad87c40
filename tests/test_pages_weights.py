"""How the binding finds the weights of the second maps in tensors as a projection leaves them, on a machine without a GPU."""
import pytest
import torch

import paper_2605_24786_amd as pkg


@pytest.fixture
def weights():
    kv = pkg.ConfKV.__new__(pkg.ConfKV)
    kv._f32, kv._device, kv.state, kv.h = torch.float32, -1, torch.empty(0), None
    return kv._weights


def _rows(lam, at, apart, shape):
    """What the call reads: `shape` rows, `apart` values from one to the next."""
    flat = torch.empty(0).set_(lam.untyped_storage())
    first = (at - flat.data_ptr()) // 4
    n = 1
    for s in shape[:-1]:
        n *= s
    return torch.stack([flat[first + i * apart:first + i * apart + shape[-1]] for i in range(n)]).reshape(shape)


@pytest.mark.parametrize("B,T,pairs", [(3, 5, 4), (1, 5, 4), (3, 1, 4), (1, 1, 2), (2, 7, 1)])
def test_slices_are_taken_as_they_are(weights, B, T, pairs):
    wide = torch.randn(B, T, 3 * pairs + 2)
    for shape in ((B, T, pairs), (B * T, pairs)):
        rows = wide.reshape(shape[:-1] + (-1,))
        for lam in (rows[..., :pairs], rows[..., pairs + 1:2 * pairs + 1], rows[..., :pairs].contiguous()):
            assert torch.equal(_rows(lam, *weights(lam, shape), shape), lam)
        lam = rows.flatten()[:pairs]
        assert weights(lam, shape) == (lam.data_ptr(), 0)
        same = lam.expand(shape)
        assert torch.equal(_rows(same, *weights(same, shape), shape), same)


def test_others_are_refused(weights):
    wide = torch.randn(3, 5, 16)
    for lam, shape in ((wide[:, :, ::2], (3, 5, 8)), (wide[:, :4, :8], (3, 4, 8)), (wide.transpose(0, 1)[..., :8], (5, 3, 8)),
                       (wide[..., :8], (3, 5, 4)), (wide[..., :8].double(), (3, 5, 8)), (wide[0, :, :8], (3, 5, 8)), (wide[0, 0, 0], (3, 5, 1)),
                       (wide[:, :, :8].flatten(0, 1)[:14], (15, 8)), (wide[:1, :, :8].expand(3, 5, 8), (3, 5, 8)), (wide[0, 0, ::2], (3, 5, 8))):
        with pytest.raises(ValueError):
            weights(lam, shape)
    assert weights(wide[:1, :4, :8], (1, 4, 8))[1] == 16

"""Pins of the normalisation's and the embedding's oracle: torch in fp64 with autograd, central differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import model_ops_oracle as orc


@pytest.mark.parametrize("rms", [False, True])
def test_norm_matches_torch_autograd_and_differences(rms):
    g = torch.Generator().manual_seed(1)
    h = torch.randn(5, 12, generator=g, dtype=torch.float64) + 0.4
    w, b = torch.randn(12, generator=g, dtype=torch.float64), torch.randn(12, generator=g, dtype=torch.float64)
    dy, dh = torch.randn(5, 12, generator=g, dtype=torch.float64), torch.randn(5, 12, generator=g, dtype=torch.float64)
    for t in (h, w, b):
        t.requires_grad_(True)
    if rms:
        y = h / (h.square().mean(1, keepdim=True) + 1e-3).sqrt() * w + b
    else:
        y = torch.nn.functional.layer_norm(h, (12,), w, b, eps=1e-3)
    ((y * dy).sum() + (h * dh).sum()).backward()
    got, mean, rstd = orc.norm_forward(h.detach().numpy(), w.detach().numpy(), b.detach().numpy(), rms, 1e-3)
    assert np.abs(got - y.detach().numpy()).max() < 1e-13
    dx, dw, db = orc.norm_backward(dy.numpy(), h.detach().numpy(), w.detach().numpy(), mean, rstd, dh.numpy(), rms)
    for a, t in ((dx, h), (dw, w), (db, b)):
        assert np.abs(a - t.grad.numpy()).max() < 1e-12
    f = lambda x: float((orc.norm_forward(x, w.detach().numpy(), None, rms, 1e-3)[0] * dy.numpy()).sum() + (x * dh.numpy()).sum())
    x, step = h.detach().numpy().copy(), 1e-5
    for i, j in ((0, 0), (2, 7), (4, 11)):
        up, down = x.copy(), x.copy()
        up[i, j] += step
        down[i, j] -= step
        assert abs((f(up) - f(down)) / (2 * step) - dx[i, j]) < 1e-7


def test_norm_of_a_constant_row_is_zero():
    y, mean, rstd = orc.norm_forward(np.full((1, 7), 3.0), eps=0.25)
    assert (y == 0).all() and mean[0] == 3.0 and rstd[0] == 2.0


def test_embedding_is_a_product_with_one_hot_rows():
    rng = np.random.default_rng(2)
    table, ids = rng.normal(size=(6, 4)), np.array([3, 3, -1, 0, 6, 5, 3])
    hot = np.zeros((7, 6))
    for t, v in enumerate(ids):
        if 0 <= v < 6:
            hot[t, v] = 1.0
    assert np.allclose(orc.embed_forward(table, ids, 0.5), 0.5 * hot @ table, atol=1e-15)
    dout, start = rng.normal(size=(7, 4)), rng.normal(size=(6, 4))
    assert np.allclose(orc.embed_backward(dout, ids, 6, 0.5), 0.5 * hot.T @ dout, atol=1e-14)
    assert np.allclose(orc.embed_backward(dout, ids, 6, 0.5, start), start + 0.5 * hot.T @ dout, atol=1e-14)

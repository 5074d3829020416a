"""Pins of the oracle's layer norm and AdamW: torch's double-precision modules, central differences, worked numbers, and the
8-bit format against torch's."""

import numpy as np
import pytest
import torch

from oracle import dense as od
from oracle import negatives


def test_layer_norm_by_hand():
    # 1 2 3 4: mean 2.5, var 1.25; eps 0.31 makes 1 / sqrt(var + eps) = 1 / 1.249 ... use eps = 1: 1 / 1.5
    y, mean, rstd = od.layer_norm([[1.0, 2.0, 3.0, 4.0]], [1.0, 2.0, 1.0, 1.0], [0.0, 0.0, 10.0, 0.0], 1.0)
    assert mean[0] == 2.5 and rstd[0] == pytest.approx(1 / 1.5)
    assert y[0] == pytest.approx([-1.0, -2 / 3, 10 + 1 / 3, 1.0])


@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_against_torch_in_double(affine):
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((7, 33)) * 3 + 1, rng.standard_normal((7, 33))
    w, b = (rng.standard_normal(33), rng.standard_normal(33)) if affine else (None, None)
    tx = torch.tensor(x, requires_grad=True)
    tw = torch.tensor(w, requires_grad=True) if affine else None
    tb = torch.tensor(b, requires_grad=True) if affine else None
    ty = torch.nn.functional.layer_norm(tx, (33,), tw, tb, 1e-5)
    ty.backward(torch.tensor(dy))
    y, mean, rstd = od.layer_norm(x, w, b, 1e-5)
    dx, dw, db = od.layer_norm_backward(x, dy, mean, rstd, w)
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=1e-10, atol=1e-12)
    if affine:
        np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=1e-12, atol=1e-13)
        np.testing.assert_allclose(db, tb.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(2)
    x, dy, w, b = rng.standard_normal((3, 6)), rng.standard_normal((3, 6)), rng.standard_normal(6), rng.standard_normal(6)
    loss = lambda x, w, b: float((od.layer_norm(x, w, b, 1e-3)[0] * dy).sum())  # noqa: E731
    _, mean, rstd = od.layer_norm(x, w, b, 1e-3)
    dx, dw, db = od.layer_norm_backward(x, dy, mean, rstd, w)
    h = 1e-6
    for a, grad, f in ((x, dx, lambda v: loss(v, w, b)), (w, dw, lambda v: loss(x, v, b)), (b, db, lambda v: loss(x, w, v))):
        for i in np.ndindex(a.shape):
            up, down = a.copy(), a.copy()
            up[i] += h
            down[i] -= h
            assert (f(up) - f(down)) / (2 * h) == pytest.approx(grad[i], abs=1e-8)


def test_adamw_against_torch_in_double():
    rng = np.random.default_rng(3)
    p0 = [rng.standard_normal(n) for n in (5, 300)]
    params = [torch.nn.Parameter(torch.tensor(p)) for p in p0]
    opt = torch.optim.AdamW([dict(params=[params[0]], weight_decay=0.1), dict(params=[params[1]], weight_decay=0.0)], lr=0.02, betas=(0.8, 0.95), eps=1e-6)
    p, m, v = [x.copy() for x in p0], [np.zeros_like(x) for x in p0], [np.zeros_like(x) for x in p0]
    for t in range(1, 8):
        g = [rng.standard_normal(x.shape) for x in p0]
        for q, x in zip(params, g):
            q.grad = torch.tensor(x)
        assert od.gradient_norm(g) == pytest.approx(float(torch.nn.utils.clip_grad_norm_(params, 3.0)), rel=1e-12)
        f = od.clip_factor(od.gradient_norm(g), 3.0)
        opt.step()
        for k in range(2):
            p[k], m[k], v[k] = od.adamw(p[k], g[k] * f, m[k], v[k], t, lr=0.02, beta1=0.8, beta2=0.95, eps=1e-6, weight_decay=(0.1, 0.0)[k])
            np.testing.assert_allclose(p[k], params[k].detach().numpy(), rtol=1e-10, atol=1e-13)


def test_codes_are_torchs_e4m3():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = od.e4m3_values()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_neighbouring_codes():
    values = np.sort(np.unique(np.abs(od.e4m3_values()[~np.isnan(od.e4m3_values())])))
    x = np.concatenate([values, (values[:-1] + values[1:]) / 2, [0.3 * od.LEAST]])
    x = np.concatenate([x, np.full(-len(x) % od.BLOCK, 448.0)])
    x[:: od.BLOCK] = 448.0                                   # scale 1 in every block
    low, step, share = od.rounded_up_share(x, od.block_scales(x), False)
    assert np.all(np.isin(low, values)) and np.all((share >= 0) & (share < 1))
    below = share > 0
    assert np.all(np.isin((low + step)[below], values)) and np.allclose(low + share * step, x)
    low, _, share = od.rounded_up_share(x, od.block_scales(x), True)
    assert np.all((low >= od.LEAST) | (x == 0))


def test_words_are_uniform_and_differ_by_step_and_tensor():
    a, b, c = od.random_words(7, 3, 0, 1 << 16), od.random_words(7, 4, 0, 1 << 16), od.random_words(7, 3, 1, 1 << 16)
    for w in (a, b, c):
        for bits in ((w >> np.uint64(12)) / 2.0**20, (w & np.uint64(0xFFFF)) / 2.0**16):
            hist = np.histogram(bits, 64, (0, 1))[0]
            assert ((hist - 1024.0) ** 2 / 1024.0).sum() < 63 + 5 * np.sqrt(2 * 63)
        # the two fractions of a word do not go together
        u, v = (w >> np.uint64(12)) / 2.0**20, (w & np.uint64(0xFFFF)) / 2.0**16
        assert abs(np.corrcoef(u, v)[0, 1]) < 5 / 256
    for x, y in ((a, b), (a, c)):
        assert abs(np.corrcoef(x.astype(float), y.astype(float))[0, 1]) < 5 / 256
    # the key is the library's counter hash
    k = int(negatives.fold(negatives.fold(np.uint64(7), 3), 0)) & 0xFFFFFFFF
    w = 5 ^ k
    w ^= w >> 16
    w = w * 0x9E3779B1 & 0xFFFFFFFF
    w ^= w >> 15
    w = w * 0x85157AF5 & 0xFFFFFFFF
    assert int(a[5]) == w ^ (w >> 16)
    far = od.random_words(7, 3, 0, 4, first=(1 << 32) - 2)
    assert len(set(far.tolist()) & set(a[:4].tolist())) == 0

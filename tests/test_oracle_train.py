"""The oracle of the retraining operators (oracle/train.py) against closed
forms, torch's fp64 autograd and differences (CPU)."""
import numpy as np
import pytest
import torch

from oracle import train


def _data(n, c, h, w, seed):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((n, c, h, w)), rng.standard_normal((n, c, h, w)), 1 + 0.3 * rng.standard_normal(c),
            0.3 * rng.standard_normal(c))


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape,groups", [((2, 6, 3, 5), 2), ((1, 4, 1, 2), 4), ((3, 5, 4, 1), 1)])
def test_group_norm_equals_torch_and_its_gradient(shape, groups, act):
    x, dy, gamma, beta = _data(*shape, 3)
    tx, tg, tb = (torch.tensor(t, requires_grad=True) for t in (x, gamma, beta))
    ty = torch.nn.functional.group_norm(tx, groups, tg, tb, 1e-5)
    ty = torch.relu(ty) if act == "relu" else torch.nn.functional.silu(ty) if act == "silu" else ty
    y, mean, rstd = train.group_norm(x, groups, gamma, beta, 1e-5, act)
    assert np.abs(y - ty.detach().numpy()).max() < 1e-12
    ty.backward(torch.tensor(dy))
    dx, dgamma, dbeta = train.group_norm_back(x, dy, groups, gamma, beta, mean, rstd, act)
    assert np.abs(dx - tx.grad.numpy()).max() < 1e-10
    assert np.abs(dgamma - tg.grad.numpy()).max() < 1e-11
    assert np.abs(dbeta - tb.grad.numpy()).max() < 1e-11


def test_group_norm_gradient_equals_differences():
    x, dy, gamma, beta = _data(1, 4, 2, 3, 5)
    loss = lambda t: float((train.group_norm(t, 2, gamma, beta, 1e-5, "silu")[0] * dy).sum())    # noqa: E731
    _, mean, rstd = train.group_norm(x, 2, gamma, beta, 1e-5, "silu")
    dx = train.group_norm_back(x, dy, 2, gamma, beta, mean, rstd, "silu")[0]
    for at in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[at] = 1e-6
        assert abs((loss(x + d) - loss(x - d)) / 2e-6 - dx[at]) < 1e-7


def test_adamw_equals_torch():
    rng = np.random.default_rng(1)
    p0 = rng.standard_normal(50)
    f = lambda x: float(np.float32(x))      # noqa: E731  (what the library is given)
    tp = torch.tensor(p0, requires_grad=True)
    opt = torch.optim.AdamW([tp], lr=f(1e-2), betas=(f(0.9), f(0.999)), eps=f(1e-8), weight_decay=f(0.1))
    p, m, v = p0, np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.standard_normal(50)
        tp.grad = torch.tensor(g)
        opt.step()
        p, m, v = train.adamw(p, g, m, v, t, 1e-2, 0.9, 0.999, 1e-8, 0.1)
        assert np.abs(p - tp.detach().numpy()).max() < 1e-13


def test_codes_are_the_nearest_and_keep_what_is_not_zero():
    rng = np.random.default_rng(2)
    m, v = rng.standard_normal(600), rng.standard_normal(600) ** 2
    m[5], v[5], v[6] = 0.0, 0.0, 1e-30
    qm, qv, scale = train.encode(m, v)
    assert qm[5] == 0 and qv[5] == 0 and qv[6] == 1 and scale.shape == (3, 2)
    assert np.abs(qm).max() == 127 and qv.max() == 255
    top = np.repeat(scale.astype(np.float64), 256, axis=0)[:600]
    root = np.sqrt(np.abs(m) / top[:, 0]) * 127
    assert np.abs(np.abs(qm) - root).max() <= 0.5 + 1e-6
    fourth = (v / top[:, 1]) ** 0.25 * 255
    assert (np.abs(qv - fourth)[v > 1e-20] <= 0.5 + 1e-6).all()
    assert np.abs(np.sqrt(np.abs(train.decode_m(qm, scale)) / top[:, 0]) * 127 - np.abs(qm)).max() < 1e-9
    # decoding and encoding again changes nothing
    again = train.encode(train.decode_m(qm, scale), train.decode_v(qv, scale))
    assert all(np.array_equal(a, b) for a, b in zip(again, (qm, qv, scale)))


def test_norm_and_factor():
    g = [np.array([3.0]), np.array([0.0, 4.0])]
    assert train.grad_norm(g) == (5.0, 1.0)
    assert train.grad_norm(g, 0.5, 1.0) == (2.5, 0.5 * 1.0 / 2.5)
    norm, factor = train.grad_norm([np.array([np.inf])], 1.0, 1.0)
    assert norm == np.inf and np.isnan(factor)

"""The oracle's Rotary and Attention: finite differences in float64, closed values, torch autograd."""
import numpy as np
import pytest
import torch

import oracle
from oracle import layers as OL
from workloads import reduced_config


def _differences(op, x, seed):
    """max |analytic - numeric| of d sum(f(x) * w) / dx over a scale of 1."""
    rng = np.random.default_rng(seed)
    y, ctx = op.forward(x)
    w = rng.standard_normal(y.shape)
    (dx,), _ = op.backward(ctx, w)
    num, h = np.zeros_like(x), 1e-6
    for i in np.ndindex(*x.shape):
        xp, xm = x.copy(), x.copy()
        xp[i] += h
        xm[i] -= h
        num[i] = ((op.forward(xp)[0] * w).sum() - (op.forward(xm)[0] * w).sum()) / (2 * h)
    return np.abs(dx - num).max()


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(interleaved):
    x = np.random.default_rng(1).standard_normal((6, 3 * 8))
    op = OL.Rotary(2, 8, 3, 4, 100.0, interleaved)
    y, _ = op.forward(x)
    np.testing.assert_array_equal(y[[0, 3]], x[[0, 3]])           # position 0 does not turn
    np.testing.assert_array_equal(y[:, 16:], x[:, 16:])           # nor does the third head
    np.testing.assert_array_equal(y[:, 4:8], x[:, 4:8])           # nor what lies behind rot
    p, q = (2, 3) if interleaved else (1, 3)
    a = 2 * 100.0 ** -0.5                                          # position 2, pair 1
    np.testing.assert_allclose(y[2, p], x[2, p] * np.cos(a) - x[2, q] * np.sin(a), rtol=1e-12)
    np.testing.assert_allclose(y[2, q], x[2, p] * np.sin(a) + x[2, q] * np.cos(a), rtol=1e-12)
    assert _differences(op, x, 2) < 1e-8


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 2), (False, 2)])
def test_attention(causal, window):
    x = np.random.default_rng(3).standard_normal((10, (4 + 2 * 2) * 3))
    op = OL.Attention(4, 2, 3, 5, causal, window)
    y, _ = op.forward(x)
    if causal:                                                     # the first row sees itself alone
        np.testing.assert_allclose(y[0, :3], x[0, 18:21], rtol=1e-12)
        np.testing.assert_allclose(y[5, 9:12], x[5, 21:24], rtol=1e-12)
    assert _differences(op, x, 4) < 1e-7


def test_against_torch():
    """Rotation and attention of a packed row, forward and gradient, from torch operations."""
    rng = np.random.default_rng(5)
    H, Hk, D, Ls, n = 4, 2, 6, 7, 2
    x = rng.standard_normal((n * Ls, (H + 2 * Hk) * D))
    w = rng.standard_normal((n * Ls, H * D))
    rot, att = OL.Rotary(H + Hk, D, Ls, 4, 50.0), OL.Attention(H, Hk, D, Ls, True, 4)
    r, _ = rot.forward(x)
    y, ctx = att.forward(r)
    (dx,), _ = rot.backward(None, att.backward(ctx, w)[0][0])
    t = torch.tensor(x, requires_grad=True)
    z = t.view(n, Ls, H + 2 * Hk, D)
    a = torch.arange(Ls)[:, None] * 50.0 ** (-2.0 * torch.arange(2, dtype=torch.float64) / 4)
    pair = torch.complex(z[..., :H + Hk, 0:2], z[..., :H + Hk, 2:4]) * torch.polar(torch.ones_like(a), a)[:, None]
    turned = torch.cat([pair.real, pair.imag, z[..., :H + Hk, 4:]], -1)
    q, k, v = turned[:, :, :H], turned[:, :, H:], z[:, :, H + Hk:]
    k, v = k.repeat_interleave(H // Hk, 2), v.repeat_interleave(H // Hk, 2)
    far = torch.arange(Ls)[:, None] - torch.arange(Ls)
    bias = torch.where((far >= 0) & (far < 4), 0.0, -torch.inf).double()
    p = torch.softmax((q[:, :, None] * k[:, None]).sum(-1) / D ** 0.5 + bias[None, :, :, None], 2)
    o = (p[..., None] * v[:, None]).sum(2).reshape(n * Ls, H * D)
    (o * torch.tensor(w)).sum().backward()
    np.testing.assert_allclose(y, o.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(dx, t.grad.numpy(), atol=1e-12)


def test_orderings_agree():
    """eager, forward-fusion (flushed) and backward-fusion of the blocks with attention, bit for bit."""
    runs = [oracle.run(reduced_config("attn12"), o, steps=2) for o in ("eager", "ff", "bf")]
    for r in runs[1:]:
        np.testing.assert_array_equal(r["losses"], runs[0]["losses"])
        for k in r["params"]:
            np.testing.assert_array_equal(r["params"][k], runs[0]["params"][k])

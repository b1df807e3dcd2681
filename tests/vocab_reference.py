"""Vocabulary losses in float64, and how far fp32 sums of the operands' exact products may be from them.

Values are formed from the definition and gradients by autograd.  Bounds, with e = 2^-24 and u the half
step of the operands' type (rounding the logits' gradient to it):
  a logit       |ds| <= (K + 8) e (|X| |W|^T), and 4 e cap more behind a cap
  lse           |dl| <= max |du| + (256 + V / 64 + 16) e + 4 e |lse|  (partial sums of at most 256 terms,
                at most V / 64 of them joined; an exponential, a logarithm, their arguments' rounding)
  probability   |dp| <= p (|du| + |dl| + 8 e (1 + |u| + |lse|)), to first order; 1.01 for the rest
  sums          dX and dW take their terms' bounds times the other operand, and (terms + 8) e of the sum
                of magnitudes
"""
import math

import torch

E = 2.0 ** -24


def target(ids, teacher, T, V):
    """Target weights per entry, and which rows count."""
    has = ids >= 0
    t = (torch.zeros_like(ids, dtype=torch.float64) if teacher is None else teacher.double() / T).masked_fill(~has, -math.inf)
    counts = (t > -math.inf).any(1)
    q = torch.softmax(torch.where(counts[:, None], t, 0.0), 1) * has * counts[:, None]
    return q, counts


class Reference:
    def __init__(self, x, w, ids, teacher=None, T=1.0, cap=0.0, z_loss=0.0, dloss=None, u=2.0 ** -24):
        """x [M, K], w [V, K], ids [M, k], all on one device; ids in [-1, V)."""
        x, w = x.double(), w.double()
        M, K = x.shape
        V = w.shape[0]
        q, counts = target(ids, teacher, T, V)
        x = x.detach().clone().requires_grad_(True)
        w = w.detach().clone().requires_grad_(True)
        s = x @ w.t()
        z = cap * torch.tanh(s / cap) if cap else s
        lse = torch.logsumexp(z / T, 1)
        zt = torch.where(ids >= 0, z.gather(1, ids.clamp_min(0)), 0.0)
        log_q = torch.where(q > 0, q, 1.0).log()
        loss = T * T * (q * (log_q - zt / T + lse[:, None])).sum(1) + z_loss * lse * lse
        loss = torch.where(counts, loss, 0.0)
        n = max(1, int(counts.sum()))
        g = torch.where(counts, dloss.double() if dloss is not None else torch.full((M,), 1.0 / n, device=x.device).double(), 0.0)
        self.mean = (loss.sum() / n).item()
        self.dx, self.dw = torch.autograd.grad((loss * g).sum(), (x, w))
        self.loss, self.lse, self.zt, self.counts, self.g = loss.detach(), lse.detach(), zt.detach(), counts, g
        with torch.no_grad():
            ds = (K + 8) * E * (x.abs() @ w.abs().t())
            dz = ds + (4 * E * cap if cap else 0.0)
            du, U = dz / T, z / T
            x, w = x.detach(), w.detach()
            self.e_lse = du.amax(1) + (256 + V / 64 + 16) * E + 4 * E * lse.abs()
            e_zt = torch.where(ids >= 0, dz.gather(1, ids.clamp_min(0)), 0.0)
            self.e_zt = e_zt + E * zt.abs() + 1e-30
            k = ids.shape[1]
            terms = (q * (log_q.abs() + zt.abs() / T + lse.abs()[:, None])).sum(1)
            # (the weights: an exponential and a quotient of a sum of k)
            self.e_loss = T * T * ((q * (e_zt / T + self.e_lse[:, None])).sum(1) + (2 * k + 32) * E * (terms + 1)) \
                + z_loss * (2 * lse.abs() * self.e_lse + 4 * E * lse * lse)
            self.e_loss = torch.where(counts, 1.01 * self.e_loss + 1e-30, 0.0)
            self.e_mean = self.e_loss.sum().item() / n + 4 * E * abs(self.mean)
            p = torch.softmax(U, 1)
            dp = 1.01 * p * (du + self.e_lse[:, None] + 8 * E * (1 + U.abs() + lse.abs()[:, None]))
            a = 1 + 2 * z_loss * lse[:, None]
            Q = torch.zeros_like(p).scatter_add_(1, ids.clamp_min(0), q)
            d = p * a - Q
            e = dp * a + p * 2 * z_loss * self.e_lse[:, None] + 8 * E * p * a + (2 * k + 16) * E * Q
            if cap:
                r = z / cap
                e = e * (1 - r * r) + d.abs() * (2 * dz / cap + 8 * E)
                d = d * (1 - r * r)
            f = (g * T)[:, None]
            d, e = d.abs() * f.abs(), e * f.abs()
            e = e + (u + 8 * E) * d + 1e-38
            self.e_dx = e @ w.abs() + (V + 8) * E * (d @ w.abs())
            self.e_dw = e.t() @ x.abs() + (M + 8) * E * (d.t() @ x.abs())


def near(name, got, want, bound, half=0.0):
    """|got - want| <= bound and the output's own rounding (half a step: 2^-8 for bf16)."""
    got = got.detach().to(want.device).double()
    bound = bound.to(want.device)
    over = (got - want).abs() - 1.01 * bound - (half + E) * want.abs() - 1e-30
    assert torch.isfinite(got).all() and (over <= 0).all(), (name, float(over.max()), int((over > 0).sum()), got.numel())

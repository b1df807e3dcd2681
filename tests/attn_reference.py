"""Attention in float64 with a bound on every output element's rounding error.

The reference follows the formulas of include/opfuse.h (of_attn_fwd, of_attn_bwd), one sequence and
head at a time.  The bounds are derived from the arithmetic the header promises, with u the half step
of the operand type (bf16 2^-8, fp32 2^-24), g that of the gradients' type, e = 2^-24:

  logits     z' = scale (q . k): D products summed in fp32, a rounding for the scale and one for the
             subtraction of the maximum or of lse, whose own error is that of a sum of nk terms:
             |dz| <= ez = (D + 4) e scale (|q| . |k|) + 4 e max|z| + (nk + 8) e
             (exp2 is within 2 e relative; log2 e is one rounding of the factor, in the 4 e |z|)
             In the backward the D sums may start from -lse / scale: each of their partial sums is
             larger by at most |lse| / scale, so ez grows by (D + 4) e |lse|.
  P          relative error rp = 2 ez (numerator and row sum), then one rounding u as an operand
             (0 in fp32, where the operand is the value)
  o          |do| <= (rp + u + (nk + 4) e) (P @ |v|) + u |o|
  dP         D products: |ddP| <= (D + 2) e (|dout| @ |v|')
  delta      |ddelta| <= |dout| . |do| + (D + 2) e (|dout| . |o|)
  dS         |ddS| <= P (|ddP| + |ddelta|) + (rp + u + 4 e) |dS|
  dq         scale (|ddS| @ |k| + (nk + 4) e |dS| @ |k|) + g |dq|, dk the same over the queries
  dv         (rp + u + (nq + 4) e) (P' @ |dout|) + g |dv|

where in fp32 the operand rounding u of P and dS is 0.  Each is doubled at the end (the products of
two small errors).
"""
import torch

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
E = 2.0 ** -24


def sees(nq, nk, causal, window):
    """[nq, nk] truth values: which keys a query sees."""
    far = torch.arange(nq)[:, None] + nk - nq - torch.arange(nk)[None]
    ok = torch.ones(nq, nk, dtype=torch.bool)
    if causal:
        ok &= far >= 0
    if window:
        ok &= far < window
        ok &= far > -window
    return ok


def forward(q, k, v, ok, scale, dtype):
    """One head: o, lse, and the bounds of both; then what the backward needs."""
    q, k, v = q.double(), k.double(), v.double()
    nk, D = k.shape
    u, uo = (HALF_STEP["bf16"], HALF_STEP["bf16"]) if dtype == "bf16" else (0.0, E)
    z = torch.where(ok, scale * (q @ k.t()), -torch.inf)
    lse = torch.logsumexp(z, 1) if nk else torch.full((q.shape[0],), -torch.inf, dtype=torch.float64)
    some = ok.any(1)
    p = torch.where(ok, torch.exp(z - torch.where(some, lse, 0.0)[:, None]), 0.0)
    zmax = torch.where(ok, z.abs(), 0.0).amax(1) if nk else torch.zeros(q.shape[0], dtype=torch.float64)
    ez = (D + 4) * E * scale * (q.abs() @ k.abs().t()) + (4 * E * zmax + (nk + 8) * E)[:, None]
    ez = torch.where(ok, ez, 0.0)
    rp = 2 * ez.amax(1, keepdim=True) if nk else torch.zeros(q.shape[0], 1, dtype=torch.float64)
    o = p @ v
    bo = 2 * ((rp + u + (nk + 4) * E) * (p @ v.abs()) + uo * o.abs())
    bl = 2 * (rp[:, 0] + E * torch.where(some, lse, 0.0).abs() + (nk + 8) * E)
    return o, lse, bo, bl, (p, rp)


def backward(q, k, v, do, ok, scale, dtype, grad_dtype):
    """One head: (dq, dk, dv) and their bounds."""
    o, lse, bo, _, (p, rp) = forward(q, k, v, ok, scale, dtype)
    rp = rp + 2 * (q.shape[1] + 4) * E * torch.where(ok.any(1), lse, 0.0).abs()[:, None]
    q, k, v, do = q.double(), k.double(), v.double(), do.double()
    nk, D = k.shape
    nq = q.shape[0]
    u = HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    g = HALF_STEP[grad_dtype]
    dp = do @ v.t()
    delta = (do * o).sum(1, keepdim=True)
    ds = p * (dp - delta)
    ddp = (D + 2) * E * (do.abs() @ v.abs().t())
    dde = (do.abs() * bo).sum(1, keepdim=True) + (D + 2) * E * (do.abs() * o.abs()).sum(1, keepdim=True)
    dds = p * (ddp + dde) + (rp + u + 4 * E) * ds.abs()
    dq, dk, dv = scale * (ds @ k), scale * (ds.t() @ q), p.t() @ do
    bq = scale * (dds @ k.abs() + (nk + 4) * E * (ds.abs() @ k.abs())) + g * dq.abs()
    bk = scale * (dds.t() @ q.abs() + (nq + 4) * E * (ds.abs().t() @ q.abs())) + g * dk.abs()
    bv = ((rp + u) * p).t() @ do.abs() + (nq + 4) * E * (p.t() @ do.abs()) + g * dv.abs()
    return (dq, dk, dv), (2 * bq, 2 * bk, 2 * bv)

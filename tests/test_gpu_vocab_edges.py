"""of_vocab_xent_* and of_vocab_distill_* where values or batches leave the ordinary: logits at their cap, operands and
gradients that are not finite, batches whose rows are gathered, other logits than the backward's own."""
import math

import pytest
import torch

from paper_2104_00237_amd import _lib as L
from tests.test_gpu_vocab import TYPES, Call
from tests.vocab_reference import near, target

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("dtype,grads", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,V,k", [(40, 300, 0), (40, 300, 3), (300, 700, 0), (512, 5000, 0), (512, 5000, 2), (2048, 8192, 0)])
def test_logits_at_their_cap(gpu, M, V, k, dtype, grads):
    """All logits between 4 and 9.5 caps: none leaves the cap, and a gradient keeps its sign and most of its bits where
    1 - tanh^2 has none left.

    Column 0 of X is 1 and the only one of W that is not zero, so that dW there is the sum of the rows' ds.  Relative
    to it: the slope 2^-18 and 2 |x| roundings of its argument (2^-17 in all), a probability's z and lse (the largest
    exponent's 4 E cap twice, 277 E of the sums, 8 E (1 + |z| + |lse|)), the sum's M E, roundings u to the type.  An entry's slope
    comes from its stored z, which is 6 E of the cap off."""
    cap = 2.0
    c = Call(gpu, M, V, 8, dtype, k=k, cap=cap, given=True, grads=grads, ids=torch.arange(max(k, 1)).repeat(M, 1))
    s = cap * torch.linspace(4.0, 9.5, V)
    s[1::2] *= -1
    s[:max(k, 1)] = 4.5 * cap + torch.arange(max(k, 1))
    c.w.zero_(), c.x.zero_()
    c.w[:, 0], c.x[:, 0] = s.to(c.w.dtype), 1
    c.dev_w.copy_(c.w), c.dev_x.copy_(c.x)
    c.dev_dloss.fill_(2.0 ** -11)
    c.fwd()
    c.bwd()
    s = c.w[:, 0].double()
    z = cap * torch.tanh(s / cap)
    e = torch.exp(-2 * s.abs() / cap)
    slope = 4 * e / (1 + e) ** 2
    p = torch.softmax(z, 0)
    q = torch.zeros(M, V).double()
    if k:
        q.scatter_(1, c.ids, torch.softmax(c.teacher.double(), 1))
    else:
        q[:, 0] = 1
    d = 2.0 ** -11 * (M * p - q.sum(0)) * slope
    got = c.dw[:, 0].double().cpu()
    u, half = TYPES[dtype][2], TYPES[grads][2]
    rel = u + half + (2 * 4 * cap + 277 + V / 64 + 8 * 12 + M) * E + 2.0 ** -17
    bound = 1.01 * rel * d.abs()
    n = max(k, 1)
    bound[:n] += 1.01 * 2.0 ** -11 * M * 16 * E
    assert (c.zt.abs() <= cap).all()
    assert (got[n:] >= 0).all(), got[n:].min()
    assert (got[:n] <= 0).all()
    over = (got - d).abs() - bound - 1e-38
    assert (over <= 0).all(), (float(over.max()), int(over.argmax()), float(got[over.argmax()]), float(d[over.argmax()]))


@pytest.mark.parametrize("M,V", [(9, 100), (50, 300), (300, 1000), (300, 8000), (500, 700), (512, 5000)])
@pytest.mark.parametrize("dtype,k", [("f32", 0), ("bf16", 0), ("f32", 2), ("bf16", 2)])
def test_rows_that_do_not_count_beside_an_infinite_head(gpu, M, V, dtype, k):
    """An entry that a head rules out (W of -infinity where every X is 1: probability 0) gets a gradient of exactly 0, with
    rows that do not count among the others, with gradients of 0, and where no row counts."""
    c = Call(gpu, M, V, 16, dtype, k=k, given=True)
    c.ids[::3] = -1
    c.ids[c.ids >= V - 3] = 0
    c.x[:, 0] = 1
    c.w[:, 0] = 0
    c.w[V - 2, 0] = -math.inf
    c.dloss[1::6] = 0.0
    for a, b in ((c.t[0], c.ids), (c.dev_x, c.x), (c.dev_w, c.w), (c.dev_dloss, c.dloss)):
        a.copy_(b)
    c.fwd()
    c.bwd(dx=False)
    c.w[V - 2, 0] = -3e4
    r = c.reference()
    near("dw", c.dw, r.dw, r.e_dw, TYPES[dtype][2])
    assert (c.dw[V - 2] == 0).all()
    c.ids[:] = -1
    c.t[0].copy_(c.ids)
    c.fwd()
    c.bwd()
    assert (c.dw == 0).all() and (c.dx == 0).all()


@pytest.mark.parametrize("dtype,M,V,k", [("f32", 12, 90, 0), ("f32", 512, 9000, 0), ("f32", 1030, 16384, 2), ("bf16", 12, 90, 0),
                                         ("bf16", 512, 5000, 2)])
def test_infinite_operands(gpu, dtype, M, V, k):
    """At every size the same: an infinite X or W that gives a row a logit of +infinity (or a NaN) makes its lse, loss and
    gradient NaN; one that gives -infinity leaves a probability of 0; other rows are as without it."""
    K, row = 16, 7
    c = Call(gpu, M, V, K, dtype, k=k, given=True, ids=None if k else torch.arange(M)[:, None] % (V - 40))
    c.ids[c.ids >= V - 40] = 1
    c.w[:, 0], c.x[:, 0] = 0, 1
    c.w[V - 20, 0] = -math.inf          # probability 0, but for X of 0 there: NaN
    nan = torch.zeros(M, dtype=torch.bool)
    nan[[2, 5, row, M - 1]] = True
    c.x[2, 0] = 0                       # 0 * -infinity
    c.x[5, 0] = -1                      # +infinity
    c.x[row, 3] = math.inf             # with W of both signs there
    c.x[M - 1, 4] = -math.inf
    c.ids[[2, 5, row, M - 1], 0] = 3
    for a, b in ((c.t[0], c.ids), (c.dev_x, c.x), (c.dev_w, c.w)):
        a.copy_(b)
    c.fwd()
    assert (c.lse.isnan().cpu() == nan).all()
    assert (c.loss.isnan().cpu() == nan).all() and c.mean.isnan().all()
    c.bwd()
    assert not torch.isfinite(c.dx.cpu()[nan].float()).any() and not torch.isfinite(c.dw.float()).any()
    clean_x, keep = c.x.clone(), ~nan
    clean_x[nan] = 0
    c.w[V - 20, 0] = -3e4
    r = c.reference(x=clean_x)
    near("lse", c.lse[keep.to(gpu)], r.lse[keep], r.e_lse[keep])
    near("loss", c.loss[keep.to(gpu)], r.loss[keep], r.e_loss[keep])
    near("dx", c.dx.cpu()[keep, 1:], r.dx[keep, 1:], r.e_dx[keep, 1:], TYPES[dtype][2])
    counts = keep & r.counts
    assert c.dx.cpu()[counts, 0].isnan().all()    # 0 * -infinity, as the product has it
    assert (c.dx.cpu()[~r.counts] == 0).all()


@pytest.mark.parametrize("M,V", [(12, 90), (512, 9000), (1030, 16384)])
def test_largest_operands(gpu, M, V):
    """fp32 operands up to the largest fp32 value keep all their bits."""
    c = Call(gpu, M, V, 16, "f32", ids=torch.arange(M)[:, None] % V)
    c.x[:, 0] = torch.linspace(3.3e38, 3.4028234e38, M)
    c.w[:, 0] = 0
    c.w[1::2, 0] = 2.0 ** -126 * 1.5
    c.dev_x.copy_(c.x), c.dev_w.copy_(c.w)
    c.fwd()
    c.check_fwd()


@pytest.mark.parametrize("M,V,k", [(2048, 90, 0), (2049, 90, 0), (3000, 90, 3), (20000, 40, 0)])
def test_many_rows_over_few_entries(gpu, M, V, k):
    """fp32, the mean's gradient: how many rows count is the same for all of them."""
    c = Call(gpu, M, V, 24, "f32", k=k)
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()


def test_time_grows_with_the_rows(gpu):
    """16 times the rows in less than 40 times the time (a workgroup a row that looks at all rows: 150 times)."""
    best = []
    for M in (1 << 14, 1 << 18):
        c = Call(gpu, M, 4, 32, "f32", ids=torch.randint(-1, 4, (M, 1), generator=torch.Generator().manual_seed(1)))
        c.fwd()
        c.bwd()
        times = []
        for _ in range(5):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            c.bwd()
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        best.append(min(times))
    assert best[1] < 40 * best[0], best


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,k", [(20, 700, 1024), (20, 9000, 1023), (33, 5000, 257), (450, 600, 301)])
def test_many_entries(gpu, dtype, M, V, k):
    """More entries than a workgroup has lanes, some named twice, over one and over several chunks of logits."""
    ids = torch.randint(-1, V, (M, k), generator=torch.Generator().manual_seed(k))
    c = Call(gpu, M, V, 40, dtype, k=k, ids=ids, T=1.5)
    c.fwd()
    c.bwd()
    c.check_fwd()
    c.check_bwd()


@pytest.mark.parametrize("step", [0.5, 0.02])
@pytest.mark.parametrize("M,V,K", [(40, 300, 40), (300, 1031, 64), (512, 5000, 64), (1030, 16384, 32)])
@pytest.mark.parametrize("dtype,k,cap", [("f32", 0, 0.0), ("bf16", 0, 0.0), ("f32", 0, 6.0), ("bf16", 0, 6.0), ("f32", 3, 0.0),
                                         ("bf16", 3, 0.0), ("f32", 70, 6.0), ("bf16", 70, 6.0)])
def test_a_head_that_moved_on(gpu, dtype, k, cap, M, V, K, step):
    """W other than the forward's: p = exp(z / T - lse) of the forward's lse and W's own z, at every size; but that
    distillation's entries have the forward's z.

    Bounds as in tests/vocab_reference.py with lse (and entries' z) given; a label's logit may be the forward's where it
    differs by 2^-16 (1 + |z|)."""
    T = 2.0 if k else 1.0
    c = Call(gpu, M, V, K, dtype, k=k, T=T, cap=cap, given=True, grads="f32")
    c.fwd()
    w = (c.w.float() * (1 + step * torch.randn(V, K, generator=torch.Generator().manual_seed(3)))).to(c.w.dtype)
    c.dev_w.copy_(w)
    c.bwd()
    x, w, lse = c.dev_x.double(), w.double().to(gpu), c.lse.double()[:, None]
    ids = c.t[0]
    place = torch.where(ids >= 0, ids, V)   # (what is no entry goes to a column behind)
    at = torch.zeros(M, V + 1, device=gpu, dtype=torch.bool).scatter_(1, place, True)[:, :V]
    q, counts = target(ids, c.t[1] if k else None, T, V)
    s = x @ w.t()
    z = cap * torch.tanh(s / cap) if cap else s
    dz = (K + 8) * E * (x.abs() @ w.abs().t()) + 4 * E * cap
    if k:
        z = torch.where(at, torch.zeros(M, V + 1, device=gpu).double().scatter_(1, place, c.zt.double())[:, :V], z)
        dz = torch.where(at, 0.0, dz)
    else:
        dz = dz + at * 2.0 ** -16 * (1 + z.abs())
    U, du, p = z / T, dz / T, torch.exp(z / T - lse)
    u = TYPES[dtype][2]
    Q = torch.zeros_like(p).scatter_add_(1, ids.clamp_min(0), q)
    f = torch.where(counts, c.dev_dloss.double() * T, 0.0)[:, None]
    d = p - Q
    e = 1.01 * p * (du + 8 * E * (1 + U.abs() + lse.abs())) + 8 * E * p + (2 * c.k + 16) * E * Q
    if cap:
        slope = 1 - (z / cap) ** 2
        e = e * slope + d.abs() * (2 * dz / cap + 8 * E)
        d = d * slope
    d, e = d * f, e * f + (u + 8 * E) * (d * f).abs() + 1e-38
    near("dx", c.dx, d @ w, e @ w.abs() + (V + 8) * E * (d.abs() @ w.abs()))
    near("dw", c.dw, d.t() @ x, e.t() @ x.abs() + (M + 8) * E * (d.abs().t() @ x.abs()))

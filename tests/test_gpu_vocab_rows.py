"""Rows of every kind (without a target, with an id past the vocabulary, of NaN and infinities) and updates of the head at the sizes
whose backward gathers the rows with a gradient (more than 384) and at those of fp32 tiles that prepare them."""
import math

import pytest
import torch

from paper_2104_00237_amd import _lib as L
from tests.test_gpu_vocab import OPTS, TYPES, Call
from tests.vocab_reference import near

pytestmark = pytest.mark.gpu
# dtype, rows, entries: gathered; fp32's and bf16's 256x256 tiles; prepared on fp32 tiles
SIZES = [("bf16", 385, 333), ("bf16", 700, 1000), ("f32", 512, 5000), ("f32", 385, 5500), ("f32", 300, 8000), ("bf16", 1500, 9000)]


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("dtype,M,V", SIZES)
def test_rows_of_every_kind(gpu, dtype, M, V, k, given):
    """A third of the rows does not count and holds NaN or infinities, some by teacher's logits of -infinity; some ids lie
    past the vocabulary: those rows count, their loss is NaN and their gradient 0."""
    K = 72
    c = Call(gpu, M, V, K, dtype, k=k, given=given)
    n = torch.arange(M)
    c.ids[:, 0] = c.ids[:, 0].clamp_min(0)
    out = n % 3 == 1
    past = (n % 50 == 2) & ~out
    c.ids[out] = -1
    if k:
        low = n % 6 == 1
        c.ids[low] = 5
        c.teacher[low] = -math.inf
        c.teacher[n % 6 == 4] = math.nan
    clean = c.ids.clone()
    c.ids[past, 0] = torch.where(n[past] % 4 == 0, V, 1 << 40)
    clean[past] = 0
    bad = torch.randn(M, K)
    bad[::2], bad[1::2] = math.nan, math.inf
    c.dev_x[out.to(gpu)] = bad[out].to(c.x.dtype).to(gpu)
    c.t[0].copy_(c.ids)
    if k:
        c.t[1].copy_(c.teacher)
    c.fwd()
    c.bwd()
    live = ~out & ~past
    r = c.reference(device=gpu, ids=clean)
    assert (r.counts.cpu() == ~out).all()
    assert (c.loss.cpu().isnan() == past).all() and c.mean.isnan().all() and (c.loss.cpu()[out] == 0).all()
    near("loss", c.loss[live.to(gpu)], r.loss[live.to(gpu)], r.e_loss[live.to(gpu)])
    near("lse", c.lse[~out.to(gpu)], r.lse[~out.to(gpu)], r.e_lse[~out.to(gpu)])
    g = c.dloss.clone() if given else torch.full((M,), 1.0 / int((~out).sum()))
    g[past] = 0
    r = c.reference(device=gpu, ids=clean, dloss=g)
    c.check_bwd(r)
    assert (c.dx.cpu()[~live] == 0).all()
    c.untouched()


@pytest.mark.parametrize("k", [0, 2])
@pytest.mark.parametrize("dtype,M,V", SIZES)
def test_no_row_counts(gpu, dtype, M, V, k):
    """Of X of NaN: no loss, no gradient, what is added to stays, and an update is one with a gradient of 0."""
    K = 40
    c = Call(gpu, M, V, K, dtype, k=k, ids=torch.full((M, max(k, 1)), -1), grads="f32")
    c.dev_x.fill_(math.nan)
    c.fwd()
    assert (c.loss == 0).all() and (c.mean == 0).all() and (c.zt == 0).all()
    c.bwd()
    assert (c.dx == 0).all() and (c.dw == 0).all()
    c.dw.fill_(3.0)
    c.bwd(accumulate=1)
    assert (c.dw == 3).all()
    w = c.dev_w.float() if dtype == "bf16" else c.dev_w
    m, v = torch.full_like(w, 0.25), torch.zeros_like(w)
    shadow = c.dev_w.data_ptr() if dtype == "bf16" else None
    c.param = L.OfParam(w.data_ptr(), m.data_ptr(), v.data_ptr(), shadow, V * K)
    old = w.clone()
    c.dx.fill_(7.0)
    c.bwd_fused(L.make_opt(dict(kind="sgd", lr=0.5, momentum=0.5), 2))
    assert (c.dx == 0).all() and (m == 0.125).all() and torch.equal(w, old - 0.5 * m)


@pytest.mark.parametrize("k", [0, 4])
@pytest.mark.parametrize("dtype,M,V", SIZES)
@pytest.mark.parametrize("hyper", [OPTS[0], OPTS[2]], ids=["sgd", "adamw"])
def test_update_of_either_loss(gpu, dtype, M, V, k, hyper):
    """Both losses' updates on tiles are those of their stored fp32 gradient, bit for bit; dX is that of the old W."""
    K = 64
    c = Call(gpu, M, V, K, dtype, k=k, grads="f32")
    g = torch.Generator().manual_seed(5)
    w = c.w.float().add(torch.randn(V, K, generator=g) * 1e-4).to(gpu) if dtype == "bf16" else c.dev_w
    m, v = (torch.randn(V, K, generator=g) * 1e-3).to(gpu), (torch.rand(V, K, generator=g) * 1e-5).to(gpu)
    extra = (torch.randn(V, K, generator=g) * 1e-4).to(gpu)
    shadow = c.dev_w if dtype == "bf16" else None
    c.fwd()
    c.bwd()
    c.check_bwd(c.reference(device=gpu))
    dx, dw = c.dx.clone(), c.dw.clone()
    ref = [t.clone() for t in (w, m, v)]
    ref_shadow = shadow.clone() if dtype == "bf16" else None
    opt = L.make_opt(hyper, 3)
    total = torch.empty_like(dw)
    L.of_add(extra.data_ptr(), dw.data_ptr(), dw.numel(), total.data_ptr(), c._stream())
    L.of_elementwise_fused_update(L.param_of(*ref, w_bf16=ref_shadow), total.data_ptr(), 1, 0, opt, c._stream())
    c.param = L.OfParam(w.data_ptr(), m.data_ptr(), v.data_ptr(), shadow.data_ptr() if dtype == "bf16" else None, V * K)
    c.dx.fill_(7.0)
    c.bwd_fused(opt, extra)
    assert torch.equal(c.dx, dx)
    for name, a, b in zip("wmv", (w, m, v), ref):
        assert torch.equal(a, b), (name, float((a - b).abs().max()))
    if dtype == "bf16":
        assert torch.equal(shadow, ref_shadow)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,K,k,gap", [(4, 3000, 64, 0, 0), (40, 300, 64, 0, 8), (70, 900, 257, 5, 0), (300, 2000, 128, 3, 3),
                                         (600, 5000, 320, 0, 16), (600, 5000, 320, 7, 0)])
def test_aligned_operands(gpu, dtype, M, V, K, k, gap):
    """What the smaller workspace of aligned operands gives is the same, and nothing behind it is touched."""
    c = Call(gpu, M, V, K, dtype, k=k, gap=gap)
    c.fwd()
    c.bwd()
    want = [t.clone() for t in (c.loss, c.lse, c.zt, c.mean, c.dx, c.dw)]
    c.d.aligned = 1
    for op in c.ws:
        c.ws[op] = torch.full((L.of_vocab_workspace_size(c.d, op) + 256,), 0xff, dtype=torch.uint8, device=gpu)
    for t in (c.loss, c.lse, c.zt, c.mean, c.dx, c.dw):
        t.fill_(7.0)
    c.fwd()
    c.bwd()
    for a, b in zip((c.loss, c.lse, c.zt, c.mean, c.dx, c.dw), want):
        assert torch.equal(a, b)
    w, m, v = (torch.zeros(V, K, device=gpu) for _ in range(3))
    if dtype == "f32":
        w = c.dev_w
    c.param = L.OfParam(w.data_ptr(), m.data_ptr(), v.data_ptr(), c.dev_w.data_ptr() if dtype == "bf16" else None, V * K)
    c.dx.fill_(7.0)
    c.bwd_fused(L.make_opt(OPTS[1], 1))
    assert torch.equal(c.dx, want[4])
    c.untouched()


@pytest.mark.parametrize("dtype,M,V,k", [("bf16", 500, 700, 0), ("bf16", 500, 700, 5), ("f32", 512, 5000, 3), ("f32", 300, 8000, 0),
                                         ("f32", 2500, 90, 0), ("bf16", 60, 300, 2)])
def test_replays_of_other_targets(gpu, dtype, M, V, k):
    """Forward, backward and update captured once and replayed with other targets: as many rows with a gradient as there are
    (all, some, one, none), and every other result as the eager calls give it."""
    c = Call(gpu, M, V, 64, dtype, k=k, ids=torch.randint(0, V, (M, max(k, 1)), generator=torch.Generator().manual_seed(4)))
    w = c.dev_w.float() if dtype == "bf16" else c.dev_w
    shadow = c.dev_w if dtype == "bf16" else torch.zeros(1, device=gpu)
    m, v = torch.zeros_like(w), torch.zeros_like(w)
    c.param = L.OfParam(w.data_ptr(), m.data_ptr(), v.data_ptr(), shadow.data_ptr() if dtype == "bf16" else None, c.V * c.K)
    step = torch.zeros(1, dtype=torch.int64, device=gpu)
    opt = L.make_opt(OPTS[1], 0, step.data_ptr())
    out, state = (c.loss, c.lse, c.zt, c.mean, c.dx, c.dw), (w, m, v, shadow, step)

    def all_calls():
        c.fwd()
        c.bwd()
        step.add_(1)
        c.bwd_fused(opt)

    start = [t.clone() for t in state]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        all_calls()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        all_calls()
    g = torch.Generator().manual_seed(2)
    for out_of in (0.0, 0.3, 1.0, 0.9, 2.0, 0.0):
        ids = c.ids.clone()
        ids[torch.rand(M, generator=g) < out_of] = -1
        if out_of == 1.0:
            ids[M // 2] = 1
        c.t[0].copy_(ids)
        results = []
        for call in (all_calls, graph.replay):
            for t, a in zip(state, start):
                t.copy_(a)
            for t in out:
                t.fill_(7.0)
            torch.cuda.synchronize()
            call()
            torch.cuda.synchronize()
            results.append([t.clone() for t in out + state])
        for a, b in zip(*results):
            assert torch.equal(a, b), out_of


@pytest.mark.parametrize("dtype,M,V,k", [("bf16", 500, 700, 0), ("bf16", 40, 300, 3), ("f32", 512, 5000, 0), ("f32", 40, 300, 2)])
def test_update_with_a_clipping_factor(gpu, dtype, M, V, k):
    """The factor of a clipped gradient applies to dW and the earlier gradient alike, as in the element-wise update."""
    K = 48
    c = Call(gpu, M, V, K, dtype, k=k, grads="f32")
    w = c.dev_w.float() if dtype == "bf16" else c.dev_w
    m, v = torch.zeros_like(w), torch.zeros_like(w)
    extra = torch.randn(V, K, generator=torch.Generator().manual_seed(6)).mul_(1e-4).to(gpu)
    factor = torch.tensor([0.37], device=gpu)
    opt = L.make_opt(OPTS[0], 3)
    opt.grad_scale = factor.data_ptr()
    c.fwd()
    c.bwd()
    ref = [t.clone() for t in (w, m, v)]
    total = c.dw + extra
    L.of_elementwise_fused_update(L.param_of(*ref), total.data_ptr(), 1, 0, opt, c._stream())
    c.param = L.OfParam(w.data_ptr(), m.data_ptr(), v.data_ptr(), c.dev_w.data_ptr() if dtype == "bf16" else None, V * K)
    c.bwd_fused(opt, extra)
    for a, b in zip((w, m, v), ref):
        assert torch.equal(a, b)

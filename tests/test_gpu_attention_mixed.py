"""fp32 gradients of bf16 operands (what a training step asks of of_attn_bwd): dO is rounded once into the
workspace and read from there by the second launch."""
import pytest
import torch

from attn_reference import backward, sees
from paper_2104_00237_amd import _lib as L
from test_gpu_attention import Call

pytestmark = pytest.mark.gpu


def test_heads_behind_each_other(gpu):
    """2^20 query heads of 72, one behind the other.  A copy of dO with a row of all heads would be
    151 MB a row, and row 29 past 32 bits.  Only a few heads have a gradient, in rows 30 and on: everything
    else adds exact zeros, so the bounds are those of these heads alone."""
    H, T, D, some = 1 << 20, 40, 72, (0, 3, (1 << 19) + 5, (1 << 20) - 1)
    gen = torch.Generator().manual_seed(3)
    bf, dev = torch.bfloat16, dict(device=gpu)
    q, o = torch.zeros(H, T, D, dtype=bf, **dev), torch.empty(H, T, D, dtype=bf, **dev)
    do, dq = torch.zeros(H, T, D, **dev), torch.full((H, T, D), 7.0, **dev)
    k, v = (torch.randn(T, 1, D, generator=gen).to(bf) for _ in range(2))
    qs, ds = torch.randn(len(some), T, D, generator=gen).to(bf), torch.randn(len(some), T, D, generator=gen)
    ds[:, :30] = 0
    for i, h in enumerate(some):
        q[h], do[h] = qs[i], ds[i]
    kd, vd = k.to(gpu), v.to(gpu)
    dk, dv = torch.empty(T, 1, D, **dev), torch.empty(T, 1, D, **dev)
    lse = torch.empty(H, T, **dev)
    d = L.OfAttnDesc(Tq=T, Tk=T, nseq=1, Hq=H, Hkv=1, D=D, dtype=L.OF_BF16, grad_dtype=L.OF_F32, causal=1,
                     ldq=D, hsq=T * D, ldo=D, hso=T * D)
    n = [L.of_attn_workspace_size(d, op) for op in (L.OF_ATTN_FWD, L.OF_ATTN_BWD)]
    ws = torch.empty(max(n), dtype=torch.uint8, **dev)
    s = torch.cuda.current_stream().cuda_stream
    L.of_attn_fwd(d, q.data_ptr(), kd.data_ptr(), vd.data_ptr(), o.data_ptr(), lse.data_ptr(), ws.data_ptr(), n[0], s)
    L.of_attn_bwd(d, *[x.data_ptr() for x in (q, kd, vd, o, lse, do, dq, dk, dv)], ws.data_ptr(), n[1], s)
    torch.cuda.synchronize()
    ok = sees(T, T, 1, 0)
    sums = [torch.zeros(T, D, dtype=torch.float64) for _ in range(4)]
    moved = 0
    for i, h in enumerate(some):
        (wq, *wkv), (bq, *bkv) = backward(qs[i], k[:, 0], v[:, 0], ds[i].to(bf), ok, D ** -0.5, "bf16", "f32")
        got = dq[h].cpu()
        Call.near(got, wq, bq, f"head {h} dq")
        moved += int(got.count_nonzero())
        for a, b in zip(sums, wkv + bkv):
            a += b
    Call.near(dk[:, 0].cpu(), sums[0], sums[2], "dk")
    Call.near(dv[:, 0].cpu(), sums[1], sums[3], "dv")
    assert sum(int(x.count_nonzero()) for x in dq.split(1 << 16)) == moved
    del q, o, do, dq, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("layout,shift", [("rows", 0), ("heads", 0), ("odd", 1)])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
def test_split_over_the_queries(gpu, D, layout, shift):
    """dK and dV in parts, from the copy of dO: few key tiles, many queries."""
    c = Call([1200, 40], [300, 40], Hq=4, Hkv=1, D=D, grad="f32", causal=1, tail=2, layout=layout, shift=shift)
    kept = 4 * (4 * c.Tq + 3) + 2 * 4 * c.Tq * D + 15      # statistics and the copy
    assert c.ws[L.OF_ATTN_BWD][1] > kept
    c.fwd().bwd().check()


def test_split_with_padded_slots(gpu):
    """Rows behind a length hold NaN, in dO too: they are neither copied nor summed."""
    c = Call([1100, 0, 700], [260, 7, 90], Hq=4, Hkv=1, D=64, grad="f32", causal=1, slots=True)
    assert c.ws[L.OF_ATTN_BWD][1] > 4 * (4 * c.Tq + 3) + 2 * 4 * c.Tq * 64 + 15
    c.fwd().bwd().check()


def test_as_a_training_step_calls_it(gpu):
    """The full-size block: 4 sequences of 1024, 16/4 heads of 64, Q, K and V in packed rows and their
    gradients in packed fp32 rows; dK and dV in parts, delta from O (more than 256 keys)."""
    T, Hq, Hkv, D = 4096, 16, 4, 64
    c = Call([1024] * 4, [1024] * 4, Hq=Hq, Hkv=Hkv, D=D, grad="f32", causal=1)
    qkv = torch.cat([c.q, c.k, c.v], 1)
    grads = torch.full((T, Hq + 2 * Hkv, D), 7.0, device=gpu)
    parts = (slice(0, Hq), slice(Hq, Hq + Hkv), slice(Hq + Hkv, None))
    c.q, c.k, c.v = (qkv[:, p] for p in parts)
    c.dq, c.dk, c.dv = (grads[:, p] for p in parts)
    c.d.ldq = c.d.ldk = c.d.ldv = (Hq + 2 * Hkv) * D
    c.d.q_off = c.d.k_off = None
    need = L.of_attn_workspace_size(c.d, L.OF_ATTN_BWD)
    assert need > 4 * Hq * T + 2 * Hq * T * D
    c.ws[L.OF_ATTN_BWD] = (torch.full((need // 4,), float("nan"), device=gpu), need)
    c.fwd().bwd().check()

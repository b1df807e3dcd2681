"""of_rotary_fwd and of_rotary_bwd against float64: both pair layouts, part of the head, scalings, far
positions, strides, in place, one row to many.

Bound per element, with u the half step of the type and e = 2^-24: the turn is reduced in float64 (an
angle error below 1e-9 at position 1e6), rounded to fp32 (e relative of at most half a turn: 2 pi e / 2)
and its cosine and sine are within 4 e; two products and a sum: |d| <= (pi + 8) e m (|u| + |v|) + u |y|.
"""
import math

import pytest
import torch

from paper_2104_00237_amd import _lib as L

pytestmark = pytest.mark.gpu
TYPES = {"f32": (torch.float32, L.OF_F32, 2.0 ** -24), "bf16": (torch.bfloat16, L.OF_BF16, 2.0 ** -8)}
E = 2.0 ** -24


def freqs(rot, base=10000.0, scaling="none", factor=1.0, orig=0.0, low=0.0, high=0.0):
    w = []
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "bands":
            n = orig * f / (2 * math.pi)
            if n <= low:
                f /= factor
            elif n < high:
                g = (n - low) / (high - low)
                f = g * f + (1 - g) * f / factor
        w.append(f)
    return torch.tensor(w, dtype=torch.float64)


def turn(x, pos, w, rot, interleaved, m, sign):
    """float64 rotation of [T, H, D] and each element's bound before the type's own rounding."""
    y, b = x.clone(), torch.zeros_like(x)
    a = pos.double()[:, None] * w
    c, s = torch.cos(a)[:, None] * m, torch.sin(a)[:, None] * (m * sign)
    i = torch.arange(rot // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    u, v = x[..., p], x[..., q]
    y[..., p], y[..., q] = u * c - v * s, u * s + v * c
    b[..., p] = b[..., q] = (math.pi + 8) * E * m * (u.abs() + v.abs()) + 1e-9 * (u.abs() + v.abs())
    return y, b


def run(gpu, T, H, D, rot, interleaved, dtype, pos=None, gap=0, shift=0, in_place=False, inverse=False, seq_len=0,
        pos0=0, m=0.0, heads_apart=False, **scale):
    t, kind, half = TYPES[dtype]
    g = torch.Generator().manual_seed(T * 31 + D)

    def place(x):
        ld, hs = (D, T * D) if heads_apart else (H * D + gap, D)
        flat = torch.full(((T - 1) * ld + (H - 1) * hs + D + shift + gap,), 7.0, dtype=t, device=gpu)
        y = flat[shift:].as_strided((T, H, D), (ld, hs, 1))
        y.copy_(x)
        return y, flat
    x, flat = place(torch.randn(T, H, D, generator=g).to(t))
    y, yflat = (x, flat) if in_place else place(torch.full((T, H, D), 7.0, dtype=t))
    x0 = x.detach().cpu().double()
    before = yflat.clone()
    d = L.OfRotaryDesc(T=T, seq_len=seq_len, pos0=pos0, H=H, D=D, rot=rot, interleaved=interleaved, dtype=kind,
                       scaling=L.ROPE_SCALINGS[scale.get("scaling", "none")], base=scale.get("base", 10000.0),
                       factor=scale.get("factor", 0.0), orig_len=scale.get("orig", 0.0),
                       low_turns=scale.get("low", 0.0), high_turns=scale.get("high", 0.0), mscale=m,
                       ldx=x.stride(0), hsx=x.stride(1), ldy=y.stride(0), hsy=y.stride(1))
    dev = pos.to(gpu) if pos is not None else None
    f = L.of_rotary_bwd if inverse else L.of_rotary_fwd
    f(d, x.data_ptr(), dev.data_ptr() if dev is not None else None, y.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    p = pos if pos is not None else pos0 + torch.arange(T) % (seq_len or T)
    want, bound = turn(x0, p, freqs(rot, **scale), rot, interleaved, m or 1.0, -1.0 if inverse else 1.0)
    err = (y.detach().cpu().double() - want).abs()
    assert (err <= bound + half * want.abs() + 1e-30).all(), float((err - bound - half * want.abs()).max())
    assert torch.equal(y.detach().cpu().double()[..., rot:], x0[..., rot:])
    # nothing between or behind the rows was written
    inside = torch.zeros(yflat.shape, dtype=torch.bool, device=gpu)
    inside[shift:].as_strided((T, H, D), y.stride()).fill_(True)
    assert torch.equal(yflat[~inside], before[~inside])


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 64), (40, 40), (34, 34), (33, 2), (80, 20), (256, 256), (520, 512)])
def test_widths(gpu, D, rot, dtype, interleaved):
    for inverse in (False, True):
        run(gpu, 37, 3, D, rot, interleaved, dtype, inverse=inverse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [0, 1])
def test_strides_and_in_place(gpu, dtype, interleaved):
    run(gpu, 21, 4, 64, 32, interleaved, dtype, gap=64)
    run(gpu, 21, 4, 64, 32, interleaved, dtype, gap=3)
    run(gpu, 21, 4, 64, 64, interleaved, dtype, shift=1)
    run(gpu, 21, 4, 64, 48, interleaved, dtype, gap=128, in_place=True)
    run(gpu, 21, 4, 36, 36, interleaved, dtype, gap=5, in_place=True, inverse=True)
    run(gpu, 21, 4, 64, 64, interleaved, dtype, heads_apart=True)


@pytest.mark.parametrize("T", [1, 2, 1000, 5001])
def test_lengths(gpu, T):
    run(gpu, T, 2, 64, 64, 0, "f32")
    run(gpu, T, 2, 64, 64, 1, "bf16", seq_len=max(1, T // 3), pos0=100)


def test_many_heads(gpu):
    run(gpu, 3, 4000, 64, 64, 0, "bf16")
    run(gpu, 3, 4000, 33, 32, 1, "f32")


@pytest.mark.parametrize("scale", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                   dict(scaling="bands", factor=8.0, orig=8192.0, low=1.0, high=4.0),
                                   dict(base=500000.0)], ids=str)
def test_scalings(gpu, scale):
    pos = torch.randint(0, 100000, (50,), generator=torch.Generator().manual_seed(1))
    for D in (2, 64):
        run(gpu, 50, 2, D, D, 0, "f32", pos=pos, **scale)
    run(gpu, 50, 2, 64, 32, 1, "bf16", pos=pos, m=1.25, inverse=True, **scale)


def test_far_and_negative_positions(gpu):
    pos = torch.tensor([0, 1, -1, -5000, 999999, 1000000, 131072])
    run(gpu, 7, 2, 64, 64, 0, "f32", pos=pos)


@pytest.mark.parametrize("ld,hs", [(1 << 21, 64), (64, (1 << 31) + 64)], ids=["rows", "heads"])
def test_offsets_past_32_bits(gpu, ld, hs):
    """Rows or heads so far apart that offsets pass 32 bits give what a contiguous call gives."""
    T, H, D = 1100, 2, 64
    x = torch.randn(T, H, D, device=gpu).to(torch.bfloat16)
    y = torch.empty_like(x)
    far = [torch.empty((T - 1) * ld + (H - 1) * hs + D, dtype=x.dtype, device=gpu).as_strided((T, H, D), (ld, hs, 1))
           for _ in range(2)]
    far[0].copy_(x)
    d = L.OfRotaryDesc(T=T, H=H, D=D, rot=D, dtype=L.OF_BF16, base=10000.0)
    w = L.OfRotaryDesc(T=T, H=H, D=D, rot=D, dtype=L.OF_BF16, base=10000.0, ldx=ld, hsx=hs, ldy=ld, hsy=hs)
    s = torch.cuda.current_stream().cuda_stream
    L.of_rotary_fwd(d, x.data_ptr(), None, y.data_ptr(), s)
    L.of_rotary_fwd(w, far[0].data_ptr(), None, far[1].data_ptr(), s)
    torch.cuda.synchronize()
    assert torch.equal(far[1].contiguous(), y)
    assert torch.equal(far[0].contiguous(), x)
    del far
    torch.cuda.empty_cache()


def test_turns_back(gpu):
    """The backward of the forward's output is the input again (a turn is orthogonal): two turns' bounds."""
    t, kind, half = TYPES["f32"]
    x = torch.randn(300, 4, 64, device=gpu)
    y, z = torch.empty_like(x), torch.empty_like(x)
    d = L.OfRotaryDesc(T=300, H=4, D=64, rot=64, dtype=kind, base=10000.0)
    s = torch.cuda.current_stream().cuda_stream
    L.of_rotary_fwd(d, x.data_ptr(), None, y.data_ptr(), s)
    L.of_rotary_bwd(d, y.data_ptr(), None, z.data_ptr(), s)
    torch.cuda.synchronize()
    size = x[..., :32].abs() + x[..., 32:].abs()
    assert ((z - x).abs() <= 4 * (math.pi + 10) * E * torch.cat([size, size], -1)).all()


def test_graph_replays(gpu):
    x = torch.randn(64, 4, 64, device=gpu).to(torch.bfloat16)
    y = torch.empty_like(x)
    pos = torch.arange(64, device=gpu)
    d = L.OfRotaryDesc(T=64, H=4, D=64, rot=64, dtype=L.OF_BF16, base=10000.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        L.of_rotary_fwd(d, x.data_ptr(), pos.data_ptr(), y.data_ptr(), side.cuda_stream)
    for k in range(3):
        pos.add_(1000)           # the replay reads what the buffer holds then
        x.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        z = torch.empty_like(x)
        L.of_rotary_fwd(d, x.data_ptr(), pos.data_ptr(), z.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(y, z)

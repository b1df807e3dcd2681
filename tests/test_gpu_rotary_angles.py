"""The rotary kernel's cosines and sines themselves: a pair (1, 0) turns to (cos a, sin a) in fp32, exactly the
kernel's factors.

Bound, with e = 2^-24: the angle is a float64 number of turns, position times frequency, whose three
roundings of 2^-53 leave 2 pi 3 2^-53 of its at most 1.6e5 turns, 4e-10 (as in the reference); the
angle does not lose more, so next to a zero of the sine or the cosine only the functions' own error and the
last rounding remain, both relative to the value: 4 e + e.  |d| <= 5 e |value| + 1e-9.
(An angle rounded to fp32 would be off by up to pi 2^-25 = 9.4e-8, 1.6 e, wherever it is.)
"""
import pytest
import torch

from paper_2104_00237_amd import _lib as L

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("far", [100, 8000, 1000000])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_cosines_and_sines(gpu, inverse, interleaved, far):
    T, D = 4000, 64
    i = torch.arange(D // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + D // 2)
    x = torch.zeros(T, 1, D)
    x[..., p] = 1.0
    pos = torch.randint(-far, far, (T,), generator=torch.Generator().manual_seed(far))
    y, dev = x.to(gpu), pos.to(gpu)
    d = L.OfRotaryDesc(T=T, H=1, D=D, rot=D, interleaved=interleaved, dtype=L.OF_F32, base=10000.0)
    f = L.of_rotary_bwd if inverse else L.of_rotary_fwd
    f(d, y.data_ptr(), dev.data_ptr(), y.data_ptr(), torch.cuda.current_stream().cuda_stream)
    got = y.cpu().double()
    a = pos.double()[:, None] * torch.tensor([10000.0 ** (-2 * k / D) for k in range(D // 2)], dtype=torch.float64)
    for at, want in ((p, a.cos()), (q, -a.sin() if inverse else a.sin())):
        err = (got[:, 0, at] - want).abs()
        bound = 5 * E * want.abs() + 1e-9
        assert (err <= bound).all(), f"{int((err > bound).sum())} of {err.numel()} off, worst {float((err / bound).max()):.3g} bounds"

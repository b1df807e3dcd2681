"""fp32 attention gradients against float64, with bounds for logits that do not start from -lse / scale.

The bounds of tests/attn_reference.py widen the backward's logits by (D + 4) e |lse| for sums that start there;
only bf16 operands' do.  Here fp32 is held to the bound without it: forward() as backward() sees
it leaves lse out, which that widening alone uses.
"""
import pytest
import torch

import attn_reference
from test_gpu_attention import MASKS, SEQS, Call

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def no_widening(monkeypatch):
    full = attn_reference.forward

    def forward(*args):
        o, lse, bo, bl, rest = full(*args)
        return o, torch.where(torch.isinf(lse), lse, 0.0), bo, bl, rest
    monkeypatch.setattr(attn_reference, "forward", forward)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("seqs", SEQS)
def test_masks_and_sequences(gpu, seqs, mask):
    causal, window = MASKS[mask]
    Call(*SEQS[seqs], Hq=4, Hkv=2, D=64, dtype="f32", causal=causal, window=window, tail=3).fwd().bwd().check()


@pytest.mark.parametrize("D", [1, 16, 33, 64, 80, 96, 128, 192, 256])
def test_head_widths(gpu, D):
    Call([100, 37], [100, 37], Hq=3, Hkv=1, D=D, dtype="f32", causal=1).fwd().bwd().check()


def test_statistics_far_from_zero(gpu):
    """Logits that share a large part: lse of hundreds, probabilities of ordinary size."""
    c = Call([260], [260], Hq=2, Hkv=1, D=64, dtype="f32", causal=1, scale=1.0)
    c.q[..., 0], c.k[..., 0] = 20.0, 15.0
    c.q[..., 1:] *= 0.25
    c.fwd().bwd().check()
    assert c.lse.min() > 250


def test_longer_sequences(gpu):
    Call([700], [700], Hq=2, Hkv=1, D=64, dtype="f32", causal=1, scale=0.5).fwd().bwd().check()
    Call([900, 300], [1100, 300], Hq=2, Hkv=1, D=64, dtype="f32", causal=1, window=150).fwd().bwd().check()

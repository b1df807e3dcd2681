"""Rotary positions, attention and their gradients as a training step uses them together: the
transformer blocks with attention against the oracle in every ordering, captured, and in fp32."""
import numpy as np
import pytest

import oracle
import test_gpu_graphs as graphs
import test_gpu_training as training
from parity import rel
from workloads import make_batch, make_params, reduced_config

pytestmark = pytest.mark.gpu


def _window(gpu, cfg, s, progress):
    """One step of every ordering from the oracle's state after step s (forward-fusion from step s - 1 with
    step s's gradient pending): loss, m, v, values and each element's move, by the rules of the blocks
    without attention.  A bias of the keys' elements that do not turn has no gradient (it shifts every
    logit of a row alike: sum_j dS_ij = 0, so sum_j dk_j = sum_i (sum_j dS_ij) q_i = 0) and one of
    slowly turning elements a small one; what rounding leaves of them Adam scales up to whole steps,
    which those rules hold to the gradient the step itself computed."""
    import torch
    ref = oracle.run(cfg, "eager", steps=s + 1, snapshots={s - 1, s} if s else {0})
    start = ref["snapshots"][s]
    out = training._tblock_orderings(torch, gpu, cfg, start, prev=ref["snapshots"][s - 1] if s else None)
    training._tblock_check(cfg, out, start, ref, ref["losses"][s:], say=progress)
    return ref, out


@pytest.mark.parametrize("s", [0, 2])
def test_step_parity(gpu, progress, s):
    """bf16 operands, Q, K, V and the attention output stored as bf16."""
    _window(gpu, reduced_config("attn12"), s, progress)


@pytest.mark.parametrize("att", [dict(), dict(window=20), dict(rope=None, causal=False)], ids=str)
def test_fp32_step_parity(gpu, progress, att):
    """fp32 operands and storage, other masks: m, v and the loss within the fp32 workloads' tolerance."""
    cfg = reduced_config("attn12", dtype="f32")
    cfg["attention"].update(att)
    ref, out = _window(gpu, cfg, 1, progress)
    for st, loss in out.values():
        assert rel(loss, ref["losses"][1:]) <= training.TOL
        for k in ref["params"]:
            assert rel(st["m"][k], ref["m"][k]) <= training.TOL, k
            assert rel(st["v"][k], ref["v"][k]) <= training.TOL, k


@pytest.mark.parametrize("ordering", ["eager", "ff", "bf"])
def test_graph_replays_match_steps(gpu, ordering):
    graphs.test_graph_replays_match_steps(gpu, "attn12", ordering)


def test_one_step_against_unfused_orderings(gpu):
    """The full-size block (4 x 1024 rows, 16/4 heads of 64), one block deep: the orderings agree bit for
    bit where they run the same contractions."""
    import torch
    from paper_2104_00237_amd.trainer import Trainer
    from workloads import get_config
    cfg = dict(get_config("attn12"), blocks=1)
    out = []
    for o in ("eager", "bf"):
        tr = Trainer(cfg, make_params(cfg), gpu)
        for t in (1, 2):
            x, y = make_batch(cfg, t)
            tr.step(torch.as_tensor(x).to(gpu), torch.as_tensor(y).to(gpu), o)
        out.append((tr.state(), tr.loss_history()))
    np.testing.assert_array_equal(out[0][1], out[1][1])
    assert np.isfinite(out[0][1]).all()
    for k in out[0][0]["params"]:
        np.testing.assert_array_equal(out[0][0]["params"][k], out[1][0]["params"][k])

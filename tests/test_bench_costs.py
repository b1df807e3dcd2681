"""bench.py's accounting of a step, without a GPU: every launch class belongs to a stage, and attention is
part of the step's flops and bytes."""
import os
import re

import pytest

import bench
from workloads import get_config, reduced_config

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_launch_class_has_a_stage():
    src = open(os.path.join(ROOT, "paper_2104_00237_amd", "trainer.py")).read()
    classes = set(re.findall(r'\._t0\(\s*"(\w+)"', src)) | set(re.findall(r'start_after\(\s*"(\w+)"', src))
    assert {"fwd", "wgrad_bf", "attn"} <= classes
    stages = [c for cs in bench.STAGES.values() for c in cs]
    assert len(stages) == len(set(stages))
    assert classes == set(stages)


def _pairs(L, causal, window):
    return sum((not causal or j <= i) and (not window or abs(i - j) < window) for i in range(L) for j in range(L))


@pytest.mark.parametrize("att", [dict(causal=True, window=0), dict(causal=False, window=0), dict(causal=True, window=5),
                                 dict(causal=False, window=5), dict(causal=False, window=1), dict(causal=True, window=99),
                                 dict(causal=False, window=99, rope=None)], ids=str)
@pytest.mark.parametrize("ordering", ["eager", "ff", "bf"])
def test_a_step_with_attention_costs_its_products_and_rows(att, ordering):
    """What attn12's step costs over the same blocks with the identity in attention's place."""
    cfg = reduced_config("attn12")
    a = cfg["attention"] = dict(cfg["attention"], **att)
    H, Hk, L = a["heads"], a["kv_heads"], a["seq_len"]
    D, n, M = cfg["hidden"] // a["heads"], cfg["batch"] // a["seq_len"], cfg["batch"]
    plain = {**cfg, "attention": None}
    f1, b1 = bench.step_cost(cfg, ordering)
    # (the QKV linear is narrower with fewer key heads: cost of a plain block with this width)
    width = cfg["hidden"] + 2 * Hk * D
    wide = [d for d in bench.layer_launches(plain) if d["name"].endswith("qkv")]
    mine = [d for d in bench.layer_launches(cfg) if d["name"].endswith("qkv")]
    f0, b0 = bench.step_cost(plain, ordering)
    keys = {"eager": ("fwd", "dgrad", "wgrad"), "ff": ("fwd_ff", "dgrad", "wgrad"), "bf": ("fwd", "dgrad", "wgrad_bf")}
    for x, y in zip(wide, mine):
        assert y["N"] == width
        f0 += sum(y[k][0] - x[k][0] for k in keys[ordering])
        b0 += sum(y[k][1] - x[k][1] for k in keys[ordering])
        if ordering == "eager":
            b0 += (y["nparams"] - x["nparams"]) * 4 * (3 + 2 * bench.n_state(cfg["opt"]))
    flops = 14 * _pairs(L, a["causal"], a["window"]) * n * H * D
    qkv, o, stats = M * width, M * H * D, 4 * M * H
    moved = 2 * (2 * qkv + 2 * o) + 2 * stats + 4 * (o + qkv)    # q, k, v, o twice; dout, dq, dk, dv in fp32
    if a.get("rope"):
        turned = M * (H + Hk) * D
        flops += 2 * 3 * M * (H + Hk) * a["rope"]["rot"]
        moved += 2 * turned * 2 + 2 * turned * 4                  # in place: bf16, then the fp32 gradients
    assert f1 - f0 == cfg["blocks"] * flops
    assert b1 - b0 == cfg["blocks"] * moved


def test_the_record_names_the_attention():
    assert "causal attention 16/4 heads over 1024 rows" in bench.describe_layers(get_config("attn12"))
    assert "attention" not in bench.describe_layers(get_config("tblock12"))

"""bench.py's accounting of a step, without a GPU: every launch class belongs to a stage."""
import os
import re

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_launch_class_has_a_stage():
    src = open(os.path.join(ROOT, "paper_2104_00237_amd", "trainer.py")).read()
    classes = set(re.findall(r'\._t0\(\s*"(\w+)"', src)) | set(re.findall(r'start_after\(\s*"(\w+)"', src))
    assert {"fwd", "wgrad_bf", "attn"} <= classes
    stages = [c for cs in bench.STAGES.values() for c in cs]
    assert len(stages) == len(set(stages))
    assert classes == set(stages)

"""How the products whose ends are fused are cut into workgroups, at the ends of the
documented sizes: on the CPU for every cut, on a GPU for one whose rows lie at odd
addresses and whose smallest tiles would be more than a launch has."""
import os
import subprocess

import pytest
import torch

import fused_ref
from paper_2609_16389_amd import build
from paper_2609_16389_amd import xgemm as xg

_SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "host", "fused_cut.cpp")


def test_every_cut_can_be_launched(tmp_path):
    exe = str(tmp_path / "fused_cut")
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++20", "-I" + os.path.join(build.PKG, "csrc"), _SRC, "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, "%d cuts that cannot run, the first ones:\n%s" % (r.stdout.count("\n"), r.stdout[:2000])


@pytest.mark.gpu
def test_more_odd_columns_than_small_tiles():
    """16384 rows of 2 200 001 logits: 2^22 workgroups of the smallest tile are fewer."""
    T, V, H = 16384, 2200001, 17
    x, w = fused_ref.matrix(T, H, torch.bfloat16, 1), fused_ref.matrix(V, H, torch.bfloat16, 2, scale=0.5)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(3)).cuda()
    targets[5], targets[T - 1] = V - 1, -1
    out = xg.head_logprobs(x, w, targets)
    assert bool(out["lse"].isfinite().all())
    rows = torch.tensor([0, 1, 5, 63, 64, 255, 256, 8191, 12345, T - 2, T - 1], device="cuda")
    for name, (value, bound) in fused_ref.head(x[rows], w, targets[rows]).items():
        fused_ref.check(out[name][rows], value, bound, name)

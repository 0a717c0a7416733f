"""The built files: what runs without the binding's extension module, and what a failed build leaves."""
import os
import shutil
import subprocess
import sys

import pytest

import paper_2603_23198_amd
from paper_2603_23198_amd import build

PACKAGE = os.path.dirname(paper_2603_23198_amd.__file__)


@pytest.mark.parametrize("there", [None, "not a library"], ids=["missing", "broken"])
def test_the_layer_needs_only_the_library(tmp_path, there):
    """A tree with libsfl.so alone: the layer's entry points work, those that take checked tensors
    say what to run."""
    copy = tmp_path / "paper_2603_23198_amd"
    copy.mkdir()
    for name in ("__init__.py", "binding.py"):
        shutil.copy(os.path.join(PACKAGE, name), copy / name)
    os.symlink(os.path.join(PACKAGE, "libsfl.so"), copy / "libsfl.so")
    if there:
        (copy / "_marshal.so").write_text(there)
    program = """
import torch
from paper_2603_23198_amd import binding as b
print(b.__file__)
assert "gfx950" in b.sfl_version()
cfg = b.make_cfg()
assert b.sfl_twell_buffer_sizes(64, 256, "bf16", cfg)[0] > 0
x, i = torch.zeros(2, 8), torch.zeros((2, 2), dtype=torch.int32)
a = b.ffn_args(x, torch.zeros(8, 256), torch.zeros(256, 8), cfg)
b.sfl_forward_workspace_size(a)
assert b.sfl_expert_workspace_size(4000, 2, 8) > 0
for call in (lambda: b.sfl_norm_forward(x, x, X_out=x, N=x), lambda: b.sfl_route_forward(x, i, x),
             lambda: b.sfl_expert_dispatch(i, 8, i, i), lambda: b.grad_list([x])):
    try:
        call()
    except ImportError as e:
        assert "paper_2603_23198_amd.build" in str(e) and "_marshal" in str(e), e
    else:
        raise AssertionError("no ImportError")
print("ran to the end")
"""
    env = {n: v for n, v in os.environ.items() if n not in ("SFL_LIB", "PYTHONPATH")}
    r = subprocess.run([sys.executable, "-c", program], cwd=tmp_path, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    lines = r.stdout.split("\n")
    assert lines[0].startswith(str(tmp_path)) and lines[1] == "ran to the end"

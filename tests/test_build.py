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


@pytest.fixture
def targets(tmp_path, monkeypatch):
    """Build targets with old contents, and a source directory that compiles in a moment."""
    try:
        build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    for name in ("LIB", "MARSHAL"):
        (tmp_path / name).write_text("old")
        monkeypatch.setattr(build, name, str(tmp_path / name))
    src = tmp_path / "csrc"
    src.mkdir()
    (src / "one.cpp").write_text('extern "C" int one() { return 1; }\n')
    return tmp_path, src


def contents(path):
    return {p.name: p.read_bytes() == b"old" for p in path.iterdir() if p.is_file()}


def broken_command(monkeypatch, part):
    """The compiler's command line that has `part` in it gets an option that does not exist."""
    run = subprocess.run

    def run_or_break(cmd, **kw):
        return run([*cmd, "-fno-such-option-at-all"] if any(part in c for c in cmd) else cmd, **kw)

    monkeypatch.setattr(build.subprocess, "run", run_or_break)


@pytest.mark.parametrize("part", ["marshal.cpp", "one.cpp", "one.cpp.o"])
def test_a_failed_build_leaves_both_files_as_they_were(targets, monkeypatch, part):
    path, src = targets
    broken_command(monkeypatch, part)
    with pytest.raises(RuntimeError, match="failed"):
        build.build(csrc=str(src))
    assert contents(path) == {"LIB": True, "MARSHAL": True}


def test_a_build_replaces_both_files(targets):
    path, src = targets
    assert build.build(csrc=str(src)) == str(path / "LIB")
    assert contents(path) == {"LIB": False, "MARSHAL": False}


def test_a_library_elsewhere_leaves_the_extension_module(targets):
    path, src = targets
    build.build(csrc=str(src), out=str(path / "other"))
    assert contents(path) == {"LIB": True, "MARSHAL": True, "other": False}

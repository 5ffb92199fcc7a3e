"""The native reading of tensor lists (csrc/grad_list.cpp): when it is built anew, and which module the binding takes."""
import os
import shutil
import subprocess
import sys
import types

import pytest

from paper_2410_01623_b200 import build as fbuild

PKG = fbuild.PKG_DIR


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """Sources and outputs of the module in a folder of their own; the compiler is one that writes its output's name."""
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    shutil.copy(os.path.join(PKG, "csrc", "grad_list.cpp"), csrc)
    header = tmp_path / "fira.h"
    shutil.copy(os.path.join(os.path.dirname(PKG), "include", "fira.h"), header)
    out = tmp_path / os.path.basename(fbuild.LISTS_PATH)
    state = types.SimpleNamespace(csrc=csrc, header=header, out=out, runs=0, works=True)

    def compiler(cmd, **_):
        state.runs += 1
        if state.works:
            with open(cmd[cmd.index("-o") + 1], "w") as f:
                f.write(f"made {state.runs}")
        return types.SimpleNamespace(returncode=0 if state.works else 1, stdout="no")

    for name, value in dict(CSRC=str(csrc), HEADER=str(header), LISTS_PATH=str(out),
                            LISTS_KEY_PATH=str(tmp_path / "_build" / "key")).items():
        monkeypatch.setattr(fbuild, name, value, raising=False)
    monkeypatch.setattr(fbuild.subprocess, "run", compiler)
    return state


def test_it_is_built_once(tree):
    for _ in range(3):
        fbuild._build_lists(False)
    assert tree.runs == 1 and tree.out.read_text() == "made 1"
    fbuild._build_lists(True)
    assert tree.runs == 2 and tree.out.read_text() == "made 2"


@pytest.mark.parametrize("what", ["header", "source", "torch"])
def test_it_is_built_anew_where_what_it_is_made_from_has_changed(tree, monkeypatch, what):
    fbuild._build_lists(False)
    if what == "torch":
        import torch
        monkeypatch.setattr(torch, "__version__", "0.0.1")
    else:
        path = tree.header if what == "header" else tree.csrc / "grad_list.cpp"
        path.write_text(path.read_text() + "\n")
        os.utime(path, (1, 1))                 # (an older file of other contents, as a checkout may bring it)
    fbuild._build_lists(False)
    assert tree.runs == 2 and tree.out.read_text() == "made 2"


def test_a_build_that_fails_leaves_nothing_older(tree, capsys):
    fbuild._build_lists(False)
    untagged = tree.out.parent / "_native_lists.so"
    untagged.write_text("older still")
    tree.header.write_text(tree.header.read_text() + "\n")
    tree.works = False
    fbuild._build_lists(False)
    assert not tree.out.exists() and not untagged.exists()
    assert "not built" in capsys.readouterr().err


@pytest.fixture
def package(tmp_path):
    """The package's Python files alone."""
    to = tmp_path / "paper_2410_01623_b200"
    to.mkdir()
    for name in os.listdir(PKG):
        if name.endswith(".py"):
            shutil.copy(os.path.join(PKG, name), to)
    return to


def run(package, code):
    done = subprocess.run([sys.executable, "-c", code], cwd=package.parent, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout
    return done.stdout


USE = """
import sys, torch
from paper_2410_01623_b200 import binding as fb
name = "paper_2410_01623_b200._native_lists"
def use():
    assert fb._native_grad_list([torch.zeros(3)], None) is None        # (not on a CUDA device)
    try:
        fb.grad_norm([torch.zeros(3)])
    except ValueError as e:
        assert "CUDA" in str(e)
    else:
        assert False
use()
assert name not in sys.modules
"""


def test_a_module_that_is_built_later_is_used(package):
    fbuild.build()
    if not os.path.exists(fbuild.LISTS_PATH):
        pytest.skip("no compiler for it here")
    run(package, USE + f"""
import shutil
shutil.copy({fbuild.LISTS_PATH!r}, {str(package)!r})
use()
assert name in sys.modules and fb._native_grad_list is sys.modules[name].grad_list
""")


@pytest.mark.parametrize("change", ["desc_bytes", "torch_version", None])
def test_a_module_of_another_layout_is_not_used(package, change):
    attributes = "import torch\nfrom .binding import GradDesc, C\ntorch_version, desc_bytes = torch.__version__, C.sizeof(GradDesc)\n"
    if change:
        attributes += f"{change} = 7\n"
    # a stand-in written in Python, beside a file of the native module's name
    run(package, USE + f"""
open({str(package / "_native_lists.py")!r}, "w").write({attributes + "def grad_list(Gs, out): raise KeyError('used')"!r})
fb._LISTS_PATH = {str(package / "_native_lists.py")!r}
try:
    use()
    assert {change is not None}
except KeyError:
    assert {change is None}
""")

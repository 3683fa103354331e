"""The build of the binding's compiled argument checks: there where a compiler and the headers
are, and no condition for the library."""
import os
import shutil
import subprocess
import sys
import sysconfig

import pytest

from paper_2606_00395_amd import binding as B
from paper_2606_00395_amd import build


def toolchain():
    import torch
    headers = (os.path.join(sysconfig.get_paths()["include"], "Python.h"),
               os.path.join(os.path.dirname(torch.__file__), "include", "torch", "csrc", "Dtype.h"))
    return shutil.which("g++") and all(map(os.path.exists, headers))


def test_the_checks_are_built_with_the_library():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libpr2.so not built")
    if not toolchain():
        pytest.skip("no compiler or headers for the compiled checks")
    assert os.path.exists(build.ARGS)
    B._torch()
    assert type(B._need).__name__ == "builtin_function_or_method"


@pytest.mark.parametrize("command", [["/nonexistent/g++"], [sys.executable, "-c", "raise SystemExit('no header')"], None],
                         ids=["no_compiler", "does_not_compile", "no_torch"])
def test_the_library_is_built_without_them(tmp_path, monkeypatch, capsys, command):
    """The units compile to nothing here, in a folder of the test's: what is looked at is that
    the library is linked and that no older checks are left beside it."""
    def args_command(out):
        if command is None:
            raise ImportError("No module named 'torch'")
        return command

    def run(cmd):
        if "hipcc" not in cmd[0]:
            return plain(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return 0, ""

    plain = build._run
    for name in ("ARGS", "LIB", "BUILD"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    monkeypatch.setattr(build, "HIPCC", "hipcc")
    monkeypatch.setattr(build, "_args_command", args_command)
    monkeypatch.setattr(build, "_run", run)
    open(build.ARGS, "w").close()
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert not os.path.exists(build.ARGS) and not os.path.exists(build.ARGS + ".tmp")
    assert "not built" in capsys.readouterr().err


def test_the_binding_serves_without_them(tmp_path):
    """The same call refused by the Python checks in a process that has no compiled ones."""
    code = ("import sys, torch; sys.modules['paper_2606_00395_amd._args'] = None\n"
            "from paper_2606_00395_amd import binding as B\n"
            "B._torch(); print(type(B._need).__name__, B._need(torch.zeros(3), 'x', (3,)) > 0)\n"
            "try:\n    B._need(torch.zeros(3), 'x', (4,))\nexcept ValueError as e:\n    print(e)\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(B.HERE), stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("function True\nx has shape (3,)"), r.stdout

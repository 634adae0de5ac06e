"""CPU test: of C names the library exports only its own, iq_*; helper names as
plain as `overlap` could be taken over by a program that has one of its own."""

import shutil
import subprocess

import pytest

from paper_2608_08081_amd import _lib, build


def test_c_names():
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("no nm")
    _lib.lib()
    out = subprocess.run([nm, "-D", "--defined-only", f"{build.PKG}/{build.LIB_NAME}"],
                         capture_output=True, text=True, check=True).stdout
    code = [line.split()[-1] for line in out.splitlines() if line.split()[-2] == "T"]
    assert any(n.startswith("iq_") for n in code)
    plain = [n for n in code if not n.startswith(("iq_", "_Z", "_init", "_fini"))]
    assert not plain, plain

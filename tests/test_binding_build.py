"""The compiled module of the binding: what it is built for, and that nothing but its own calls needs it."""
import importlib
import subprocess
import sys
import sysconfig
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def build():
    from paper_2106_09886_b200 import build as b
    b.build()
    return b


def test_name_carries_the_abi_and_no_other_module_is_left(build):
    assert build.BINDING.name == "_binding" + sysconfig.get_config_var("EXT_SUFFIX") and "cpython" in build.BINDING.name
    assert build.BINDING.exists() and not build.needs_build()
    assert [p.name for p in build.PKG.glob("_binding*.so")] == [build.BINDING.name]


def test_another_torch_python_or_command_makes_the_module_stale_but_not_the_library(build, monkeypatch):
    library = build._digest()
    for target, name, value in ((importlib.metadata, "version", lambda _: "0.0.0"), (sys, "version", "0.0.0"),
                                (build, "_binding_command", lambda out: ["another", "command"])):
        with monkeypatch.context() as m:
            m.setattr(target, name, value)
            assert build._binding_stale() and build.needs_build() and build._digest() == library
    assert not build.needs_build()


def test_calls_without_the_module(build):
    """A process whose binding module cannot be loaded imports the package and makes the ctypes calls; a call on 4-bit weights
    says what is missing."""
    script = """
import sys
sys.modules["paper_2106_09886_b200._binding"] = None
from paper_2106_09886_b200 import qnn
assert qnn.version() > 0 and qnn.planes_bytes(4, 100, 2) > 0
import torch
w = qnn.G4Weights(torch.zeros((1, 1, 1, 4, 128, 4), dtype=torch.int32), torch.zeros((1, 1, 1, 4, 128), dtype=torch.uint8), torch.ones(1), 8, 64, 32)
try:
    qnn.g4_matvec(torch.zeros(2, 64), w)
except ImportError as exc:
    assert "paper_2106_09886_b200.build" in str(exc)
    print("refused")
"""
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and "refused" in r.stdout, r.stderr

"""The binding's module is compiled again for another PyTorch or interpreter, and refuses to work beside one it is not for."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def compiled(monkeypatch):
    """The sources that a build would compile for the module."""
    from paper_2608_28003_gb300 import build
    build.build()
    asked = []
    monkeypatch.setattr(build, "_compile_calls", asked.append)
    build.build()
    assert not asked  # up to date
    return build, asked


def test_another_torch(compiled, monkeypatch):
    build, asked = compiled
    monkeypatch.setattr(torch, "__version__", "2.99.0")
    build.build()
    assert [os.path.basename(s) for s in asked] == ["calls.cc"]


def test_the_same_version_of_another_build(compiled, monkeypatch):
    build, asked = compiled
    monkeypatch.setattr(torch.version, "git_version", "0" * 40)
    build.build()
    assert len(asked) == 1


def test_another_interpreter(compiled, monkeypatch):
    build, asked = compiled
    monkeypatch.setattr(sys, "version", "3.99.0")
    build.build()
    assert len(asked) == 1


def test_the_module_refuses_another_torch():
    from paper_2608_28003_gb300 import build
    build.build()
    program = ("import torch\nfrom paper_2608_28003_gb300 import binding as B\nassert B._calls()\nB._CALLS = None\n"
               "was, torch.__version__ = torch.__version__, '2.99.0'\n"
               "try:\n    B._calls()\n"
               "except ImportError as e:\n    assert was in str(e) and '2.99.0' in str(e) and 'build()' in str(e), e\n"
               "else:\n    raise SystemExit('taken')\n"
               "torch.__version__ = was\nassert B._calls()\n")
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr

"""What the extension module looks into tensors with is compiled against one torch's C++ objects: another torch, or another build of the same version,
has one of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

LOADS = """
import sys
import torch, torch.version
setattr(torch.version, sys.argv[1], sys.argv[2])
if sys.argv[1] == "__version__": torch.__version__ = sys.argv[2]
from paper_2504_14152_amd import build, fgmp
built, told = [], []
def build_tensors():
    built.append(1)
    raise RuntimeError("no compiler")
build.build_tensors = build_tensors
fgmp._load_tensors(type("Module", (), {"look_into_tensors": staticmethod(told.append)}))
print(build.tensors_are_stale(), len(built), len(told))
"""


def _version(name):
    import torch.version
    return getattr(torch.version, name)


@pytest.mark.parametrize("name,value,want", [("git_version", None, "False 0 1"), ("git_version", "0123456789abcdef", "True 1 0"), ("__version__", "local", "True 1 0"),
                                             ("__version__", "9.9.9", "True 1 0")])
def test_it_is_built_again_for_another_torch(name, value, want):
    from paper_2504_14152_amd import build
    if build.tensors_are_stale():
        build.build_tensors()
    if value == "local":
        value = _version("__version__").split("+")[0] + "+another"
    res = subprocess.run([sys.executable, "-c", LOADS, name, value or _version(name)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    assert res.stdout.split("\n")[-2] == want

"""The build's decisions, with the compilers replaced by something that only writes the files it is asked for."""
import importlib.util
import os

import pytest

from paper_1310_4645_b200 import build as B


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """Every command the build runs; outputs go to tmp_path."""
    ran = []

    def run(cmd, *a, **k):
        ran.append([str(c) for c in cmd])
        with open(cmd[list(cmd).index("-o") + 1], "w") as f:
            f.write("built")

    monkeypatch.setattr(B.subprocess, "check_call", run)
    monkeypatch.setattr(B, "LIB", str(tmp_path / "librd.so"))
    monkeypatch.setattr(B, "TORCH_LIB", str(tmp_path / "_rd_torch.so"))
    return ran


def without_torch(monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))


def test_both_libraries_are_built(compilers):
    assert B.stale()
    assert B.build() == B.LIB
    assert os.path.exists(B.LIB) and os.path.exists(B.TORCH_LIB) and not B.stale()
    count = len(compilers)
    B.build()
    assert len(compilers) == count


def test_the_c_library_needs_no_torch(compilers, monkeypatch):
    without_torch(monkeypatch)
    assert B.build() == B.LIB
    assert os.path.exists(B.LIB) and not os.path.exists(B.TORCH_LIB) and not B.stale()
    assert not any("rd_torch" in word for cmd in compilers for word in cmd)


def test_the_c_library_outlives_a_failure_of_the_tensor_module(compilers, monkeypatch):
    run = B.subprocess.check_call

    def fail(cmd, *a, **k):
        if any("rd_torch" in str(word) for word in cmd):
            raise B.subprocess.CalledProcessError(1, cmd)
        return run(cmd, *a, **k)

    monkeypatch.setattr(B.subprocess, "check_call", fail)
    with pytest.raises(B.subprocess.CalledProcessError):
        B.build()
    assert os.path.exists(B.LIB) and not os.path.exists(B.TORCH_LIB) and B.stale()


def test_another_torch_means_another_tensor_module(compilers, monkeypatch, tmp_path):
    """A torch whose version differs from the one that _rd_torch.so was built against, whatever the files' times say."""
    torch_dir = tmp_path / "torch"
    (torch_dir / "lib").mkdir(parents=True)
    (torch_dir / "lib" / "libc10_cuda.so").write_text("")
    (torch_dir / "version.py").write_text("__version__ = '2.11.0+cu128'\n")
    spec = importlib.util.spec_from_loader("torch", None)
    spec.submodule_search_locations = [str(torch_dir)]
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: spec if name == "torch" else find(name, *a))
    B.build()
    assert not B.stale()
    (torch_dir / "version.py").write_text("__version__ = '2.12.0+cu128'\n")
    for f in (torch_dir / "version.py", torch_dir / "lib" / "libc10_cuda.so"):
        os.utime(f, (1, 1))                                   # an installer keeps the files' own, older times
    assert B.stale()
    B.build()
    assert not B.stale()

"""What the build takes for up to date, and that a build that fails leaves nothing behind."""
import os
import subprocess
import time

import pytest
import torch

from paper_2609_09721_b200 import binding, build


def test_another_torch_makes_the_extension_stale(monkeypatch):
    """efq_tensorcall.so is compiled against torch's C++ headers: the files' times alone do not tell whether it still fits."""
    build.build()
    assert not build._stale()
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    assert build._stale()


def test_an_extension_of_another_torch_is_not_called(monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_tensors", None)
    assert binding._tensorcall().built_for == build.target()
    monkeypatch.setattr(binding, "_tensors", None)
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    with pytest.raises(RuntimeError, match="was built for torch .* this is torch 9.9.9"):
        binding._tensorcall()


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """A build of one source into a folder of its own, by compilers that are scripts: what they leave is theirs to say."""
    def script(name, text):
        path = tmp_path / name
        path.write_text("#!/bin/sh\nfor last; do if [ \"$was\" = -o ]; then out=$last; fi; was=$last; done\n" + text)
        path.chmod(0o755)
        return str(path)

    (tmp_path / "one.cu").write_text("")
    for name, file in (("LIB", "lib.so"), ("FASTCALL", "fast.so"), ("TENSORCALL", "tensor.so"), ("BUILT_FOR", "built_for")):
        monkeypatch.setattr(build, name, str(tmp_path / file))
    monkeypatch.setattr(build, "_HERE", str(tmp_path))
    monkeypatch.setattr(build, "sources", lambda: [str(tmp_path / "one.cu")])
    monkeypatch.setenv("CC", script("cc", "echo > $out\n"))
    return tmp_path, script


def _left(folder):
    return sorted(x for x in os.listdir(folder) if ".tmp" in x or x.endswith(".so"))


def test_a_failed_library_leaves_nothing_running(elsewhere, monkeypatch):
    folder, script = elsewhere
    monkeypatch.setattr(build, "NVCC", script("nvcc", "exit 1\n"))
    monkeypatch.setenv("CXX", script("cxx", f"echo > $out; echo $$ > {folder}/pid; exec sleep 60\n"))
    started = time.time()
    real = subprocess.Popen

    def slowly(cmd, *args, **more):             # the extension's compiler is at work when the library's fails
        p = real(cmd, *args, **more)
        while cmd[0].endswith("cxx") and not os.path.exists(folder / "pid"):
            time.sleep(0.01)
        return p

    monkeypatch.setattr(subprocess, "Popen", slowly)
    with pytest.raises(RuntimeError, match="nvcc failed"):
        build.build(force=True)
    assert time.time() - started < 30 and _left(folder) == []
    with pytest.raises(ProcessLookupError):
        os.kill(int((folder / "pid").read_text()), 0)


def test_a_failed_extension_leaves_the_library(elsewhere, monkeypatch):
    folder, script = elsewhere
    monkeypatch.setattr(build, "NVCC", script("nvcc", "echo > $out\n"))
    monkeypatch.setenv("CXX", script("cxx", "echo > $out; exit 1\n"))
    with pytest.raises(RuntimeError, match="cxx failed"):
        build.build(force=True)
    assert _left(folder) == ["fast.so", "lib.so"] and build._stale()
    monkeypatch.setenv("CXX", script("cxx", "echo > $out\n"))
    build.build()
    assert _left(folder) == ["fast.so", "lib.so", "tensor.so"] and not build._stale()

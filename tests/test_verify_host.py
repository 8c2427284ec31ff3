"""Host-side logic of the verification-step operators' package, without a GPU."""
import contextlib
import os
import subprocess
import types

import pytest
import torch

from paper_2410_03960_b200 import build, verify


@pytest.mark.parametrize("device,stream_on,want", [(None, None, 3), ("cuda", None, 3), (torch.device("cuda"), None, 3), ("cuda:1", None, 1), (2, None, 2), ("cuda:0", None, 0),
                                                   (None, 5, 5), ("cuda", 5, 5), ("cuda:5", 5, 5)])
def test_op_status_asks_the_device_that_is_meant(monkeypatch, device, stream_on, want):
    """A device without a number is the current one (3 here), not the first."""
    asked = []

    @contextlib.contextmanager
    def made_current(index):
        asked.append(index)
        yield

    streams = {i: types.SimpleNamespace(cuda_stream=100 + i, device_index=i) for i in range(6)}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "device", made_current)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: streams[asked[-1]])
    monkeypatch.setattr(verify, "load_library", lambda: types.SimpleNamespace(swiftkv_op_status=lambda s: asked.append(s) or 0))
    verify.op_status(device, stream=None if stream_on is None else streams[stream_on])
    assert asked == [want, 100 + want]


def test_op_status_refuses_a_stream_of_another_device():
    with pytest.raises(ValueError):
        verify.op_status("cuda:0", stream=types.SimpleNamespace(cuda_stream=1, device_index=1))


class Compilers:
    """Stands in for subprocess.run: notes the commands, lets those of one compiler fail."""

    def __init__(self, failing=None):
        self.commands, self.failing = [], failing

    def __call__(self, cmd, **kw):
        self.commands.append(cmd)
        bad = self.failing is not None and os.path.basename(cmd[0]) == self.failing
        return types.SimpleNamespace(returncode=int(bad), stdout="", stderr="")

    def names(self):
        return [os.path.basename(c[0]) for c in self.commands]


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    run = Compilers()
    monkeypatch.setattr(subprocess, "run", run)
    monkeypatch.setenv("SWIFTKV_BUILD_LOG_DIR", str(tmp_path))
    return run


def test_the_library_is_built_before_the_extension_and_without_it(compilers):
    assert build.build_library(force=True) == build.LIB and compilers.names() == ["nvcc"]
    compilers.commands.clear()
    compilers.failing = "g++"
    with pytest.raises(RuntimeError):
        build.build(force=True)
    assert compilers.names() == ["nvcc", "g++"]


def test_the_extension_takes_the_headers_beside_nvcc(compilers, monkeypatch, tmp_path):
    (tmp_path / "cuda" / "bin").mkdir(parents=True)
    nvcc = tmp_path / "cuda" / "bin" / "nvcc"
    nvcc.write_text("")
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    build.build_ext()
    assert f"-I{tmp_path / 'cuda' / 'include'}" in compilers.commands[-1] and "-I/usr/local/cuda/include" not in compilers.commands[-1]


def test_the_extension_is_stale_where_torch_is_newer(monkeypatch, tmp_path):
    ext, version = tmp_path / "_verify.so", tmp_path / "version.py"
    for i, f in enumerate((ext, version)):
        f.write_text("")
        os.utime(f, (4e9 + 100 * i,) * 2)
    monkeypatch.setattr(build, "EXT", str(ext))
    monkeypatch.setattr(build, "_torch_version_file", lambda: str(version))
    assert build._ext_stale()
    os.utime(ext, (4e9 + 300,) * 2)
    assert not build._ext_stale()


def test_an_extension_of_another_torch_is_refused(monkeypatch):
    build.build()
    monkeypatch.setattr(verify, "_EXT", None)
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    with pytest.raises(RuntimeError, match="built for torch"):
        verify._load()
    monkeypatch.undo()
    assert verify._load().built_for_torch == torch.__version__

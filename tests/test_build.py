"""What the build does when a compiler fails, with the compilers' part played by a stand-in: no GPU."""
import os
import subprocess

import pytest

from paper_2512_12928_b200 import build as ps_build


class Compilers:
    """Stands in for subprocess.run: writes the output file, or fails."""

    def __init__(self):
        self.ran, self.failing = [], ()

    def __call__(self, cmd, **kw):
        name = os.path.basename(cmd[0])
        self.ran.append(name)
        out = cmd[cmd.index("-o") + 1]
        with open(out, "w") as f:
            f.write("half" if name in self.failing else " ".join(self.ran))
        return subprocess.CompletedProcess(cmd, 1 if name in self.failing else 0, "stand-in")


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    c = Compilers()
    monkeypatch.setattr(ps_build, "LIB_DIR", str(tmp_path))
    monkeypatch.setattr(ps_build, "LIB_PATH", str(tmp_path / "libps_kvswap.so"))
    monkeypatch.setattr(ps_build, "TENSOR_ARGS_PATH", str(tmp_path / "_ps_tensor_args.so"))
    monkeypatch.setattr(ps_build, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    monkeypatch.setattr(ps_build.shutil, "which", lambda name: "/usr/bin/" + name)
    monkeypatch.setattr(ps_build.subprocess, "run", c)
    return c


def test_the_library_is_built_where_the_module_fails(compilers, tmp_path):
    compilers.failing = ("g++",)
    with pytest.raises(RuntimeError, match="g.. failed"):
        ps_build.build()
    assert compilers.ran == ["nvcc", "g++"] and "libps_kvswap.so" in os.listdir(tmp_path)


def test_torch_without_cuda_needs_no_module(compilers, monkeypatch, tmp_path):
    import torch
    monkeypatch.setattr(torch.version, "cuda", None)
    assert ps_build.build() == str(tmp_path / "libps_kvswap.so")
    assert compilers.ran == ["nvcc"] and os.listdir(tmp_path) == ["libps_kvswap.so"]

"""What the build does when a compiler fails or torch changes, with the compilers' part played by a stand-in: no GPU."""
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
    monkeypatch.setattr(ps_build, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    monkeypatch.setattr(ps_build.shutil, "which", lambda name: "/usr/bin/" + name)
    monkeypatch.setattr(ps_build.subprocess, "run", c)
    return c


def test_the_library_is_built_where_the_module_fails(compilers, tmp_path):
    compilers.failing = ("g++",)
    with pytest.raises(RuntimeError, match="g.. failed"):
        ps_build.build()
    assert compilers.ran == ["nvcc", "g++"] and os.listdir(tmp_path) == ["libps_kvswap.so"]


def test_torch_without_cuda_needs_no_module(compilers, monkeypatch, tmp_path):
    import torch
    monkeypatch.setattr(torch.version, "cuda", None)
    assert ps_build.build() == str(tmp_path / "libps_kvswap.so")
    assert compilers.ran == ["nvcc"] and os.listdir(tmp_path) == ["libps_kvswap.so"]


def test_the_module_is_of_one_torch_and_one_python(compilers, monkeypatch):
    import sysconfig

    import torch
    first = ps_build.build_tensor_args()
    assert ps_build.build_tensor_args() == first == ps_build.tensor_args_path() and compilers.ran == ["g++"]
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    second = ps_build.build_tensor_args()
    assert second != first and compilers.ran == ["g++"] * 2
    monkeypatch.setattr(sysconfig, "get_config_var", lambda name: ".cpython-399.so")
    assert ps_build.build_tensor_args() not in (first, second) and compilers.ran == ["g++"] * 3


def test_a_failed_or_unfinished_module_replaces_nothing(compilers, tmp_path):
    path = ps_build.build_tensor_args()
    was = open(path).read()
    compilers.failing = ("g++",)
    with pytest.raises(RuntimeError):
        ps_build.build_tensor_args(force=True)
    assert open(path).read() == was and os.listdir(tmp_path) == [os.path.basename(path)]


def test_the_binding_looks_for_this_torchs_module(compilers, monkeypatch):
    from paper_2512_12928_b200 import binding as B
    monkeypatch.setattr(B, "_tensor_args", None)
    with pytest.raises(ImportError, match="is missing: build it with"):
        B.ps_build_slots(*[None] * 7, block_size=1, num_gpu_blocks=1)

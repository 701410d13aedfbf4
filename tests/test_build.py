"""What the build makes, in which order, and when it makes it again.  The compilers are replaced; no GPU needed."""
import subprocess
import sys

import pytest

from paper_2411_02581_b200 import build as build_mod


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """Commands that the build runs, each making its output; those whose program is in `broken` fail."""
    ran, broken = [], set()

    def check_call(cmd, **kw):
        ran.append("g++" if cmd[0] == "g++" else "nvcc")
        if ran[-1] in broken:
            raise FileNotFoundError(cmd[0])
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(build_mod.subprocess, "check_call", check_call)
    monkeypatch.setattr(build_mod, "LIB_DIR", str(tmp_path))
    monkeypatch.setattr(build_mod, "LIB_PATH", str(tmp_path / "libtuna.so"))
    monkeypatch.setattr(build_mod, "TORCH_PATH", str(tmp_path / "tuna_torch.so"))
    return ran, broken, tmp_path


def test_library_is_built_where_the_marshalling_cannot_be(commands):
    ran, broken, where = commands
    broken.add("g++")
    with pytest.warns(RuntimeWarning, match="marshalling"):
        assert build_mod.build() == str(where / "libtuna.so")
    assert (where / "libtuna.so").exists() and not (where / "tuna_torch.so").exists()


def test_library_is_built_without_torch():
    code = ("import subprocess, sys, tempfile, os\n"
            "class NoTorch:\n"
            "    def find_spec(self, name, path=None, target=None):\n"
            "        if name.split('.')[0] == 'torch': raise ModuleNotFoundError(name)\n"
            "sys.meta_path.insert(0, NoTorch())\n"
            "import importlib.util\n"
            "real = importlib.util.find_spec\n"
            "importlib.util.find_spec = lambda name, *a: None if name == 'torch' else real(name, *a)\n"
            "from paper_2411_02581_b200 import build as b\n"
            "d = tempfile.mkdtemp(); b.LIB_DIR = d; b.LIB_PATH = d + '/l.so'; b.TORCH_PATH = d + '/t.so'\n"
            "b.subprocess.check_call = lambda cmd, **kw: open(cmd[cmd.index('-o') + 1], 'w').close()\n"
            "b.build(); print('made', os.listdir(d), 'torch' in sys.modules)\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=build_mod.ROOT)
    assert r.returncode == 0 and "made ['l.so'] False" in r.stdout, (r.stdout, r.stderr)


def test_marshalling_is_built_again_for_another_torch(commands, monkeypatch):
    ran, _, where = commands
    build_mod.build()
    assert ran == ["nvcc", "g++"]
    build_mod.build()
    assert ran == ["nvcc", "g++"]                      # everything is there
    import torch
    monkeypatch.setattr(torch, "__version__", "0.0+another")
    build_mod.build()
    assert ran == ["nvcc", "g++", "g++"]


def test_failed_marshalling_leaves_no_old_one(commands, monkeypatch):
    ran, broken, where = commands
    build_mod.build()
    import torch
    monkeypatch.setattr(torch, "__version__", "0.0+another")
    broken.add("g++")
    with pytest.warns(RuntimeWarning):
        build_mod.build()
    assert not (where / "tuna_torch.so").exists()
    from paper_2411_02581_b200 import moe
    monkeypatch.setattr(moe, "_marshal", None)
    with pytest.raises(RuntimeError, match="is missing: build it"):
        moe._fast()

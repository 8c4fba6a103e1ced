"""What build() compiles, by what is installed: the commands alone, nothing is run."""
import importlib
import sys
import types

import pytest

hip_build = importlib.import_module("paper_2606_01556_amd.build")


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """The commands of a build into an empty directory."""
    ran = []

    def run(cmd, check):
        assert check
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(hip_build.subprocess, "run", run)
    monkeypatch.setattr(hip_build, "LIB", str(tmp_path / "libtq.so"))
    monkeypatch.setattr(hip_build, "BINDING", str(tmp_path / "_tqtorch.so"))
    return ran


def built(tmp_path):
    return sorted(p.name for p in tmp_path.iterdir())


def test_library_without_torch(commands, monkeypatch, tmp_path, capsys):
    """The C library needs neither torch nor its headers."""
    monkeypatch.setitem(sys.modules, "torch", None)          # import raises ImportError
    assert hip_build.build() == hip_build.LIB
    assert len(commands) == 1 and commands[0][0] == hip_build.HIPCC and built(tmp_path) == ["libtq.so"]
    assert "without _tqtorch.so" in capsys.readouterr().out


def test_library_beside_another_torch(commands, monkeypatch, tmp_path):
    other = types.ModuleType("torch")
    other.version = types.SimpleNamespace(hip=None)
    monkeypatch.setitem(sys.modules, "torch", other)
    hip_build.build()
    assert len(commands) == 1 and built(tmp_path) == ["libtq.so"]


def test_both(commands, tmp_path):
    torch = pytest.importorskip("torch")
    if torch.version.hip is None:
        pytest.skip("torch is not built for ROCm")
    hip_build.build()
    assert [c[0] for c in commands] == [hip_build.HIPCC, hip_build.CXX] and built(tmp_path) == ["_tqtorch.so", "libtq.so"]

"""The C library is built and loaded where `_marshal.so` cannot be; what was built for another torch is built again."""
import os
import subprocess
import sys

import pytest

from paper_2603_05035_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def apart(tmp_path, monkeypatch):
    """`_marshal.so` and what it was built for, somewhere else, after the library itself is up to date."""
    build.build()
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(build, "MARSHAL_FOR", str(tmp_path / "marshal.for"))
    return tmp_path


def test_library_is_built_without_torch(apart, monkeypatch, capfd):
    monkeypatch.setattr(build, "_torch_dir", lambda: None)
    (apart / "_marshal.so").write_text("of a torch that is gone")
    assert os.path.exists(build.build())
    assert not os.path.exists(build.MARSHAL) and "for want of torch" in capfd.readouterr().err


def test_library_is_built_without_headers(apart, monkeypatch, capfd):
    monkeypatch.setattr(build, "_torch_dir", lambda: str(apart))
    assert os.path.exists(build.build())
    assert not os.path.exists(build.MARSHAL) and "CUDAStream.h" in capfd.readouterr().err


def test_marshalling_is_built_again_for_another_torch(apart, monkeypatch):
    made = []

    def compiler(cmd, **_):
        made.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build.subprocess, "run", compiler)
    build.build()
    build.build()
    assert len(made) == 1
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "another")
    build.build()
    build.build()
    assert len(made) == 2


def test_library_is_loaded_without_the_marshalling():
    """Calls that do not go through it work, the others say what is missing."""
    code = """
import sys
sys.modules["paper_2603_05035_b200._marshal"] = None
from paper_2603_05035_b200 import binding
assert binding.load_library().gelo_mixing_ld(68) == 128
try:
    binding._marshal.rms_norm(0)
except ImportError as e:
    print(e)
"""
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "rms_norm needs _marshal.so" in run.stdout, run.stdout + run.stderr

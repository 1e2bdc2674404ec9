"""The marshalling lets go of Python's lock while the library launches.

A stand-in for the library, which says whether the calling thread holds the lock, takes its place beside a copy of the module in a process of its own."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2603_05035_b200 import binding

pytestmark = pytest.mark.gpu

CALLS = ("gelo_rms_norm", "gelo_project_e4m3_rows", "gelo_rotary", "gelo_append_kv", "gelo_paged_attention")
SCRIPT = """
import ctypes, importlib.util, sys
import torch
sys.path.insert(0, sys.argv[2])
from paper_2603_05035_b200 import binding                 # structures only: the library is not loaded
spec = importlib.util.spec_from_file_location("_marshal", sys.argv[1])
m = importlib.util.module_from_spec(spec)
spec.loader.exec_module(m)
x = torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda")
i = torch.zeros(2, dtype=torch.int32, device="cuda")
f = torch.ones(2, device="cuda")
u8 = torch.zeros((2, 64), dtype=torch.uint8, device="cuda")
w8 = torch.zeros((64, 64), dtype=torch.uint8, device="cuda")
pages = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
cache = binding.PagedCache(pages, pages, torch.zeros((2, 1), dtype=torch.int32, device="cuda"))
held = [m.rms_norm(1, 0, x, x, None, 1e-5, None, None, None, None, None),
        m.project_e4m3_rows(1, 0, u8, f, w8, f[:1], 2, 64, 64, x, None),
        m.rotary(1, 0, x, 1, i, 0, None, None),
        m.append_kv(1, 0, cache.ref, x, x, i, None, None, None, None, None),
        m.paged_attention(1, 0, cache.ref, x, i, x, 0.1, 0, None, None)]
assert held == [0] * 5, held
print("let go of")
"""


def test_the_lock_is_let_go_of_during_a_launch(tmp_path):
    source, script = tmp_path / "stand_in.cpp", tmp_path / "run.py"
    source.write_text('extern "C" int PyGILState_Check(void);\n' + "".join(f'extern "C" int {name}() {{ return PyGILState_Check(); }}\n' for name in CALLS))
    subprocess.run(["g++", "-shared", "-fPIC", "-o", str(tmp_path / "libgelo.so"), str(source)], check=True)
    script.write_text(SCRIPT)
    here = os.path.dirname(binding.library_path())
    shutil.copy(os.path.join(here, "_marshal.so"), tmp_path / "_marshal.so")
    run = subprocess.run([sys.executable, str(script), str(tmp_path / "_marshal.so"), os.path.dirname(here)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "let go of" in run.stdout, run.stdout + run.stderr

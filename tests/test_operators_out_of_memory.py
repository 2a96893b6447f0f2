"""Host memory that runs out in a call of the log probabilities or the orthogonalised
updates gives SB_ENOMEM: no exception leaves the C entry.  In a process of its own,
whose operator new fails while a flag is set; the calls are ones that would be
refused, so nothing is launched either way."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

import pytest

b = pytest.importorskip("paper_2011_12025_amd._binding")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NEW = r"""
#include <cstdlib>
#include <new>
extern "C" { int new_fails = 0; int new_calls = 0; }
void* operator new(std::size_t n) {
    if (new_fails) { ++new_calls; throw std::bad_alloc(); }
    if (void* p = std::malloc(n ? n : 1)) return p;
    throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
"""

CALLS = r"""
import ctypes, os, sys
sys.path.insert(0, {root!r})
from paper_2011_12025_amd import _binding as b
lib, new = b.lib(), ctypes.CDLL({so!r})
fails, calls = ctypes.c_int.in_dll(new, "new_fails"), ctypes.c_int.in_dll(new, "new_calls")
p = lambda i: ctypes.c_void_p(0x100000000 * (i + 1))
m = b.Matrix(p(0).value, p(0).value, 1, 64, 576, 576, 576, 0, 0)
c, n = (ctypes.c_double * 3)(1.0, 0.0, 0.0), ctypes.c_size_t(0)
entries = {{
    "segblocks_log_probs": lambda: lib.segblocks_log_probs(p(0), 1, 1, 4, 19, 8, 8, 24, p(1), 255, 0, p(2), p(2), None, None, None,
                                                           None, 0, None),
    "segblocks_log_probs refused": lambda: lib.segblocks_log_probs(p(0), 9, 1, 4, 19, 8, 8, 24, p(1), 255, 0, p(2), p(2), None,
                                                                   None, None, None, 0, None),
    "segblocks_log_probs_workspace_size": lambda: lib.segblocks_log_probs_workspace_size(9, 1, 4, 19, 8, 8, 24, 0, ctypes.byref(n)),
    "segblocks_log_probs_backward": lambda: lib.segblocks_log_probs_backward(p(0), 1, 1, 4, 19, 8, 8, 24, p(1), 255, p(2), p(3),
                                                                             None, None, 0, None, None, 24, p(0), None),
    "segblocks_orthogonalize": lambda: lib.segblocks_orthogonalize(ctypes.pointer(m), 1, 1, 1, c, 0.0, p(5), 1 << 40, None),
    "segblocks_orthogonalize_workspace_size": lambda: lib.segblocks_orthogonalize_workspace_size(ctypes.pointer(m), 1, 1,
                                                                                                 ctypes.byref(n)),
}}
for name, call in entries.items():
    before = calls.value
    fails.value = 1
    code = call()
    fails.value = 0
    print(name, code, calls.value > before, flush=True)
    assert code == -4 and calls.value > before, name
    assert call() != -4, name
print("done")
"""


def test_no_exception_leaves_the_entries(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src, so = tmp_path / "new.cpp", tmp_path / "libnew.so"
    src.write_text(NEW)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", str(src), "-o", str(so)], check=True)
    # (no device is seen: the calls end before any would be used)
    preload = " ".join(filter(None, [os.environ.get("LD_PRELOAD"), str(so)]))
    env = dict(os.environ, LD_PRELOAD=preload, HIP_VISIBLE_DEVICES="-1")
    run = subprocess.run([sys.executable, "-c", CALLS.format(root=ROOT, so=str(so))], env=env, capture_output=True, text=True,
                         timeout=300)
    assert run.returncode == 0 and run.stdout.endswith("done\n"), (run.returncode, run.stdout, run.stderr[-600:])

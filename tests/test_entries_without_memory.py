"""Calls of the library whose host memory has run out: no GPU is needed, nothing is launched."""
import os
import subprocess

import paper_1801_00829_amd as F


def test_no_exception_leaves_an_entry_without_memory(tmp_path):
    """Host memory that has run out where a call says what it refuses (no_memory_at_entry.cpp)."""
    exe, root, lib = str(tmp_path / "no_memory_at_entry"), os.path.dirname(os.path.abspath(__file__)), F.lib_path()
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", os.path.join(root, "no_memory_at_entry.cpp"), "-L" + os.path.dirname(lib), "-l:libfuse.so",
                    "-o", exe, "-Wl,-rpath," + os.path.dirname(lib), "-Wl,-rpath,/opt/rocm/lib", "-L/opt/rocm/lib", "-Wl,-rpath-link,/opt/rocm/lib"], check=True)
    r = subprocess.run([exe], timeout=120, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)

"""C++ programs against the library's own headers and internals, compiled for the host alone and run without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2609_12378_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

HEAD = r"""
#include <cmath>
#include <cstdio>
#include <cstring>
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
"""


def run(tmp_path, text, *args):
    """The program's output; it fails by a status that is not 0."""
    from paper_2609_12378_amd import LIB_PATH, build as b
    if not os.path.exists(LIB_PATH):
        b.build()
    src, exe = tmp_path / "main.hip", str(tmp_path / "main")
    src.write_text(HEAD + text)
    subprocess.run([b.hipcc(), "-O1", "-std=c++17", "-Wall", "-Wno-unused-function", "--offload-host-only",
                    "-I", os.path.join(ROOT, "include"), "-I", b.CSRC, "-c", str(src), "-o", exe + ".o"], check=True,
                   capture_output=True, text=True)
    subprocess.run([b.hipcc(), exe + ".o", "-L", PKG, "-lckks_mi", "-Wl,-rpath," + PKG,
                    "-Wl,-rpath," + os.path.join(ROCM, "lib"), "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    return r.stdout

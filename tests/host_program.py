"""Small C++ programs over the library's host code, for tests without a GPU: what lies behind the C-ABI and asks
the CUDA runtime nothing."""
import os
import subprocess

from paper_2609_32046_gb300 import build as b


def run(tmp_path, source: str, objects=()) -> list:
    """Compile `source` (which may include the library's headers) with the library's objects, run it, and return
    its output's lines."""
    objs = [os.path.join(b.BUILD_DIR, o + ".o") for o in objects]
    b.build(force=not all(map(os.path.exists, objs)))
    src, exe = str(tmp_path / "program.cu"), str(tmp_path / "program")
    with open(src, "w") as f:
        f.write(source)
    res = subprocess.run([b.nvcc(), *b.NVCC_FLAGS, "-o", exe, src, *objs], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    return res.stdout.split("\n")[:-1]

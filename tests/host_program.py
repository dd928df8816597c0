"""Compiles a C++ program against the library's internal headers and runs it here: host-side rules of the kernels, checked
without a GPU (the programs make no CUDA call)."""
import os
import subprocess

from paper_2405_01943_b200 import build


def run(tmp_path, text, flags=()):
    """The program's exit code and output."""
    src, exe = os.path.join(tmp_path, "program.cu"), os.path.join(tmp_path, "program")
    with open(src, "w") as f:
        f.write(text)
    cmd = [os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "static", *flags,
           "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, src, "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    return res.returncode, res.stdout

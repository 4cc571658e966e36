"""Several C threads on one context (tests/c_threads.c): between Python's threads the interpreter's lock leaves no two calls at quite the
same time. Compiled on CPU machines too, run where a GPU exists."""
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")


def build_program(tmp_path):
    from paper_2609_34162_b200.build import build
    lib, exe = build(), str(tmp_path / "c_threads")
    subprocess.run(["gcc", "-std=c99", "-O1", "-Wall", "-o", exe, os.path.join(ROOT, "tests", "c_threads.c"), "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(CUDA, "include"), lib, "-L", os.path.join(CUDA, "lib64"), "-lcudart", "-lpthread",
                    f"-Wl,-rpath,{os.path.dirname(lib)}", f"-Wl,-rpath,{os.path.join(CUDA, 'lib64')}"], check=True)
    return exe


def test_the_program_links(tmp_path):
    assert os.path.exists(build_program(tmp_path))


@pytest.mark.gpu
def test_block_norms_of_several_widths_in_several_threads(tmp_path):
    """Widths and sets of inputs that one kernel serves with different amounts of shared memory."""
    assert torch.cuda.is_available()
    r = subprocess.run([build_program(tmp_path)], capture_output=True, text=True, timeout=300)
    print(r.stdout, r.stderr)
    assert r.returncode == 0 and r.stdout.startswith("PASS"), r.stdout + r.stderr

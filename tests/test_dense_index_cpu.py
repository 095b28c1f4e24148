"""The indices of the dense product's epilogue on the host (tests/dense_index.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_element_of_a_part(tmp_path):
    exe = str(tmp_path / "dense_index")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2401_14110_amd", "csrc"),
                    os.path.join(ROOT, "tests", "dense_index.cpp"), "-o", exe], check=True)
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0 and "indices ok" in run.stdout, run.stdout[-2000:]

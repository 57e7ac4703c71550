"""How a wave divides a short row of logits, gone through on the host: every division leaves fewer of them, also where the distances to the largest are
all the same in 64 bits, and what is found is the nth of the order."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_divisions_of_a_row_end(tmp_path):
    exe = str(tmp_path / "sample_bins")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", os.path.join(ROOT, "paper_1907_07346_amd", "csrc"),
                    os.path.join(ROOT, "tests", "sanitize", "sample_bins_cases.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    sys.stdout.write(out.stdout)
    assert out.returncode == 0, out.stdout[-2000:]
    assert "sample bins ok" in out.stdout

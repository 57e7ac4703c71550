"""The products' reads of a message, gone through on the host for every block size and for widths around every border: none leaves its row,
and each brings the words that it should."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_reads_stay_inside_their_rows(tmp_path):
    exe = str(tmp_path / "message_reads")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", os.path.join(ROOT, "paper_1907_07346_amd", "csrc"),
                    os.path.join(ROOT, "tests", "sanitize", "message_reads_cases.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    sys.stdout.write(out.stdout)
    assert out.returncode == 0, out.stdout[-2000:]
    assert "message reads ok" in out.stdout

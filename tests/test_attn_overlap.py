"""Which strides of an output are refused because its vectors would share elements (csrc/attn_plan.h, on the CPU)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_vectors_that_share_elements(tmp_path):
    exe = str(tmp_path / "attn_overlap")
    r = subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2503_05931_amd", "csrc"), os.path.join(ROOT, "tests", "native", "attn_overlap.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]

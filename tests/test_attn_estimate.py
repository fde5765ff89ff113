"""Host side of ragged attention's key splits: the estimate decides (csrc/attn_plan.h)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_splits_follow_their_estimate(tmp_path):
    exe = str(tmp_path / "attn_estimate")
    r = subprocess.run(["/opt/rocm/llvm/bin/clang++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2503_05931_amd", "csrc"), os.path.join(ROOT, "tests", "native", "attn_estimate.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    print(r.stdout)

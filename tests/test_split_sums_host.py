"""CPU-only check of how attention of few rows splits its keys where results are fp32."""
import os
import subprocess

from paper_2307_02628_b200 import build


def test_sums_are_short_where_there_is_room(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "split_sums_host.cu")
    exe = str(tmp_path / "split_sums_host")
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, src], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok")

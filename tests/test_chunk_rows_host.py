"""CPU-only check of the rows that attention over chunks looks up masks and slopes for."""
import os
import subprocess

from paper_2307_02628_b200 import build


def test_no_row_or_token_behind_the_last_one(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "chunk_rows_host.cu")
    exe = str(tmp_path / "chunk_rows_host")
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, "-o", exe, src], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert out.stdout.startswith("ok")

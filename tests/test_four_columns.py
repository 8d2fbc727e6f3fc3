"""CPU check of which lane of small_loss_kernel keeps which columns (csrc/tile_index.h): tests/four_columns_check.hip, compiled with hipcc and run on the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_column_has_one_writer(tmp_path):
    exe = str(tmp_path / "four_columns_check")
    build = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O1", "-std=c++17", "-Wno-unused-command-line-argument",
                            "-x", "hip", os.path.join(ROOT, "tests", "four_columns_check.hip"), "-o", exe], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and "four columns ok" in run.stdout, run.stdout[-3000:] + run.stderr[-1000:]

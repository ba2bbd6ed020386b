"""How the paged cache's kernels find a slot's row, and that a bad table entry finds none: their own code, on the host (no GPU needed)."""
import subprocess
from pathlib import Path

from paper_2410_03804_amd import build

HERE = Path(__file__).resolve().parent


def test_rows_and_division_on_the_host(tmp_path):
    exe = tmp_path / "kv_rows"
    subprocess.run([build._hipcc(), "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-I", str(build.CSRC), "-x", "hip",
                    str(HERE / "kv_rows_driver.cpp"), "-o", str(exe)], check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout

"""The rows and elements that a tile's loads read (csrc/dfx_tiles.h, compiled for the device and the host alike), walked on the CPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tiles_read_inside_the_matrix(tmp_path):
    exe = str(tmp_path / "tiles_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(ROOT, "tests", "rules", "tiles_check.cpp"), "-o", exe], check=True, timeout=120)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout

"""The feed-forward kernels' launch sizes, checked in C++."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_ffn_launches(tmp_path):
    exe = str(tmp_path / "ffn_launch_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                    "-I", os.path.join(ROOT, "paper_2606_13894_amd", "csrc"),
                    os.path.join(ROOT, "tests", "ffn_launch_check.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout

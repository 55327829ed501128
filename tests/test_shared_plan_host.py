"""Runs tests/shared_plan_host.cu on the CPU: how the shared-prefix attention divides its work."""
import os
import subprocess

from paper_2412_00061_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_division_of_the_work(tmp_path):
    exe = str(tmp_path / "shared_plan_host")
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, os.path.join(HERE, "shared_plan_host.cu"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout

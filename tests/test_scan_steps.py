"""Where the steps of a scan lie, without a GPU: nothing outside a lane's own rows is read or stored at any accepted stride."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_offsets_stay_in_a_lanes_rows(tmp_path):
    compiler = shutil.which("g++")
    if compiler is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "scan_steps_host")
    subprocess.run([compiler, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I",
                    os.path.join(ROOT, "paper_1712_01887_amd", "csrc"), os.path.join(ROOT, "tests", "scan_steps_host.cc"),
                    "-o", exe], check=True, capture_output=True, text=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.startswith("ok "), run.stdout + run.stderr

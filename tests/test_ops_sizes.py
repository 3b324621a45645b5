"""Sizes and layouts of the training operators: what the host decides about them, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["ops_sizes_check", "ops_columns_check"])
def test_host_decisions(tmp_path, name):
    exe = tmp_path / name
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I",
                           os.path.join(ROOT, "paper_2609_34162_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", name + ".cpp"), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout

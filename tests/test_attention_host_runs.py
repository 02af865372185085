"""The blocks that a split row is joined through, on the host."""
import os
import shutil
import subprocess

import pytest


def test_split_rows_stay_within_the_workspace(tmp_path):
    """Random rows, among them such as no split gave (lengths that were changed while a call ran), under the host sanitizers."""
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "attn_runs_driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", os.path.join(root, "paper_2411_11217_amd", "csrc"),
                        os.path.join(root, "tests", "attn_runs_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])

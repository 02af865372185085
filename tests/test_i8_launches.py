"""The kernels of the layer in 8-bit integers that the library holds, against those that its rules reach (by the host's formulas, tests/util.py)."""
import itertools
import re
import shutil
import subprocess

import pytest

from paper_2411_11217_amd import build
from util import i8_expert_launches, i8_linear_launch


def kernels():
    """(operands' kind, name, template arguments) of the library's kernels on 8-bit integers, by its symbols."""
    nm = shutil.which("nm") or shutil.which("llvm-nm", path="/opt/rocm/llvm/bin")
    if nm is None:
        pytest.skip("no nm")
    if build.is_stale():
        build.build()
    out = subprocess.run([nm, build.LIB], capture_output=True, text=True, check=True).stdout
    found = set()
    for line in out.splitlines():
        symbol = line.split()[-1]
        m = re.search(r"GLOBAL__N_1\d+(ffn_rows|ffn_thin|ffn_gemm)INS_4Int8I(f|DF16b)EE((?:L[ib]\d+E)+)E", symbol)
        if m and line.split()[-2] in "dD":
            found.add((m[2], m[1]) + tuple(int(v) for v in re.findall(r"L[ib](\d+)E", m[3])))
    return found


def test_every_linear_and_expert_kernel_is_reached_and_there():
    lines = sorted({*range(1, 40), *range(40, 400, 8), *range(400, 5000, 64), 63, 65, 95, 97, 127, 129, 161, 20000})
    reached = set()
    for K, N in itertools.product([256, 512, 1024, 1536, 2048, 2560, 2816, 4096, 6144, 14336], [128 * n for n in (*range(1, 24), *range(25, 50), *range(50, 170, 6), 128, 161, 256, 512)]):
        reached |= {("f",) + i8_linear_launch(T, K, N) for T in lines}
    for (H, F), E in itertools.product([(256, 512), (256, 4096), (512, 768), (1024, 2816), (2048, 1024), (2048, 4096), (4096, 14336), (6144, 10752), (1280, 768)], (1, 2, 5, 8, 16, 64)):
        for T in lines:
            gate, down, _ = i8_expert_launches(T, H, F, E, 1)
            reached |= {("f",) + gate, ("DF16b",) + down}
    held = kernels()
    assert reached - held == set()
    assert held - reached == set()

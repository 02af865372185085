"""The kernels of the layer in 8-bit integers that the library holds, against those that its rules reach (by the host's formulas, tests/util.py)."""
import itertools
import re
import shutil
import subprocess

import pytest

from paper_2411_11217_amd import build
from util import i8_expert_launches, i8_linear_launch


def symbols():
    """The library's kernels, by the symbols of their handles on the host."""
    nm = shutil.which("nm") or shutil.which("llvm-nm", path="/opt/rocm/llvm/bin")
    if nm is None:
        pytest.skip("no nm")
    if build.is_stale():
        build.build()
    out = subprocess.run([nm, build.LIB], capture_output=True, text=True, check=True).stdout
    return [line.split()[-1] for line in out.splitlines() if line.split()[-2] in "dD"]


def arguments(text):
    return tuple(int(v) for v in re.findall(r"L[ib](\d+)E", text))


def kernels():
    """(operands' kind, name, template arguments) of those that multiply 8-bit integers."""
    found = (re.search(r"GLOBAL__N_1\d+(ffn_rows|ffn_thin|ffn_gemm)INS_4Int8I(f|DF16b)EE((?:L[ib]\d+E)+)E", s) for s in symbols())
    return {(m[2], m[1]) + arguments(m[3]) for m in found if m}


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


def test_every_kernel_of_rows_in_8_bits_is_another():
    """Element type, elements of a load, wavefronts to a row, loads of a thread, hint on loads, hint on stores: rows that are read twice have no hint, and the one on
    stores is for h, which is read eight bf16 at a time."""
    found = (re.search(r"quantize_kernelI([ft])((?:L[ib]\d+E)+)E", s) for s in symbols())
    held = {(m[1],) + arguments(m[2]) for m in found if m}
    lengths = [(1, 1), (1, 2), (4, 2), (8, 2), (16, 2), (16, 4)]
    want = {(t, vec, waves, per, far, 0) for t, vec in (("f", 4), ("t", 4), ("t", 8)) for waves, per in lengths for far in (0, 1)}
    want |= {("t", 8, waves, per, 1, 1) for waves, per in lengths} | {("f", 4, 16, 0, 0, 0), ("t", 4, 16, 0, 0, 0), ("t", 8, 16, 0, 0, 0)}
    assert held == want

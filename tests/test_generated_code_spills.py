"""No kernel keeps values in scratch memory: rows, sums and shares that the comments call kept in registers are.  CPU only: it reads the library as built."""
import os
import subprocess

from paper_2604_00785_amd import binding as B
from test_generated_code import OBJDUMP, _code_objects, _parse


def spilling(path):
    """(kernels, {those that touch scratch memory: how often})"""
    n, found = 0, {}
    for i, obj in enumerate(_code_objects(path)):
        file = "/tmp/moe_spills_%d_%d.o" % (os.getpid(), i)
        with open(file, "wb") as f:
            f.write(obj)
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", file], capture_output=True, text=True, check=True).stdout
        os.remove(file)
        for name, code in _parse(out).items():
            n += 1
            touches = sum(text.startswith("scratch_") for _, text in code)
            if touches:
                found[name] = touches
    return n, found


def test_no_kernel_spills():
    B.load()
    n, found = spilling(B.LIB_PATH)
    assert n > 100 and not found, found

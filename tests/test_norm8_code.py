"""The compiled kernels of the norm, dropout and the products in 8 bits: the device code in the built library."""
import os
import re
import subprocess

import pytest

from paper_2504_03871_amd import build
from tests.test_gemm_code import OBJDUMP, device_code


def test_no_kernel_spills_registers(tmp_path):
    """A value that comes back from scratch memory waits for every load in flight.  Left out: rows of more than 8192 (norm's backward) or
    16384 values (quantising) that no eight divides, which hold the most registers and meet no layer's width."""
    if not os.path.exists(build.LIB):
        pytest.skip("library not built")
    found, spilled, name = set(), set(), ""
    for code in device_code(build.LIB):
        (tmp_path / "code").write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(tmp_path / "code")], capture_output=True, text=True, check=True).stdout
        for line in listing.splitlines():
            if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
                name = m[1]
            elif re.search(r"gemm8_kernel|few8|join8|norm_(fwd|bwd|dgamma)|dropout_kernel|quant_(rows|weight)", name):
                found.add(name)
                if line.strip().startswith("scratch_"):
                    spilled.add(name)
    assert len(found) > 150
    wide = {n for n in spilled if re.search(r"norm_bwd_kernel\w+Lb1ELi8ELi4E|quant_rows_kernel\w+Lb1ELi16E", n)}
    assert spilled == wide, spilled - wide

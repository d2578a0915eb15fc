"""The compiled kernels of the operators beside the expert layer: the device code in the built library."""
import os
import re
import subprocess

import pytest

from paper_2504_03871_amd import build
from tests.test_gemm_code import OBJDUMP, device_code


def test_no_product_kernel_spills_registers(tmp_path):
    """A value that comes back from scratch memory waits for every load in flight; in a main loop that is the next stages'."""
    if not os.path.exists(build.LIB):
        pytest.skip("library not built")
    found, spilled, name = set(), set(), ""
    for code in device_code(build.LIB):
        (tmp_path / "code").write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(tmp_path / "code")], capture_output=True, text=True, check=True).stdout
        for line in listing.splitlines():
            if m := re.match(r"[0-9a-f]+ <(\S+)>:", line):
                name = m[1]
            elif re.search(r"linear_(rows|f32|pair|join)|score_(kernel|bwd|dx|logits)|act_bwd|sum_(many_)?rows|pack8|restore8", name):
                found.add(name)
                if line.strip().startswith("scratch_"):
                    spilled.add(name)
    assert len(found) > 60
    assert not spilled, spilled

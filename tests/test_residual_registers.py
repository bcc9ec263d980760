"""What the compiler made of the kernels between the layers of a residual block: rows, operands and sums that wait in registers stay
there."""
import os
import re
import subprocess

import pytest

import paper_1805_04170_amd.binding as binding
from test_kernel_registers import READELF, code_objects


@pytest.mark.skipif(READELF is None or not os.path.exists(binding.LIB_PATH), reason="no llvm-readelf, or the library is not built")
def test_residual_operators_keep_their_values_in_registers(tmp_path):
    seen = {}
    for i, obj in enumerate(code_objects()):
        path = os.path.join(str(tmp_path), "%d.o" % i)
        with open(path, "wb") as f:
            f.write(obj)
        notes = subprocess.run([READELF, "--notes", path], capture_output=True, text=True, check=True).stdout
        for name, spilled in re.findall(r"\.symbol:\s+(\S+)\.kd.*?\.vgpr_spill_count:\s+(\d+)", notes, re.S):
            kernel = re.search(r"(dropout|norm_(?:forward|backward|gain|stats)(?:_long)?|(?:un)?rows8(?:_long)?|weights8(?:_most)?|fc8_(?:tile|few|join|gather))_kernel", name)
            if kernel:
                seen.setdefault(kernel.group(1), []).append((name, int(spilled)))
    assert len(seen) == 1 + 6 + 3 + 2 + 4
    assert not [k for ks in seen.values() for k in ks if k[1]]

"""The products of the linear layer read LDS behind the compiler's back too: no register is used before its
read has landed (tests/test_lds_waits.py says how that is checked)."""
import os
import subprocess

import pytest

from paper_2512_06989_amd import build
from tests.test_lds_waits import early_uses, kernels


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
def test_no_register_is_used_before_its_lds_read_has_landed(tmp_path):
    asm = str(tmp_path / "kernels.asm")
    subprocess.run([build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", "-o", asm,
                    os.path.join(build.CSRC, "linear_bf16.hip")], check=True, capture_output=True)
    found, reads = {}, 0
    for name, (ins, labels) in kernels(open(asm).read()).items():
        reads += sum(i.fills for i in ins)
        bad = early_uses(ins, labels)
        if bad:
            found[name] = bad[:4]
    assert reads > 100
    assert not found, found

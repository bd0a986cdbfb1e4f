"""The waits between matrix instructions and what reads their results
(test_matrix_waits_asm, test_matrix_operands_asm), followed in the paged
attention's compiled code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B
from test_matrix_operands_asm import early_products
from test_matrix_waits_asm import early_readers


def test_readers_and_operands_wait_for_the_products(tmp_path):
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "code.s")
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out,
                                              os.path.join(B.CSRC, "gs_paged_attn.hip")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    total = 0
    for name, body in re.findall(r"^(_Z\S*kernel\S*):[^\n]*\n(.*?)^\s*\.section", open(out).read(), re.S | re.M):
        for look in (early_readers, early_products):
            products, found = look(body)
            assert not found, (name, found[0])
        total += products
    assert total > 0

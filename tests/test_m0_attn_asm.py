"""The direct-to-LDS loads of the cross-attention gradient set M0 in inline
assembly, which the compiler cannot take into account.  That is safe only while
nothing else in the code object writes or reads M0: this test compiles the
translation unit for gfx950 to AMD assembly, with the library's flags, and
checks that every instruction that names m0 is such a block's own `s_mov_b32 m0,
sN`, followed by `s_nop 0` and its one `buffer_load_dwordx4 ... lds`, and that
nothing that reads M0 implicitly appears anywhere."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B

SRC = os.path.join(B.CSRC, "gs_xattn_grad.hip")
IMPLICIT_M0 = re.compile(r"^(s_movrel|v_movrel|s_sendmsg|ds_gws|ds_append|ds_consume|v_interp|s_set_gpr_idx"
                         r"|ds_read_addtid|ds_write_addtid|global_load_lds)")


def test_m0_belongs_to_the_loads(tmp_path):
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "grad.s")
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out, SRC], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    ins = []
    for line in open(out):
        m = re.match(r"^\s+([a-z_][a-z0-9_]*)(\s[^;]*)?", line.split(";")[0].rstrip())
        if m and not line.lstrip().startswith("."):
            ins.append((m.group(1), (m.group(2) or "").strip()))
    blocks = 0
    for i, (op, args) in enumerate(ins):
        assert not IMPLICIT_M0.match(op), (op, args)
        if re.search(r"\bm0\b", args):
            assert op == "s_mov_b32" and re.fullmatch(r"m0,\s*s\d+", args), (op, args)
            assert ins[i + 1] == ("s_nop", "0"), ins[i + 1]
            assert ins[i + 2][0] == "buffer_load_dwordx4" and re.search(r"\blds\b", ins[i + 2][1]), ins[i + 2]
            blocks += 1
    loads = sum(op.startswith("buffer_load") and bool(re.search(r"\blds\b", args)) for op, args in ins)
    assert blocks == loads > 0

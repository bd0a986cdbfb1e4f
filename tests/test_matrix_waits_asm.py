"""A matrix instruction writes its result some cycles after it was issued, and
the compiler has to keep other readers of it that far away.  Where a branch lay
between the last product of a loop and the loop's end it has been seen to count
the longer way round for both.  This test compiles the cross-attention sources
for gfx950 to AMD assembly, with the library's flags, and follows every path
from every matrix instruction to the first vector or memory instruction that
reads its result, counting an instruction as one wait state and `s_nop n` as
n + 1."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B

# Wait states before another unit may read the result: 16 passes (fp32) and 8
# passes (bf16).
NEED = {"v_mfma_f32_32x32x2_f32": 18, "v_mfma_f32_32x32x16_bf16": 11}
STORES = ("ds_write", "ds_bpermute", "global_store", "buffer_store", "scratch_store", "flat_store", "global_atomic")


def registers(text):
    return [(m[1] or m[4], int(m[2] or m[5]), int(m[3] or m[5]))
            for m in re.finditer(r"(?<![a-z0-9_])([va])\[(\d+):(\d+)\]|(?<![a-z0-9_\[])([va])(\d+)\b", text)]


def parse(body):
    """Instructions (name, written, read, arguments) and the positions of labels."""
    ins, labels = [], {}
    for line in body.split("\n"):
        m = re.match(r"^(\.LBB\S+):", line)
        if m:
            labels[m[1]] = len(ins)
            continue
        m = re.match(r"^\s+([a-z]\S*)\s*([^;]*)", line)
        if not m:
            continue
        op, args = m[1], m[2].strip()
        parts = re.split(r",(?![^\[]*\])", args)
        wrote = [] if op.startswith(STORES[:1] + STORES[2:]) else registers(parts[0])
        read = registers(args) if not wrote else [r for p in parts[1:] for r in registers(p)]
        ins.append((op, wrote, read, args))
    return ins, labels


def early_readers(body):
    ins, labels = parse(body)
    overlap = lambda a, b: a[0] == b[0] and a[1] <= b[2] and b[1] <= a[2]  # noqa: E731

    def after(i):
        op, args = ins[i][0], ins[i][3]
        if op == "s_endpgm":
            return []
        jump = [labels[args.split()[0]]] if op.startswith(("s_branch", "s_cbranch")) else []
        return jump + ([] if op == "s_branch" or i + 1 == len(ins) else [i + 1])

    products, found = 0, []
    for i, (op, wrote, _, _) in enumerate(ins):
        if not op.startswith("v_mfma"):
            continue
        products += 1
        result, need = wrote[0], NEED[op]
        least, todo = {}, [(j, 0) for j in after(i)]
        while todo:
            j, waited = todo.pop()
            if waited >= need or least.get(j, need) <= waited:
                continue
            least[j] = waited
            name, w, r, args = ins[j]
            if name.startswith("v_mfma"):
                if result in w:         # the next product of the chain: followed from there
                    continue
            elif any(overlap(result, x) for x in r):
                found.append((ins[i][0], ins[i][3], name, args, waited))
                continue
            step = int(args, 0) + 1 if name == "s_nop" else 1
            todo += [(k, waited + step) for k in after(j)]
    return products, found


def test_the_check_sees_an_early_reader():
    body = "\tv_mfma_f32_32x32x2_f32 v[0:15], v20, v21, v[0:15]\n\ts_cbranch_scc1 .LBB0_2\n\ts_nop 15\n\ts_nop 3\n.LBB0_2:\n%s\tv_mov_b32_e32 v30, v15\n\ts_endpgm"
    assert early_readers(body % "")[1] and early_readers(body % "\ts_nop 15\n")[1]      # 1 and 17 states
    assert early_readers(body % "\ts_nop 15\n\ts_nop 0\n") == (1, [])


@pytest.mark.parametrize("source", ["gs_xattn.hip", "gs_xattn_grad.hip"])
def test_readers_wait_for_the_products(source, tmp_path):
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "code.s")
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(B.CSRC, source)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    text = open(out).read()
    kernels = re.findall(r"^(_Z\S*kernel\S*):[^\n]*\n(.*?)^\s*\.section", text, re.S | re.M)
    total = 0
    for name, body in kernels:
        products, found = early_readers(body)
        assert not found, (name, found[0])
        total += products
    assert total > 0

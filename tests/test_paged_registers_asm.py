"""The paged operators' compiled kernels keep what they work with in registers: a value
kept in memory would be read back between the loads that are on their way, and wait
for them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_01528_amd import build as B


def kernels(source, tmp_path):
    """{name: (bytes of memory a lane, registers that found no place, bytes of LDS)}"""
    if not (os.path.exists(B.HIPCC) or shutil.which(B.HIPCC)):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "code.s")
    r = subprocess.run([B.HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", "-o", out, os.path.join(B.CSRC, source)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = {}
    for entry in re.findall(r"- \.agpr_count:.*?\.wavefront_size", open(out).read(), re.S):
        value = lambda k: re.search(r"\.%s:\s*(\S+)" % k, entry).group(1)  # noqa: E731
        found[value("name")] = tuple(int(value(k)) for k in ("private_segment_fixed_size", "vgpr_spill_count",
                                                             "group_segment_fixed_size"))
    assert found
    return found


def test_attention(tmp_path):
    found = kernels("gs_paged_attn.hip", tmp_path)
    assert sum("10few_kernel" in n for n in found) == 24 and sum("11many_kernel" in n for n in found) == 12
    for name, (memory, spilled, _) in found.items():
        assert memory == 0 and spilled == 0, name


def test_pages_and_rows(tmp_path):
    """The plan's sums are all that it keeps in LDS: 4 for each of 1024 requests in one
    work-group, of 2048 in the launch that follows them."""
    found = kernels("gs_paged.hip", tmp_path)
    for name, (memory, spilled, lds) in found.items():
        assert memory == 0 and spilled == 0, name
        assert lds <= 4 * (4 * (2048 if "plan_fill" in name else 1024) + 4) + 1024, (name, lds)

"""Waves per SIMD and LDS of the paged cache's kernels (CPU only: hipcc
cross-compiles), which the launches count on: a kernel that takes more
registers runs fewer workgroups per CU and no parity test would notice."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_01065_amd import build as BUILD

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")

# kernel, template arguments -> waves per SIMD at least, bytes of LDS at most (static)
WANTED = {
    "paged_attn_kernelI.*Li64E": (3, 160 * 1024 // 3),      # three workgroups of four waves per CU
    "paged_attn_kernelI.*Li128E": (2, 160 * 1024 // 2),     # two
    "paged_attn_kernelI.*Li256E": (1, 160 * 1024),          # one
    "paged_decode_lds_kernelI.*Li1ELi8E": (4, 32 * 1024),   # one of 16 waves, beside 128 KiB of codewords
    "paged_decode_lds_kernelI.*Li2ELi4E": (2, 32 * 1024),
    "paged_row_decode_stages_kernel": (4, 160 * 1024),      # one of 16 waves
    "paged_append_kernel": (8, 1024),
}


def _resources(src, tmp):
    res = subprocess.run([BUILD.hipcc(), *BUILD.flags_for(src), "-c", "-I", BUILD.INCLUDE, "-o", os.path.join(tmp, "x.o"), src,
                          "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    out, name = {}, None
    for line in res.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            name = m.group(1)
            out[name] = {}
        m = re.search(r"(Occupancy \[waves/SIMD\]|LDS Size \[bytes/block\]|VGPRs Spill): (\d+)", line)
        if m and name:
            out[name][m.group(1).split(" [")[0]] = int(m.group(2))
    return out


def test_waves_and_lds(tmp_path):
    found = {}
    for src in BUILD.SRCS:
        if "paged" in os.path.basename(src):
            found.update(_resources(src, str(tmp_path)))
    for pattern, (waves, lds) in WANTED.items():
        kernels = {k: v for k, v in found.items() if re.search(pattern, k)}
        assert kernels, pattern
        for k, v in kernels.items():
            assert v["Occupancy"] >= waves and v["LDS Size"] <= lds and v["VGPRs Spill"] == 0, (k, v)

"""Registers, waves per SIMD and LDS of the 8-bit cache's and the serving
kernels (CPU only: hipcc cross-compiles), which the launches count on."""
import os
import re
import shutil

import pytest

from paper_2607_01065_amd import build as BUILD
from tests.test_build_resources import _remarks, _scratch_loop_depths
from tests.test_paged_occupancy import _resources

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")

# file -> kernel, template arguments -> waves per SIMD at least, bytes of LDS at most
WANTED = {
    "gsrq_cache8.hip": {
        "cache8_attn_kernelI.*Li64E": (2, 160 * 1024 // 2),        # two workgroups of four waves per CU
        "cache8_attn_kernelI.*Li128E": (2, 160 * 1024 // 2),
        "cache8_attn_kernelI.*Li256E": (1, 160 * 1024),
        "cache8_append_kernelIDF16b?": (4, 160 * 1024 // 4),
        "cache8_append_kernelIf": (3, 160 * 1024 // 3),
    },
    "gsrq_serving.hip": {
        "plan_update_kernel": (4, 160 * 1024),                     # one workgroup of at most 16 waves
        "verify_sums_kernel": (8, 1024),
        "verify_row_kernel": (4, 1024),
        "verify_finalize_kernel": (4, 1024),
    },
}


@pytest.mark.parametrize("name", WANTED)
def test_waves_lds_and_scratch(name, tmp_path):
    src = [f for f in BUILD.SRCS if os.path.basename(f) == name][0]
    found = _resources(src, str(tmp_path))
    for pattern, (waves, lds) in WANTED[name].items():
        kernels = {k: v for k, v in found.items() if re.search(pattern, k)}
        assert kernels, pattern
        for k, v in kernels.items():
            assert v["Occupancy"] >= waves and v["LDS Size"] <= lds and v["VGPRs Spill"] <= 4, (k, v)
    kernels = re.compile("cache8_|plan_|verify_")
    depths = {k: max(v) for k, v in _scratch_loop_depths(src).items() if kernels.search(k) and v and max(v) >= 1}
    assert not depths, depths
    assert max(v for k, v in _remarks(src).items() if kernels.search(k)) <= 16

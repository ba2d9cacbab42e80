"""Registers of the paged cache's kernels (CPU only: hipcc cross-compiles): none
touches scratch memory inside a loop, and none keeps more than a few bytes
there."""
import os
import re
import shutil

import pytest

from paper_2607_01065_amd import build as BUILD
from tests.test_build_resources import _remarks, _scratch_loop_depths

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="hipcc not available")
PAGED = [f for f in BUILD.SRCS if "paged" in os.path.basename(f)]
KERNELS = re.compile(r"paged_(append|decode_lds|row_decode|row_decode_stages|attn|attn_merge)_kernel")


@pytest.mark.parametrize("tu", PAGED)
def test_no_scratch_in_loops(tu):
    depths = {k: v for k, v in _scratch_loop_depths(tu).items() if KERNELS.search(k)}
    assert len(depths) >= 12, sorted(depths)
    assert not {k: max(v) for k, v in depths.items() if v and max(v) >= 1}
    small = {k: v for k, v in _remarks(tu).items() if KERNELS.search(k)}
    assert small and max(small.values()) <= 16, small

"""The cache operators' launch plans under the host sanitizers, and their kernels' registers: no kernel of csrc/bpd_cache.hip may use scratch memory (a spill in one
kernel slows every other one of a step)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1811_03115_amd import build
from test_host_logic import HERE, build_and_run


def test_launch_plans(tmp_path):
    assert build_and_run(os.path.join(HERE, "host", "cache_logic_check.cpp"), str(tmp_path)).strip() == "ok"


def test_no_cache_kernel_uses_scratch(tmp_path):
    hipcc = build.hipcc()
    if shutil.which(hipcc) is None and not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    source = next(s for s in build.SOURCES if s.endswith("bpd_cache.hip"))
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([hipcc] + flags + ["--cuda-device-only", "-c", source, "-o", str(tmp_path / "dev.o"), "-Rpass-analysis=kernel-resource-usage"],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-2000:]
    found, cur = {}, None
    for line in res.stdout.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            cur = m.group(1)
        m = re.search(r"ScratchSize \[bytes/lane\]: (\d+)", line)
        if m:
            found[cur] = int(m.group(1))
    for kernel in ("tree_attention_kernel", "tree_attention_rows_kernel", "tree_rows_kernel", "tree_join_kernel", "store_groups_kernel", "store_rows_kernel",
                   "block_bounds_kernel", "block_pick_kernel", "tree_accept_kernel", "tree_move_kernel"):
        assert any(kernel in name for name in found), f"{kernel} not found"
    assert not {n: s for n, s in found.items() if s > 0}

"""What the compiler makes of the append: its work-groups hold a block's values in registers, and an instance that spills them takes several times as long."""
import os
import re
import subprocess

import pytest

from paper_2508_09204_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")


def test_append_keeps_its_values_in_registers(tmp_path):
    cmd = [build.HIPCC] + build.FLAGS + ["-Rpass-analysis=kernel-resource-usage", "--offload-device-only", "-c", os.path.join(build.CSRC, "kv_append.hip"), "-o", str(tmp_path / "a.o")]
    report = subprocess.run(cmd, check=True, capture_output=True, text=True).stderr
    got = {}
    for name, rest in re.findall(r"Function Name: (\S+)(.*?)(?=Function Name|\Z)", report, re.S):
        m = re.search(r"k_kv_appendILi(\d+)ELb([01])ELi(\d+)E", name)
        if m:
            got[tuple(map(int, m.groups()))] = int(re.search(r"ScratchSize \[bytes/lane\]: (\d+)", rest).group(1))
    assert len(got) == 8
    # fp32 rows in work-groups of 1024 threads, of blocks of 128 tokens with 256 dims, keep 21 registers in scratch: 60 us where a copy of as many bytes takes 38
    assert all(n == 0 for (dh, bf16, threads), n in got.items() if bf16 or threads <= 512), got

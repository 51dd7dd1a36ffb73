"""What the library is built from: no kernel that nothing launches."""
import re
import shutil
import subprocess

import pytest

from paper_2609_14237_b200 import binding as B


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm")
def test_a_stage_kernel_is_compiled_in_one_namespace_only():
    """Translation units that take the attention kernels or their helpers under a namespace of their own leave the stage's small
    kernels, which they never launch, to the main one."""
    B.build()
    names = subprocess.run(["nm", "-C", B.LIB_PATH], check=True, capture_output=True, text=True).stdout
    for kernel in ("kv_append_kernel", "advance_kernel", "table_delta_kernel", "wait_probe_kernel", "read_probe_kernel"):
        spaces = set(re.findall(rf"\b(\w+)::{kernel}\(", names))
        assert spaces == {"opw"}, (kernel, spaces)

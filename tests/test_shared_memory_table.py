"""A context notes the kernels that it has opted into more shared memory, once each: its table holds all that the library has."""
import re
import shutil
import subprocess

import pytest

from paper_2503_17469_b200 import build

# the kernels whose launches ask for it, by name
KERNELS = ("attention_rows_kernel", "attention_forward_kernel", "attention_backward_kernel", "attention_forward_join_kernel",
           "attention_backward_join_kernel", "sort_tokens_kernel", "policy_kernel", "rotary_forward_wide_kernel", "rotary_backward_wide_kernel")


@pytest.mark.skipif(not shutil.which("nm"), reason="no nm")
def test_table_holds_every_kernel_that_opts_in():
    names = subprocess.run(["nm", "-C", str(build.LIB)], capture_output=True, text=True, check=True).stdout
    host = {m.group(2): m.group(1) for m in re.finditer(r"^\S+ [tTwW] (?:void )?omni::(?:\(anonymous namespace\)::)?((\w+)[<(].*)$", names, re.M)}
    found = {m.group(0) for m in re.finditer(r"^\S+ [tTwW] (?:void )?omni::(?:\(anonymous namespace\)::)?(?:%s)[<(].*$" % "|".join(KERNELS), names, re.M)}
    assert set(KERNELS) <= set(host)
    room = int(re.search(r"opted\[(\d+)\]", (build.CSRC / "omni.cu").read_text()).group(1))
    assert 60 < len(found) <= room, (len(found), room)

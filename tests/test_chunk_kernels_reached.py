"""The chunk kernels that the library holds are those that a call can reach: keys of packed rows are never cut, so that no launch plans them."""
import os
import re

import pytest

from paper_2507_04610_amd import binding
from test_kernel_metadata import device_code_objects


def test_packed_rows_have_no_planning_kernel():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("libany4.so has not been built")
    names = set()
    for image in device_code_objects(binding.LIB_PATH):
        names |= set(re.findall(rb"attn_chunk\w*kernelILi\d+E\w*", image))
    sources = {kind: {int(m.group(1)) for n in names if (m := re.match(kind + rb"ILi(\d+)E", n))} for kind in (b"attn_chunk_kernel", b"attn_chunk_plan_kernel")}
    assert sources == {b"attn_chunk_kernel": {0, 4, 8, 16}, b"attn_chunk_plan_kernel": {4, 8, 16}}

"""The device code (gfx950) of the adapters' and the router's kernels: their tiles stay in registers, nothing lies in scratch memory."""
import re

import pytest

from test_device_code import _code_object, _tool


@pytest.mark.parametrize("kernel,least", [(b"fused_few_kernel", 30), (b"router_prepare_kernel", 20)])
def test_no_kernel_uses_scratch_memory(tmp_path_factory, kernel, least):
    notes = _tool("llvm-readelf", "--notes", _code_object(tmp_path_factory, kernel))
    kernels = {re.search(r"\.name:\s+(\S+)", k).group(1): (int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", k).group(1)),
                                                           int(re.search(r"\.vgpr_spill_count:\s+(\d+)", k).group(1)))
               for k in re.split(r"- \.agpr_count:", notes)[1:]}
    assert len(kernels) >= least, sorted(kernels)
    assert not any(any(v) for v in kernels.values()), {n: v for n, v in kernels.items() if any(v)}

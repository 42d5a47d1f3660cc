"""Regression test (CPU): the plan of a cache that may be cut is one kernel without scratch memory, which never touches the
destination of an LDS read in flight and uses no packed fp32 instruction."""
import os
import re

import pytest

from isa_check import hazards
from test_isa_hazards import HIPCC, _asm


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_kernel(tmp_path):
    kernels = {k: v for k, v in _asm(tmp_path, "pages_kept.hip").items() if "kernel" in k}
    assert len(kernels) == 1
    text = (tmp_path / "pages_kept.hip.s").read_text()
    assert re.findall(r"\.private_segment_fixed_size: +(\d+)", text) == ["0"]
    for name, body in kernels.items():
        assert not any(l.strip().startswith(("scratch_", "v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for l in body), name
        assert not hazards(body), name

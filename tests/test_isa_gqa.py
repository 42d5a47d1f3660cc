"""Regression test (CPU): the grouped-head attention's kernels hold their state in
registers (no scratch memory), never touch the destination of an LDS read in
flight, and use no packed fp32 instruction."""
import os
import re

import pytest

from isa_check import hazards, kernel_bodies
from test_isa_hazards import HIPCC, _asm


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
@pytest.mark.parametrize("src,count", [("attn_gqa.hip", 28), ("attn_gqa_f32.hip", 6), ("pages.hip", 2)])
def test_kernels(tmp_path, src, count):
    kernels = {k: v for k, v in _asm(tmp_path, src).items() if "kernel" in k}
    assert len(kernels) == count
    text = (tmp_path / (src + ".s")).read_text()
    sizes = re.findall(r"\.private_segment_fixed_size: +(\d+)", text)
    assert len(sizes) == count and set(sizes) == {"0"}
    for name, body in kernels.items():
        assert not any(l.strip().startswith(("scratch_", "v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for l in body), name
        bad = hazards(body)
        assert not bad, "%s: %s" % (name, bad[:3])

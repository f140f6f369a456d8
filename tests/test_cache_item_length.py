"""The attention kernels over the 4-bit cache and the kernel that joins their parts find the items' length each for itself: to the same
bits, so no product in it may be fused with a sum, which the compiler does kernel by kernel (AMD assembly, compiled here; no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2506_19651_amd import build as B

PROBE = """
#include "attn_kv4.h"
using namespace pevlm;
extern "C" __global__ void place(Kv4Attn p, int32_t *to)
{
    const Place at = find_place<%s, %s, %s>(p, blockIdx.x);
    to[0] = at.s;
    to[1] = at.rest;
    to[2] = at.splits;
}
"""


@pytest.mark.parametrize("units", ["true", "false"])
@pytest.mark.parametrize("few", ["true", "false"])
@pytest.mark.parametrize("shared", ["true", "false"])
def test_no_product_is_fused_with_a_sum(tmp_path, units, few, shared):
    source, out = tmp_path / "place.hip", tmp_path / "place.s"
    source.write_text(PROBE % (units, few, shared))
    subprocess.run([B.HIPCC, *B.FLAGS, "--cuda-device-only", "-S", str(source), "-o", str(out)], check=True, capture_output=True)
    code = re.findall(r"^\s+([sv]_\w+)", out.read_text(), re.M)
    assert any(op.startswith("v_rcp_f32") for op in code) and any(op.startswith("v_mul_f32") for op in code)  # it is there
    fused = [op for op in code if re.match(r"[sv]_(fma|fmac|mad|mac|fmamk|fmaak)\w*_f32|[sv]_pk_fma", op)]
    assert not fused, fused

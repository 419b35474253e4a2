"""What the compiler made of the operators' registers, read from the metadata of the library that is built here: where a kernel of 256 registers
spills, how much at most, and that no other one does."""
import os
import re

import pytest

from test_register_budget import LIB, kernels

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="the library is not built")


def allowed(name):
    """Registers that a kernel may spill."""
    m = re.search(r"(k_attn_\w+?)INS_(?:3F16|4BF16)ELi(\d+)E((?:Li\d+E)*)", name)
    if not m or m.group(2) != "128":
        return 0
    kernel, rest, half = m.group(1), [int(x) for x in re.findall(r"Li(\d+)E", m.group(3))], "3F16" in name
    if kernel == "k_attn_forward":                      # waves with rows, waves with keys, mode
        return {(8, 1, 0): 4, (4, 1, 1): 14, (4, 1, 2): 14}.get(tuple(rest), 0)
    if kernel == "k_attn_dq":                           # waves, mode
        return 2 if half and rest == [4, 1] else 0
    if kernel == "k_attn_dkv":
        return {(4, True): 18, (4, False): 10, (8, True): 8, (8, False): 0}[rest[0], half]
    return 0


def test_spills():
    of_operators = {n: k for n, k in kernels(LIB).items() if re.search("k_attn_|k_product|k_tokens|k_sum_parts|k_grad_", n)}
    assert len(of_operators) >= 150
    for name, k in of_operators.items():
        assert k[".vgpr_spill_count"] <= allowed(name), (name, k[".vgpr_spill_count"])
        assert k[".group_segment_fixed_size"] <= 160 << 10, name

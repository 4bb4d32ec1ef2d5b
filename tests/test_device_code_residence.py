"""How many workgroups a compute unit holds of the kernels whose comments state it, from
their registers and LDS as compiled: 512 registers per SIMD in steps of eight, 160
KiB, eight workgroups of four wavefronts."""
from __future__ import annotations

import re

from test_device_code_serving import _kernels


def residents(lds, registers):
    return min(8, 512 // (-(-registers // 8) * 8), 160 * 1024 // lds)


def test_norms_with_rotary_positions():
    """By type, head dim, append, wide accesses and neighbouring pairs."""
    want = {}
    for t in "tf":
        for d in (64, 128):
            want.update({(t, d, append, False, inter): 8 for append in (False, True) for inter in (False, True)})
            want.update({(t, d, append, True, False): 7 if t == "f" and d == 64 else 5 for append in (False, True)})
            want[t, d, False, True, True] = 8
            want[t, d, True, True, True] = 5 if d == 128 else 7
    found = {}
    for name, (_, lds, registers) in _kernels("verify_norm_rotary.hip").items():
        t, d, *flags = re.search(r"norm_rotate_rowsI([tf])Li(\d+)ELb(\d)ELb(\d)ELb(\d)E", name).groups()
        found[(t, int(d), *(f == "1" for f in flags))] = residents(lds, registers)
    assert found == want


def test_changed_logits():
    """Seven workgroups in bf16, by LDS, and six in fp32, by registers."""
    found = {}
    for name, (_, lds, registers) in _kernels("verify_logits.hip").items():
        if "adjust_rows" in name:
            found.setdefault(re.search(r"adjust_rowsI([tf])", name)[1], set()).add(residents(lds, registers))
    assert found == {"t": {7}, "f": {6}}

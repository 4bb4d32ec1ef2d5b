"""What the compiled kernels of shared prefixes, norms with rotary positions and changed
logits must hold, read from their device assembly: the waits around loads to LDS, and
that everything a thread works on is in registers."""
from __future__ import annotations

import re

import pytest

from test_device_code import _assembly, _faults


def _kernels(name):
    """(scratch bytes, LDS bytes, vector registers) of each kernel in a file."""
    found = {}
    for block in re.split(r"\n  - \.agpr_count", _assembly(name))[1:]:
        value = lambda key: int(re.search(r"\.%s:\s+(\d+)" % key, block)[1])  # noqa: E731
        found[re.search(r"\.name:\s+(\S+)", block)[1]] = (
            value("private_segment_fixed_size"), value("group_segment_fixed_size"), value("vgpr_count"))
    return found


def test_loads_to_lds_wait_for_their_scalars():
    loads, bad = _faults(_assembly("verify_shared.hip"))
    assert loads >= 7
    assert not bad, "%d of %d loads, first: %s" % (len(bad), loads, bad[0])


@pytest.mark.parametrize("name,least", [("verify_shared.hip", 20), ("verify_norm_rotary.hip", 32), ("verify_logits.hip", 6)])
def test_no_kernel_uses_scratch_memory(name, least):
    kernels = _kernels(name)
    assert len(kernels) >= least
    assert not {n: k for n, k in kernels.items() if k[0]}


def test_two_workgroups_of_the_shared_walk_fit_a_compute_unit():
    """Its schedule and its flat walks count on all workgroups being resident at once."""
    walks = {n: k for n, k in _kernels("verify_shared.hip").items() if "shared_walk" in n}
    assert len(walks) == 8
    for scratch, lds, registers in walks.values():
        assert lds <= 80 * 1024 and registers <= 256

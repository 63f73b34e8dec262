"""What the built library says of the kernels of the recurrence, the distillation and the verification: none keeps registers in memory."""
import re

import pytest

from test_built_kernels import _kernels


@pytest.mark.parametrize("kernel", ["k_scan_fwd", "k_scan_bwd", "k_scan_chain", "k_scan_fwd_walk", "k_scan_bwd_walk", "k_distill_lists", "k_draft_verify"])
def test_no_instance_spills(kernel, tmp_path):
    found = {n: v for n, v in _kernels(tmp_path).items() if re.search(r"\d" + kernel + r"[IE]", n)}
    assert found, "no such kernel in the library"
    assert not {n: v for n, v in found.items() if v != (0, 0)}

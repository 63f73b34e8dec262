"""The launch that brings a word's tiles of dz to one scale keeps no registers in memory either."""
import re

from test_built_kernels import _kernels


def test_no_instance_spills(tmp_path):
    found = {n: v for n, v in _kernels(tmp_path).items() if re.search(r"\dk_vocab_levelI", n)}
    assert len(found) == 2 and not {n: v for n, v in found.items() if v != (0, 0)}, found

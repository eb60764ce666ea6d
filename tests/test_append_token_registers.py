"""Registers of the kernels that append single tokens, as the compiler reports them of the built library: as many as there were before positions
on several axes came to them.  Two more are the sign of copied code in the kernel's chain of reads, which cost a token's call 0.14 us of 5.2."""
import os
import re

import pytest

pytest.importorskip("msgpack")

from kernel_resources import kernels  # noqa: E402
from paper_2605_21226_amd import binding  # noqa: E402


def test_single_tokens():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("liboctopus.so is not built")
    found = {name: k[".vgpr_count"] for name, k in kernels(binding.LIB_PATH).items() if re.search(r"append_token_(axes_)?kernel", name)}
    assert len(found) == 36 and {name: n for name, n in found.items() if n > 59} == {}

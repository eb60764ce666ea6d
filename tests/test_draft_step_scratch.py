"""Scratch memory per lane, as the compiler reports it of the built library, of the kernels that work between a server's steps: none, but for a few words
of a prompt's kernel with two bit widths to a key.  And LDS that no source asks for: a choice between elements of an array or a struct that the
compiler cannot keep in registers goes there, and cost a call 12 us."""
import os
import re

import pytest

pytest.importorskip("msgpack")

from kernel_resources import kernels  # noqa: E402
from paper_2605_21226_amd import binding  # noqa: E402
from test_serve_scratch import PLANS, _scratch  # noqa: E402


@pytest.fixture(scope="module")
def library():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("liboctopus.so is not built")
    return kernels(binding.LIB_PATH)


def test_pages_and_verification(library):
    found = {name: k for name, k in library.items() if re.search(r"(pages_(share|assign|rows|compact|count|pair|apply|rename|copy)|verify_(row|sums|pick))_kernel", name)}
    assert len(found) == 3 + 8 + 6
    assert {n: k[".private_segment_fixed_size"] for n, k in found.items() if k[".private_segment_fixed_size"]} == {}
    assert {n for n, k in found.items() if re.search(r"(rows|apply|rename|copy|sums|pick)_kernel", n) and k[".group_segment_fixed_size"]} == set()


def test_appending_by_several_axes(library):
    assert _scratch(library, "append_token_axes_kernel") == {(d, b): 0 for d in (64, 128, 256) for b in PLANS}
    found = _scratch(library, "append_tile_axes_kernel")
    assert len(found) == 18 and {k: v for k, v in found.items() if v > {(128, "2.5"): 16}.get(k, 0)} == {}
    for name, k in library.items():          # as much LDS as the kernels of one position
        if re.search(r"append_(token|tile)_axes_kernel", name):
            one = re.sub(r"\d+append_(token|tile)_axes_kernel(INS_5PlanTI\w+?EEEE?).*", lambda m: f"append_{m[1]}_kernel{m[2]}", name)
            like = [v for n, v in library.items() if one.split("octopus")[-1] in n]
            assert len(like) == 1 and like[0][".group_segment_fixed_size"] == k[".group_segment_fixed_size"], name

"""Scratch memory per lane, as the compiler reports it of the built library, of the kernels over pages that a server calls around the
attention: no more than when they were measured."""
import os
import re

import pytest

pytest.importorskip("msgpack")

from kernel_resources import kernels  # noqa: E402
from paper_2605_21226_amd import binding  # noqa: E402

PLANS = {"1": (1, 1, 0, 0), "1.5": (3, 1, 1, 1), "2": (3, 1, 0, 0), "2.5": (4, 2, 3, 1), "3": (4, 2, 0, 0), "4": (5, 3, 0, 0)}


@pytest.fixture(scope="module")
def library():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("liboctopus.so is not built")
    return kernels(binding.LIB_PATH)


def _scratch(library, kernel, tail=""):
    """{(head dimension, bits, what `tail` matched): bytes per lane}"""
    names = {plan: bits for bits, plan in PLANS.items()}
    pat = re.compile(rf"{len(kernel)}{kernel}INS_5PlanTILi(\d+)ELi(\d)ELi(\d)ELi(\d)ELi(\d)EEE{tail}")
    found = {}
    for name, k in library.items():
        m = pat.search(name)
        if m:
            found[(int(m[1]), names[tuple(int(x) for x in m.groups()[1:5])], *m.groups()[5:])] = k[".private_segment_fixed_size"]
    return found


def test_shared_prefix_kernels(library):
    """At head dimension 128 two wavefronts a SIMD leave 256 registers, and queries' operands and accumulators alone take 144: some
    words of a lane live in scratch memory.  Nearly all of them are put there and fetched outside the loop over steps; inside it, of 108
    matrix and 500 to 760 vector instructions, 1 and 3 bits store and fetch none, the others store one and fetch one or two (causal
    ones: up to four).  At 64 and 256 there are none."""
    found = _scratch(library, "prefix_attention_kernel", r"Lb(\d)E")
    assert len(found) == 3 * 6 * 2
    assert {k: v for k, v in found.items() if k[0] != 128 and v} == {}
    most = {"1": 40, "1.5": 112, "2": 96, "2.5": 128, "3": 80, "4": 144}
    assert {k: v for k, v in found.items() if k[0] == 128 and v > most[k[1]]} == {}


def test_appending_kernels(library):
    """Two of the prompts' kernels with two bit widths to a key: a few words of a lane, outside the triplets' loop."""
    assert _scratch(library, "append_token_kernel") == {(d, b): 0 for d in (64, 128, 256) for b in PLANS}
    found = _scratch(library, "append_tile_kernel")
    assert len(found) == 18
    assert {k: v for k, v in found.items() if v > {(128, "2.5"): 32, (64, "1.5"): 16}.get(k, 0)} == {}


def test_reading_and_merging_kernels(library):
    assert _scratch(library, "read_tokens_kernel") == {(d, b): 0 for d in (64, 128, 256) for b in PLANS}
    merge = [k[".private_segment_fixed_size"] for name, k in library.items() if "19prefix_merge_kernel" in name]
    assert merge == [0, 0, 0]

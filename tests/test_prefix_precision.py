"""On the CPU: the shared-prefix attention's operands keep the tolerance that its GPU test goes by, and leaving any one correction out
is at least twice beyond it, so that the GPU test would notice."""
import pytest

from prefix_model import CASES, TOLERANCE, Inputs, model, off


@pytest.mark.parametrize("d,bits", CASES)
def test_every_correction_counts(d, bits):
    x = Inputs(d, bits)
    want = x.exact()
    assert off(model(x), want) <= TOLERANCE / 2
    for part in ("key", "query", "middle", "last"):
        assert off(model(x, without=part), want) > 2 * TOLERANCE, part

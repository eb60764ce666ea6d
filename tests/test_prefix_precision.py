"""On the CPU: the shared-prefix attention's operands keep the tolerance that its GPU test goes by, and leaving any one correction out
is several times beyond it, so that the GPU test would notice."""
import pytest

from prefix_model import CASES, TOLERANCE, Inputs, model, off


@pytest.mark.parametrize("d,bits", CASES)
def test_every_correction_counts(d, bits):
    x = Inputs(d, bits)
    want = x.exact()
    assert off(model(x), want) <= TOLERANCE
    for part in ("key", "query", "probability"):
        assert off(model(x, without=part), want) > 4 * TOLERANCE, part

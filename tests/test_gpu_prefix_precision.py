"""octopus_attn_decode_paged_prefix against 64 bits in the root mean square of a whole output: a tolerance that the loss of any part of
its operands is beyond (tests/test_prefix_precision.py shows that on the CPU, for the same inputs)."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding, layout

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, sign_bits_dev, to_dev  # noqa: E402
from prefix_model import CASES, G, N_KV, OWN, PREFIX, TOLERANCE, Inputs, off  # noqa: E402


def pages_of(cb, rec):
    """rec [kv, n, bytes] as pages [page, kv, ...]"""
    n = -(-rec.shape[1] // 64)
    return layout.records_to_cache(rec[None], cb.plan.granules, 64 * n).reshape(N_KV, n, -1).transpose(1, 0, 2)


def rows_of(v):
    n = -(-v.shape[1] // 64)
    return np.pad(v, ((0, 0), (0, 64 * n - v.shape[1]), (0, 0))).reshape(N_KV, n, 64, -1).transpose(1, 0, 2, 3)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d,bits", CASES)
def test_root_mean_square(d, bits, causal):
    x, cb = Inputs(d, bits), binding.octopus_build_codebooks(d, bits)
    k = np.concatenate([pages_of(cb, x.rec[:, :PREFIX]), pages_of(cb, x.rec[:, PREFIX:])])
    v = np.concatenate([rows_of(x.v[:, :PREFIX]), rows_of(x.v[:, PREFIX:])])
    shared = -(-PREFIX // 64)
    ints = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)  # noqa: E731
    ws = torch.empty(binding.octopus_attn_prefix_workspace(cb, 1, N_KV * G, N_KV, 1, PREFIX, OWN), dtype=torch.uint8, device=DEV)
    out = torch.zeros(x.q.shape, device=DEV)
    binding.octopus_attn_decode_paged_prefix(cb, to_dev(x.q, "fp32"), sign_bits_dev(x.signs), torch.from_numpy(np.ascontiguousarray(k)).to(DEV), to_dev(v, "bf16"),
                                             ints(list(range(shared))), ints([PREFIX]), PREFIX, ints([list(range(shared, len(k)))]), ints([OWN]), OWN,
                                             x.scale, out, ws, causal=causal)
    torch.cuda.synchronize()
    got = off(out.double().cpu().numpy(), x.exact())
    print(f"off by {got:.3g}")
    assert got <= TOLERANCE

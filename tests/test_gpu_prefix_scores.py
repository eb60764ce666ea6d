"""octopus_attn_decode_paged_prefix over scores of any size that fp32 holds: a softmax does not care how large they are.

Tolerance, by arithmetic.  A score is off by at most b = (d + 8) 2^-23 scale |q| |k| (as in test_gpu_prefix.py) plus half a step of its
own size, which b exceeds.  Where a row's largest score leads the others by more than 2 b + 60, their weights are below 2^-80 and the
output is that token's value: its probability is one, in bf16 as in fp32, and the values are bf16 (two roundings, of the sum and of the
division: 2^-23).  Any other row is an average of values, off by the 2^-16 of its probabilities."""
import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import to_dev  # noqa: E402
from test_gpu_prefix import Batch  # noqa: E402


def check(b, out):
    out = out.double().cpu().numpy()
    assert np.all(np.isfinite(out))
    sharp = 0
    for s, n in enumerate(b.lens):
        seen = b.prefix + n
        for h in range(b.n_qh):
            kvh = h * b.n_kv // b.n_qh
            keys, v = oracle.reconstruct(b.plan, b.rec[s, kvh, :seen], b.signs[kvh]), b.v[s, kvh, :seen].astype(np.float64)
            for i in range(b.n_q):
                q = b.q[s, i, h].astype(np.float64)
                score = b.scale * (keys @ q)
                slack = 2 * (b.d + 8) * 2.0 ** -23 * abs(b.scale) * np.linalg.norm(q) * np.max(np.linalg.norm(keys, axis=-1)) + 60.0
                best = int(np.argmax(score))
                big = np.max(np.abs(v))
                if np.max(np.delete(score, best), initial=-np.inf) < score[best] - slack:
                    assert np.all(np.abs(out[s, i, h] - v[best]) <= 2.0 ** -23 * np.abs(v[best])), (s, i, h)
                    sharp += 1
                else:
                    assert np.all(out[s, i, h] <= np.max(v, axis=0) + 2.0 ** -16 * big) and np.all(out[s, i, h] >= np.min(v, axis=0) - 2.0 ** -16 * big)
    return sharp


@pytest.mark.parametrize("size", [1e5, 1e9, 1e12, 1e20, 1e33])
@pytest.mark.parametrize("d,bits", [(64, 4), (128, 3), (128, 1.5), (256, 2.5)])
def test_large_scores(d, bits, size):
    """Queries of any size: the largest score's token, whatever steps fp32 has there."""
    b = Batch(d, bits, 4, 2, 2, 70, [90, 300, 20], seed=d, q_dtype="fp32")
    b.q = (b.q.astype(np.float64) * size).astype(np.float32)
    b.q_dev = to_dev(b.q, "fp32")
    assert check(b, b.call()) >= 16                  # of 24 rows


@pytest.mark.parametrize("size", [1.0, 1e31, -1e34])
def test_one_token_is_seen_whatever_its_score(size):
    """A single token's weight is one: also where its score is far below zero."""
    b = Batch(128, 3, 8, 2, 1, 0, [1, 1, 1], seed=3, q_dtype="fp32")
    b.q = (b.q.astype(np.float64) * size).astype(np.float32)
    b.q_dev = to_dev(b.q, "fp32")
    assert check(b, b.call()) == 24


def test_large_scales():
    """The same by way of the scale, with queries in bf16."""
    for scale in (1e7, -1e12, 1e30):
        b = Batch(128, 3, 4, 2, 1, 64, [40, 7], seed=9)
        b.scale = scale
        assert check(b, b.call()) >= 4               # of 8 rows

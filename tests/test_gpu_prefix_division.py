"""octopus_attn_decode_paged_prefix where a workgroup takes several segments one after the other (its tables kept, its staging areas
used again), and where a wavefront's steps outlast the page numbers that it holds.  Tolerances as in test_gpu_prefix.py."""
import numpy as np
import pytest

import oracle
from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, sign_bits_dev, to_dev  # noqa: E402
from prefix_shapes import LONG_RANGES, MANY_SEGMENTS  # noqa: E402
from test_gpu_prefix import Batch, bound, ints  # noqa: E402


@pytest.mark.parametrize("shape", MANY_SEGMENTS)
def test_workgroups_that_take_several_segments(shape):
    d, bits, n_qh, n_kv, n_q, prefix, lens, causal, q_lens = shape
    b = Batch(d, bits, n_qh, n_kv, n_q, prefix, lens, seed=d + n_q)
    out = b.call(q_lens=q_lens, causal=causal)
    b.check(out, q_lens=q_lens, causal=causal)
    assert torch.equal(b.call(q_lens=q_lens, causal=causal), out)


@pytest.mark.parametrize("shape", LONG_RANGES)
def test_ranges_that_outlast_the_held_page_numbers(shape):
    """Long contexts out of a few pages in random order: a page's tokens count as often as the table names it.  Every page's values
    have a level of their own, so that a wrong page moves the average."""
    d, bits, n_qh, n_kv, n_q, n_seq, prefix, own, causal = shape
    rng = np.random.default_rng(d + own)
    n_pages, g, scale = 48, n_qh // n_kv, d ** -0.5
    cb, plan = binding.octopus_build_codebooks(d, bits), oracle.make_plan(d, bits)
    signs = rng.integers(0, 2, size=(n_kv, d)).astype(np.int8) * 2 - 1
    keys = rng.standard_normal((1, n_pages * 64, n_kv, d)).astype(np.float32)
    v = to_dev(rng.standard_normal((n_pages, n_kv, 64, d)) + rng.permutation(n_pages)[:, None, None, None] / 8.0 - 3.0, "bf16")
    q = rng.standard_normal((n_seq, n_q, n_qh, d)).astype(np.float32)
    k_pool = torch.zeros(binding.octopus_paged_pool_bytes(cb, n_pages, n_kv), dtype=torch.uint8, device=DEV)
    signs_dev = sign_bits_dev(signs)
    binding.octopus_encode_paged(cb, to_dev(keys, "fp32"), signs_dev, k_pool, n_pages, ints(np.arange(n_pages)[None]))
    lens = rng.integers(own - own // 40, own + 1, n_seq)
    lens[0], lens[-1] = own, own
    prefix_table, table = rng.integers(0, n_pages, -(-prefix // 64)), rng.integers(0, n_pages, (n_seq, -(-own // 64)))
    ws = torch.empty(binding.octopus_attn_prefix_workspace(cb, n_seq, n_qh, n_kv, n_q, prefix, own), dtype=torch.uint8, device=DEV)
    out = torch.full((n_seq, n_q, n_qh, d), 77.0, device=DEV)
    binding.octopus_attn_decode_paged_prefix(cb, to_dev(q, "fp32"), signs_dev, k_pool, v, ints(prefix_table) if prefix else None, ints([prefix]), prefix,
                                             ints(table) if own else None, ints(lens), own, scale, out, ws, causal=causal)
    torch.cuda.synchronize()
    out = out.double().cpu().numpy()

    rec = k_pool.cpu().numpy().reshape(n_pages, n_kv, cb.plan.granules, 64, 16).transpose(1, 0, 3, 2, 4).reshape(n_kv, n_pages * 64, -1)
    rec = np.ascontiguousarray(rec[:, :, :cb.plan.record_bytes])
    values = v.double().cpu().numpy().transpose(1, 0, 2, 3).reshape(n_kv, n_pages * 64, d)

    def counts(pages, n):
        w = np.zeros(n_pages * 64)
        t = np.arange(n)
        np.add.at(w, np.asarray(pages)[t // 64] * 64 + t % 64, 1.0)
        return w

    shared = counts(prefix_table, prefix)
    mine = np.stack([[shared + counts(table[s], lens[s] - (n_q - 1 - i if causal else 0)) for i in range(n_q)] for s in range(n_seq)])
    for h in range(n_kv):
        k = oracle.reconstruct(plan, rec[h], signs[h])
        rows = q[:, :, h * g:(h + 1) * g].astype(np.float64)
        score = scale * (rows.reshape(-1, d) @ k.T).reshape(n_seq, n_q, g, -1)
        p = mine[:, :, None] * np.exp(score - score.max(axis=-1, keepdims=True))
        want = ((p / p.sum(axis=-1, keepdims=True)).reshape(-1, n_pages * 64) @ values[h]).reshape(n_seq, n_q, g, d)
        tol = bound(rows.reshape(-1, d)[np.argmax(np.linalg.norm(rows.reshape(-1, d), axis=-1))], np.linalg.norm(k, axis=-1), values[h], scale)
        assert np.max(np.abs(out[:, :, h * g:(h + 1) * g] - want)) <= tol

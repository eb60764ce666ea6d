"""The largest launches of octopus_read_paged: what the host lets through can be launched, and the next larger call is refused."""
import ctypes

import pytest

from paper_2605_21226_amd import binding

FAKE = 0x1000          # never dereferenced: the calls end before a launch
# head dimension, tokens of a sequence, KV heads, sequences
MOST = [(64, 2 ** 29 - 65, 1, 1), (256, 2 ** 29 - 128, 1, 1), (256, 64 * 1023 - 1, 8, 1024), (128, 64 * 2047 - 1, 64, 64)]
TOO_MANY = [(64, 2 ** 29 - 64, 1, 1), (256, 2 ** 29 - 127, 1, 1), (256, 64 * 1023, 8, 1024), (128, 64 * 2047, 64, 64)]


def call(cb, n_tok, n_kv, n_seq, table, pages, start, lens, pool, signs, out):
    return binding.load().octopus_read_paged(ctypes.byref(cb), signs, pool, None, 0, 0, 1, table, pages, n_seq, n_kv, start, n_tok, lens, out, None,
                                             binding.DTYPE_BF16, None)


@pytest.mark.parametrize("d,n_tok,n_kv,n_seq", TOO_MANY)
def test_larger_launches_are_refused(d, n_tok, n_kv, n_seq):
    cb = binding.octopus_build_codebooks(d, 2)
    assert call(cb, n_tok, n_kv, n_seq, FAKE, 4, FAKE, None, FAKE, FAKE, FAKE) == binding.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("d,n_tok,n_kv,n_seq", MOST)
def test_the_largest_launches(d, n_tok, n_kv, n_seq):
    """(no token of any sequence counts: the workgroups end at once, and neither pools nor outputs are looked at)"""
    torch = pytest.importorskip("torch")
    cb = binding.octopus_build_codebooks(d, 2)
    none = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    table = torch.zeros((n_seq, 4), dtype=torch.int32, device="cuda")
    pool = torch.zeros(binding.octopus_paged_pool_bytes(cb, 1, n_kv), dtype=torch.uint8, device="cuda")
    signs = torch.zeros((n_kv, d // 8), dtype=torch.uint8, device="cuda")
    out = torch.full((64, d), 3.0, dtype=torch.bfloat16, device="cuda")
    p = lambda t: t.data_ptr()  # noqa: E731
    assert call(cb, n_tok, n_kv, n_seq, p(table), 4, p(none), p(none), p(pool), p(signs), p(out)) == binding.OK
    torch.cuda.synchronize()
    assert bool((out == 3.0).all())

"""Calls over pages that the documentation allows beside the usual ones: queries and outputs that begin at any four bytes, keys and
values that heads or sequences share (strides of zero), queries of another type than the keys, counts outside their range."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV  # noqa: E402
from test_gpu_append import FILL, Setup, ints  # noqa: E402
from test_gpu_prefix import Batch  # noqa: E402


@pytest.mark.parametrize("d,bits", [(64, 4), (128, 3), (256, 2.5)])
@pytest.mark.parametrize("q_dtype,skip", [("fp32", 1), ("fp32", 3), ("bf16", 2), ("bf16", 6)])
def test_queries_and_outputs_that_begin_at_any_four_bytes(d, bits, q_dtype, skip):
    b = Batch(d, bits, 6, 2, 3, 100, [40, 7, 90], seed=d + skip, q_dtype=q_dtype)
    want = b.call(causal=True)
    n = b.q_dev.numel()
    room = torch.full((n + 8,), float("nan"), dtype=b.q_dev.dtype, device=DEV)
    room[skip:skip + n] = b.q_dev.flatten()
    q, b.q_dev = b.q_dev, room[skip:skip + n].view(b.q_dev.shape)
    assert b.q_dev.data_ptr() % 16 != 0 and b.q_dev.is_contiguous()
    out = torch.full((n + 8,), 77.0, device=DEV)
    got = b.call(causal=True, out=out[3:3 + n].view(q.shape))
    assert torch.equal(got, want) and bool((out[:3] == 77.0).all()) and bool((out[3 + n:] == 77.0).all())


def test_query_counts_outside_their_range():
    b = Batch(128, 3, 4, 2, 4, 50, [30, 30, 30], seed=5)
    want = b.call(q_lens=[4, 0, 0], causal=True)
    assert torch.equal(b.call(q_lens=[2 ** 31 - 1, -1, -2 ** 31], causal=True), want)


@pytest.mark.parametrize("n_new", [1, 70])
def test_keys_and_values_that_heads_or_sequences_share(n_new):
    for shared in (0, 2):                              # the sequences', or the heads' dimension
        a, b = (Setup(128, 3, 2, 4, 2, n_new, [3, 60], seed=4) for _ in range(2))
        k, v = (t.narrow(shared, 0, 1).expand(t.shape) for t in (a.k_dev, a.v_dev))
        assert k.stride(shared) == 0
        a.k_dev, a.v_dev, b.k_dev, b.v_dev = k, v, k.contiguous(), v.contiguous()
        a.append()
        b.append()
        assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool) and not bool((a.k_pool == FILL).all())


@pytest.mark.parametrize("n_new", [1, 70])
@pytest.mark.parametrize("kv,q,q_out", [("fp32", "bf16", "fp32"), ("bf16", "fp32", "bf16"), ("bf16", "bf16", "fp32"), ("fp32", "fp32", "bf16")])
def test_types_of_their_own(n_new, kv, q, q_out):
    """Keys, queries and rotated queries of any type each: the pages of the keys' type, the queries of theirs, rounded once."""
    kind = {"fp32": torch.float32, "bf16": torch.bfloat16}
    s = Setup(128, 3, 2, 2, 4, n_new, [5, 64], dtype=kv, seed=8)
    s.append()
    pages, values = s.k_pool.clone(), s.v_pool.clone()
    s.k_pool.fill_(FILL), s.v_pool.fill_(FILL)
    rows = s.q_dev.contiguous().to(kind[q])
    exact = torch.empty(rows.shape, dtype=torch.float32, device=DEV)
    s.append(q=rows.float(), q_out=exact)
    got = torch.empty(rows.shape, dtype=kind[q_out], device=DEV)
    s.append(q=rows, q_out=got)
    assert torch.equal(s.k_pool, pages) and torch.equal(s.v_pool, values)
    assert torch.equal(got, exact.to(kind[q_out]))


@pytest.mark.parametrize("heads", [1, 3, 24])
def test_one_sequences_and_many_in_a_call_give_the_same_bytes(heads):
    """A sequence's pages do not depend on the batch around it."""
    s = Setup(64, 2, 5, heads, 1, 40, [0, 63, 1, 200, 17], new_lens=[40, 3, 0, 40, 39], seed=heads)
    s.append()
    t = Setup(64, 2, 5, heads, 1, 40, [0, 63, 1, 200, 17], new_lens=[40, 3, 0, 40, 39], seed=heads)
    for i in range(5):
        one = slice(i, i + 1)
        out = torch.full((1, 40, heads, 64), 7.0, dtype=t.q_out.dtype, device=DEV)
        binding.octopus_append_paged(t.cb, t.k_dev[one], t.v_dev[one], t.signs_dev, t.k_pool, t.v_pool.view(torch.bfloat16), t.n_pages,
                                     t.block_dev[one].contiguous(), start_pos=ints(np.asarray(t.start)[one]), new_lens=ints(np.asarray(t.new_lens)[one]),
                                     rope=t.rope, q=t.q_dev[one], q_out=out)
        t.q_out[one] = out
    torch.cuda.synchronize()
    assert torch.equal(s.k_pool, t.k_pool) and torch.equal(s.v_pool, t.v_pool) and torch.equal(s.q_out, t.q_out)

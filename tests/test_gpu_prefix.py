"""GPU parity of octopus_attn_decode_paged_prefix against the oracle: sequences whose tokens are a shared prefix in pages of its own
and their own tokens in theirs.  The oracle sees each sequence whole and knows nothing of pages, prefixes or splits.

Tolerance, by arithmetic.  A score is a sum of d products of 22-bit operands added in fp32, so it is off by at most
(d + 8) 2^-23 scale |q| |k| (Cauchy-Schwarz); a probability by twice that (the score and the sum it is divided by) and by 2^-16 for
its two bf16 parts, the exponential and the sums; an output is an average of values with weights so far off."""
import numpy as np
import pytest

import oracle
from paper_2605_21226_amd import binding, layout, synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, record_gammas, sign_bits_dev, to_dev  # noqa: E402
from test_gpu_parity import make_inputs, oracle_attention_all  # noqa: E402


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def bound(q_row, gammas, v, scale):
    d = q_row.shape[-1]
    score = (d + 8) * 2.0 ** -23 * abs(scale) * np.linalg.norm(q_row) * np.max(gammas)
    return (2.0 ** -16 + 2.0 * score) * np.max(np.abs(v))


class Batch:
    """Keys, values and queries of sequences with a common prefix, in shuffled pages among unused ones full of garbage."""

    def __init__(self, d, bits, n_qh, n_kv, n_q, prefix, lens, seed, q_dtype="bf16", spare=3, slack=1):
        rng = np.random.default_rng(seed)
        self.d, self.n_qh, self.n_kv, self.n_q, self.prefix, self.lens = d, n_qh, n_kv, n_q, prefix, list(lens)
        self.cb, self.plan = binding.octopus_build_codebooks(d, bits), oracle.make_plan(d, bits)
        n_seq, longest = len(lens), max(max(lens), 1)
        self.scale = 1.0 / np.sqrt(d)
        keys, vals, self.signs = make_inputs(seed, n_seq, n_kv, prefix + longest, d, "bf16")
        self.v = vals.copy()                                    # [seq, kv, token, d]
        self.v[:, :, :prefix] = vals[:1, :, :prefix]
        enc = lambda k, h: oracle.encode(self.plan, k.astype(np.float64), self.signs[h])  # noqa: E731
        rb = self.plan.record_bytes
        self.rec = np.zeros((n_seq, n_kv, prefix + longest, rb), dtype=np.uint8)
        for h in range(n_kv):
            if prefix:
                self.rec[:, h, :prefix] = enc(keys[0, :prefix, h], h)
            for s in range(n_seq):
                self.rec[s, h, prefix:] = enc(keys[s, prefix:, h], h)
        self.q = synth.queries(seed, synth.Workload("t", n_seq, n_qh, n_kv, d, 64, bits, q_dtype, n_q=n_q))
        self.q_dev = to_dev(self.q, q_dtype)
        self.pp, self.op = -(-prefix // 64) + slack, -(-longest // 64) + slack
        self.n_pages = self.pp + n_seq * self.op + spare
        ids = rng.permutation(self.n_pages).astype(np.int32)
        self.prefix_table, self.table = ids[:self.pp], ids[self.pp:self.pp + n_seq * self.op].reshape(n_seq, self.op)
        tb = self.cb.plan.granules * 64 * 16
        k_pool = np.full((self.n_pages, n_kv, tb), 0xFF, dtype=np.uint8)        # norms that are no numbers
        v_pool = np.full((self.n_pages, n_kv, 64, d), np.nan, dtype=np.float32)

        def put(pages, rec, v):                                  # rec [kv, n, rb], v [kv, n, d]
            n = rec.shape[1]
            cap = -(-n // 64) * 64
            img = layout.records_to_cache(rec[None], self.cb.plan.granules, cap).reshape(n_kv, cap // 64, -1, 64, 16)
            for j in range(cap // 64):
                m = min(64, n - 64 * j)
                k_pool[pages[j]].reshape(n_kv, -1, 64, 16)[:, :, :m] = img[:, j, :, :m]
                v_pool[pages[j], :, :m] = v[:, 64 * j:64 * j + m]
        if prefix:
            put(self.prefix_table, self.rec[0, :, :prefix], self.v[0, :, :prefix])
        for s, n in enumerate(lens):
            if n:
                put(self.table[s], self.rec[s, :, prefix:prefix + n], self.v[s, :, prefix:prefix + n])
        self.k_pool, self.v_pool = torch.from_numpy(k_pool).to(DEV), to_dev(v_pool, "bf16")
        self.signs_dev = sign_bits_dev(self.signs)
        self.max_len = max(lens)

    def call(self, q_lens=None, causal=False, max_prefix=None, max_len=None, out=None, ws=None, stream=None):
        max_prefix = self.prefix if max_prefix is None else max_prefix
        max_len = self.max_len if max_len is None else max_len
        n_seq = len(self.lens)
        if ws is None:
            ws = torch.empty(binding.octopus_attn_prefix_workspace(self.cb, n_seq, self.n_qh, self.n_kv, self.n_q, max_prefix, max_len),
                             dtype=torch.uint8, device=DEV).fill_(0xFF)
        if out is None:
            out = torch.full((n_seq, self.n_q, self.n_qh, self.d), 77.0, dtype=torch.float32, device=DEV)
        binding.octopus_attn_decode_paged_prefix(
            self.cb, self.q_dev, self.signs_dev, self.k_pool, self.v_pool, ints(self.prefix_table), ints([self.prefix]), max_prefix,
            ints(self.table), ints(self.lens), max_len, self.scale, out, ws, q_lens=None if q_lens is None else ints(q_lens),
            causal=causal, stream=stream)
        torch.cuda.synchronize()
        return out

    def check(self, out, q_lens=None, causal=False):
        out = out.cpu().numpy()
        n_seq = len(self.lens)
        q_lens = [self.n_q] * n_seq if q_lens is None else q_lens
        gammas = record_gammas(self.rec)
        worst = 0.0
        for i in range(self.n_q):
            seen = [self.prefix + (max(0, min(n, n - m + i + 1)) if causal else n) for n, m in zip(self.lens, q_lens)]
            ref, _ = oracle_attention_all(self.plan, self.rec, self.signs, self.q[:, i:i + 1], self.v, seen, self.scale)
            for s in range(n_seq):
                for h in range(self.n_qh):
                    got = out[s, i, h]
                    if i >= q_lens[s]:
                        assert np.all(got == 77.0)
                    elif seen[s] == 0:
                        assert np.all(got == 0.0)
                    else:
                        kvh = h * self.n_kv // self.n_qh
                        tol = bound(self.q[s, i, h], gammas[s, kvh, :seen[s]], self.v[s, kvh, :seen[s]], self.scale)
                        err = np.max(np.abs(got - ref[s, 0, h]))
                        assert err <= tol, (s, i, h, err, tol)
                        worst = max(worst, err / tol)
        print(f"worst error {worst:.3g} of the bound")


@pytest.mark.parametrize("bits", [1, 1.5, 2, 2.5, 3, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_width(d, bits):
    b = Batch(d, bits, 4, 2, 1, 200, [70, 0, 33], seed=int(100 * bits) + d)
    b.check(b.call())


@pytest.mark.parametrize("n_qh,n_kv,n_q,prefix,lens", [
    (1, 1, 1, 1, [1]),                      # a token each
    (1, 1, 1, 0, [1, 0]),                   # no prefix; a sequence without a token
    (8, 1, 1, 64, [0, 0]),                  # no own tokens
    (4, 4, 1, 65, [63, 64, 65, 1, 31, 32]),
    (8, 2, 1, 1000, [5] * 9),               # 36 rows of the prefix per KV head: two groups
    (3, 1, 7, 31, [40, 300]),               # 21 own rows, one group, 42 of the prefix
    (6, 2, 12, 33, [12, 500]),              # 36 own rows: two groups
    (2, 2, 1, 3001, [2900, 1])])
def test_shapes(n_qh, n_kv, n_q, prefix, lens):
    b = Batch(128, 3, n_qh, n_kv, n_q, prefix, lens, seed=prefix + 7 * n_q)
    b.check(b.call())


@pytest.mark.parametrize("d,bits,n_q,prefix,lens,q_lens", [
    (128, 3, 5, 100, [5, 40, 133], None),
    (64, 4, 5, 70, [300, 5, 64], [5, 3, 1]),
    (64, 2, 40, 10, [40, 60], [40, 7]),
    (256, 2.5, 3, 0, [3, 1, 0], [3, 2, 3]),       # queries of more tokens than there are: the first see none
    (128, 2, 4, 20, [2, 0], [4, 0])])
def test_causal_and_padded(d, bits, n_q, prefix, lens, q_lens):
    b = Batch(d, bits, 4, 2, n_q, prefix, lens, seed=31 * n_q + prefix)
    b.check(b.call(q_lens=q_lens, causal=True), q_lens=q_lens, causal=True)
    b.check(b.call(q_lens=q_lens), q_lens=q_lens)


def test_fp32_queries_of_all_sizes_and_loose_bounds():
    """Queries as large as 10^6 and as small as 10^-6 (a row's scale is its own), host bounds far above the lengths."""
    b = Batch(128, 2.5, 8, 2, 1, 150, [20, 90], seed=5, q_dtype="fp32", slack=40)
    b.check(b.call(max_prefix=150 + 2000, max_len=90 + 2500))
    want = b.call()
    for factor in (1e6, 1e-6):
        b.q_dev = (b.q_dev * factor).contiguous()
        b.scale = b.scale / factor
        got = b.call()
        assert torch.allclose(got, want, rtol=2e-5, atol=2e-5)   # (the same scores, rounded anew)
        b.q_dev = to_dev(b.q, "fp32")
        b.scale = b.scale * factor


def test_the_same_call_gives_the_same_bits():
    b = Batch(128, 3, 8, 2, 2, 700, [90, 300, 20], seed=9)
    first = b.call(causal=True)
    for _ in range(5):
        assert torch.equal(b.call(causal=True), first)


def test_one_table_for_prefix_and_own_pages_agrees_with_the_paged_call():
    """A prefix of whole pages: octopus_attn_decode_paged over tables that begin with the prefix's pages."""
    b = Batch(128, 3, 8, 2, 1, 128, [50, 64, 7], seed=21)
    table = np.concatenate([np.tile(b.prefix_table[:2], (3, 1)), b.table], axis=1)
    lens = [128 + n for n in b.lens]
    ws = torch.empty(binding.octopus_attn_decode_workspace(b.cb, 3, 8, 2, 1, max(lens)), dtype=torch.uint8, device=DEV)
    out = torch.zeros((3, 1, 8, 128), dtype=torch.float32, device=DEV)
    binding.octopus_attn_decode_paged(b.cb, b.q_dev, b.signs_dev, b.k_pool, b.v_pool, ints(table), ints(lens), max(lens), b.scale, out, ws)
    torch.cuda.synchronize()
    got = b.call()
    assert torch.allclose(got, out, rtol=0, atol=2e-4 * float(out.abs().max()))   # (2^-13 of the row-group kernel's bf16 pairs)


@pytest.mark.parametrize("d,bits", [(64, 4), (128, 3), (128, 1.5), (256, 2.5)])
def test_tokens_a_query_does_not_see_have_no_say_whatever_they_are(d, bits):
    """Causal queries over own tokens whose last ones have values and keys that are no numbers: the queries that do not see them give
    the bits that they give with zeros there; of a value's channel that is none, those that do give none."""
    b = Batch(d, bits, 6, 2, 9, 40, [9, 70, 33], seed=d + 3)
    b.v_pool[b.v_pool.isnan()] = 0.0
    clean = b.call(causal=True)
    token = [5, 66, 30]                                     # of 9, 70 and 33: seen by the queries from 5, 5 and 6 on
    first = [5, 5, 6]
    for bad in (float("nan"), float("inf"), float("-inf")):
        v = b.v_pool.clone()
        for s, t in enumerate(token):
            v[b.table[s][t // 64], :, t % 64, 1::7] = bad
        b.v_pool, v = v, b.v_pool
        out = b.call(causal=True)
        b.v_pool = v
        for s in range(3):
            assert torch.equal(out[s, :first[s]], clean[s, :first[s]])
            hit = ~torch.isfinite(out[s, first[s]:])
            assert bool(hit[..., 1::7].all()) and int(hit.sum()) == hit[..., 1::7].numel()
    kp = b.k_pool.clone()
    for s, t in enumerate(token):                           # a norm that is no number, in the first four bytes of the record
        kp.view(b.n_pages, b.n_kv, -1, 64, 16)[int(b.table[s][t // 64]), :, 0, t % 64, :4] = 0xFF
    b.k_pool = kp
    out = b.call(causal=True)
    for s in range(3):
        assert torch.equal(out[s, :first[s]], clean[s, :first[s]]) and bool(out[s, first[s]:].isnan().all())


def test_values_that_are_no_numbers_stay_in_their_channel_and_sequence():
    b = Batch(128, 3, 8, 2, 1, 100, [50, 30], seed=14)
    clean = b.call()
    b.v_pool[int(b.table[0][0]), 1, 20, 5] = float("inf")
    out = b.call()
    assert torch.equal(out[1], clean[1]) and torch.equal(out[0, :, :4], clean[0, :, :4])      # (KV head 1 has query heads 4 .. 7)
    hit = ~torch.isfinite(out[0, :, 4:])
    assert bool(hit[..., 5].all()) and int(hit.sum()) == hit[..., 5].numel()


def test_garbage_in_queries_that_do_not_count():
    b = Batch(64, 3, 4, 2, 5, 60, [20, 40, 8], seed=8)
    q_lens = [5, 2, 0]
    want = b.call(q_lens=q_lens, causal=True)
    for s, n in enumerate(q_lens):
        b.q_dev[s, n:] = float("nan")
    assert torch.equal(b.call(q_lens=q_lens, causal=True), want)


@pytest.mark.parametrize("causal", [False, True])
def test_no_tokens_at_all(causal):
    b = Batch(128, 3, 8, 2, 2, 70, [30, 40], seed=3)
    assert bool((b.call(max_prefix=0, max_len=0, causal=causal) == 0).all())          # neither table is looked at
    b.prefix, b.lens = 0, [0, 0]
    assert bool((b.call(max_prefix=70, max_len=40, causal=causal) == 0).all())        # bounds of the host, lengths of the device
    b.prefix, b.lens = -5, [-1, -2 ** 31]
    assert bool((b.call(max_prefix=70, max_len=40, causal=causal) == 0).all())


def test_lengths_and_pages_outside_their_bounds_are_clamped():
    b = Batch(128, 3, 8, 2, 1, 128, [64, 64], seed=4, slack=0, spare=0)
    want = b.call()
    b.prefix, b.lens = 2 ** 31 - 1, [1000, 2 ** 31 - 1]
    assert torch.equal(b.call(max_prefix=128, max_len=64), want)
    b = Batch(128, 3, 8, 2, 1, 64, [64, 64], seed=4, slack=0, spare=0)
    b.prefix_table[0], b.table[0][0], b.table[1][0] = 0, b.n_pages - 1, 0
    want = b.call()
    b.prefix_table[0], b.table[0][0], b.table[1][0] = -7, 2 ** 31 - 1, -2 ** 31
    assert torch.equal(b.call(), want)


@pytest.mark.parametrize("scale", [0.0, -0.4, 3.0])
def test_scales(scale):
    b = Batch(128, 2, 4, 2, 1, 50, [40, 3], seed=6)
    b.scale = scale
    b.check(b.call())


def test_another_stream():
    """The call waits for what is on the stream that it is given, and for nothing else."""
    b = Batch(128, 3, 8, 2, 1, 900, [200, 100], seed=12)
    want = b.call()
    q, stream = b.q_dev.clone(), torch.cuda.Stream()
    for _ in range(3):
        b.q_dev.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            big = torch.ones(4096, 4096, device=DEV)
            for _ in range(4):
                big = big @ big * 1e-4                       # the stream has something to do first
            b.q_dev.copy_(q)
            assert torch.equal(b.call(stream=stream), want)


def test_profile_events_enclose_the_attention():
    b = Batch(128, 3, 8, 2, 1, 4000, [200, 100], seed=13)
    want = b.call()
    before, after = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    before.record(), after.record()
    torch.cuda.synchronize()
    binding.octopus_profile_events(before, after)
    assert torch.equal(b.call(), want)
    assert 0.0 < before.elapsed_time(after) < 1000.0
    first = before.elapsed_time(after)
    assert torch.equal(b.call(), want) and before.elapsed_time(after) == first       # one call only


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    d, bits = int(rng.choice([64, 128, 256])), float(rng.choice([1, 1.5, 2, 2.5, 3, 4]))
    n_kv, g, n_q = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 5, 8])), int(rng.choice([1, 1, 2, 3, 7, 11]))
    n_seq, prefix = int(rng.integers(1, 6)), int(rng.choice([0, 1, 31, 64, 97, 200, 450]))
    lens = [int(x) for x in rng.integers(0, 150, n_seq) * rng.integers(0, 2, n_seq) + rng.integers(0, 12, n_seq)]
    q_lens = [int(x) for x in rng.integers(0, n_q + 1, n_seq)] if seed % 2 else None
    b = Batch(d, bits, g * n_kv, n_kv, n_q, prefix, lens, seed=seed, q_dtype="fp32" if seed % 3 == 0 else "bf16")
    causal = bool(rng.integers(0, 2))
    b.check(b.call(q_lens=q_lens, causal=causal), q_lens=q_lens, causal=causal)
    b.check(b.call(q_lens=q_lens, causal=causal, max_prefix=64 * b.pp, max_len=64 * b.op), q_lens=q_lens, causal=causal)

"""GPU parity of octopus_append_paged and octopus_read_paged: records against the oracle's of keys rotated in 64 bits, values byte for
byte, rotated queries and reconstructed keys against 64 bits, and everything that a call may not touch.

Tolerances, by arithmetic.  A rotated channel is two products and a sum of fp32 numbers: off by at most 4 * 2^-24 of its pair's larger
channel; a rounding to bf16 adds 2^-8 of the value.  A reconstructed key is gamma s_j (H u^)_j: log2 d + 6 roundings of sums that
Cauchy-Schwarz bounds by gamma |u^|."""
import numpy as np
import pytest

import oracle
from paper_2605_21226_amd import binding, layout, synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, sign_bits_dev  # noqa: E402
from test_gpu_parity import compare_records  # noqa: E402

FILL = 0xA5


def ints(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def rope_table(n_pos, dim, seed=0):
    """(cos, sin) pairs, a little longer than one: tables may carry a scale."""
    angle = np.arange(n_pos)[:, None] * 10000.0 ** (-2.0 * np.arange(dim // 2) / dim)
    return (np.stack([np.cos(angle), np.sin(angle)], axis=-1) * 1.1).astype(np.float32)


def turned(x, table, pos, interleaved):
    """x [..., heads, d] of tokens at positions pos [...], in 64 bits."""
    y = x.astype(np.float64).copy()
    dim = 2 * table.shape[1]
    cs = table.astype(np.float64)[np.clip(pos, 0, len(table) - 1)][..., None, :, :]
    i = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    a, b = x[..., i[0]].astype(np.float64), x[..., i[1]].astype(np.float64)
    y[..., i[0]], y[..., i[1]] = a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]
    return y


class Setup:
    def __init__(self, d, bits, n_seq, n_kv, g, n_new, start, new_lens=None, dtype="bf16", rot=None, interleaved=False, rope_pos=None,
                 v_bits=0, v_group=0, pages=None, n_pos=4096, with_q=True, seed=0):
        rng = np.random.default_rng(seed + d + n_new)
        self.d, self.n_seq, self.n_kv, self.n_new, self.dtype = d, n_seq, n_kv, n_new, dtype
        self.cb, self.plan = binding.octopus_build_codebooks(d, bits), oracle.make_plan(d, bits)
        self.start = [0] * n_seq if start is None else list(start)
        self.new_lens = [n_new] * n_seq if new_lens is None else list(new_lens)
        self.v_bits, self.v_group, self.interleaved = v_bits, v_group, interleaved
        qkv = rng.standard_normal((n_seq, n_new, (g + 2) * n_kv, d)) * np.exp(0.5 * rng.standard_normal((1, 1, 1, d)))
        qkv = synth.round_to_bf16(qkv) if dtype == "bf16" else qkv.astype(np.float32)
        self.q, self.k, self.v = np.split(qkv, [g * n_kv, (g + 1) * n_kv], axis=2)
        self.qkv = torch.from_numpy(qkv).to(DEV, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
        self.q_dev, self.k_dev, self.v_dev = self.qkv.split([g * n_kv, n_kv, n_kv], dim=2)      # views with strides of their own
        if not with_q:
            self.q_dev = None
        self.table = None if rot == 0 else rope_table(n_pos, d if rot is None else rot)
        self.rope = None if self.table is None else torch.from_numpy(self.table).to(DEV)
        self.rope_pos = rope_pos
        s = rng.integers(0, 2, size=(n_kv, d)).astype(np.int8) * 2 - 1
        self.signs, self.signs_dev = s, sign_bits_dev(s)
        per = -(-(max(self.start) + n_new) // 64) if pages is None else pages
        self.n_pages = n_seq * per + 3
        self.block = rng.permutation(self.n_pages)[:n_seq * per].reshape(n_seq, per).astype(np.int32)
        self.block_dev, self.reach = ints(self.block), 64 * per
        self.k_pool = torch.full((binding.octopus_paged_pool_bytes(self.cb, self.n_pages, n_kv),), FILL, dtype=torch.uint8, device=DEV)
        row = binding.octopus_vq_row_bytes(d, v_bits, v_group) if v_bits else 2 * d
        self.v_pool = torch.full((self.n_pages, n_kv, 64, row), FILL, dtype=torch.uint8, device=DEV)
        self.q_out = torch.full((n_seq, n_new, g * n_kv, d), 7.0, dtype=self.qkv.dtype, device=DEV) if with_q else None
        self.start_dev = None if start is None else ints(start)
        self.lens_dev = None if new_lens is None else ints(new_lens)

    def positions(self):
        first = self.start if self.rope_pos is None else self.rope_pos
        return np.asarray(first)[:, None] + np.arange(self.n_new)[None]

    def append(self, part=slice(None), **more):
        v_pool = self.v_pool if self.v_bits else self.v_pool.view(torch.bfloat16)
        args = dict(start_pos=self.start_dev, new_lens=self.lens_dev, rope=self.rope, rope_interleaved=self.interleaved,
                    rope_pos=ints(self.rope_pos), q=self.q_dev, q_out=self.q_out, v_bits=self.v_bits, v_group=self.v_group)
        args.update(more)
        binding.octopus_append_paged(self.cb, self.k_dev[:, part], self.v_dev[:, part], self.signs_dev, self.k_pool, v_pool, self.n_pages,
                                     self.block_dev, **args)
        torch.cuda.synchronize()

    def written(self):
        """mask [page, slot] of what the call may write"""
        m = np.zeros((self.n_pages, 64), dtype=bool)
        for s in range(self.n_seq):
            for t in range(max(0, min(self.new_lens[s], self.n_new))):
                slot = self.start[s] + t
                if slot < self.reach:
                    m[self.block[s, slot // 64], slot % 64] = True
        return m

    def tokens(self, s):
        n = max(0, min(self.new_lens[s], self.n_new, self.reach - self.start[s]))
        slots = self.start[s] + np.arange(n)
        return n, self.block[s, slots // 64], slots % 64

    def check(self):
        gran = self.cb.plan.granules
        k = self.k_pool.cpu().numpy().reshape(self.n_pages, self.n_kv, gran, 64, 16)
        v = self.v_pool.cpu().numpy()
        m = self.written()
        assert np.all(np.moveaxis(k, 3, 1)[~m] == FILL) and np.all(np.moveaxis(v, 2, 1)[~m] == FILL)
        pos = self.positions()
        keys = self.k.astype(np.float64) if self.table is None else turned(self.k, self.table, pos, self.interleaved)
        for s in range(self.n_seq):
            n, page, off = self.tokens(s)
            if n == 0:
                continue
            rec = np.moveaxis(k[page, :, :, off], 1, 0).reshape(self.n_kv, n, gran * 16)
            assert np.all(rec[..., self.cb.plan.record_bytes:] == 0)
            compare_records(self.plan, keys[s:s + 1, :n], self.signs, rec[None, :, :, :self.cb.plan.record_bytes], f"append seq {s}", max_ties=2 + n // 50)
            rows = v[page, :, off]
            if self.v_bits:
                for h in range(self.n_kv):
                    want = oracle.vq_encode(self.v[s, :n, h].astype(np.float64), self.v_bits, self.v_group)
                    got = np.ascontiguousarray(rows[:, h])
                    assert np.mean(np.any(got != want, axis=-1)) <= 0.02      # (a quotient next to a half: see the byte-for-byte test)
            else:
                want = synth.round_to_bf16(self.v[s, :n])
                assert np.array_equal(np.ascontiguousarray(rows).view(np.uint16), synth.bf16_bits(want))
        if self.q_out is None:
            return
        out = self.q_out.float().cpu().numpy().astype(np.float64)
        want = self.q.astype(np.float64) if self.table is None else turned(self.q, self.table, pos, self.interleaved)
        big = np.max(np.abs(self.q), axis=-1, keepdims=True)
        tol = 4 * 1.1 * 2.0 ** -24 * big + (2.0 ** -8 * np.abs(want) if self.q_out.dtype == torch.bfloat16 else 0.0)
        for s in range(self.n_seq):
            n = max(0, min(self.new_lens[s], self.n_new))
            assert np.all(np.abs(out[s, :n] - want[s, :n]) <= tol[s, :n])
            assert np.all(out[s, n:] == 7.0)


@pytest.mark.parametrize("bits", [1, 1.5, 2, 2.5, 3, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_width_token_and_prompt(d, bits):
    a = Setup(d, bits, 3, 2, 2, 1, [5, 63, 64])               # a token per sequence
    a.append()
    a.check()
    a = Setup(d, bits, 2, 4, 2, 150, [0, 37])                 # workgroups over tiles
    a.append()
    a.check()


@pytest.mark.parametrize("kw", [
    dict(d=128, bits=3, n_seq=1, n_kv=1, g=1, n_new=1, start=None),
    dict(d=128, bits=3, n_seq=1, n_kv=8, g=1, n_new=200, start=None, rot=0),                       # no rotation
    dict(d=128, bits=2, n_seq=2, n_kv=8, g=4, n_new=70, start=[60, 1], rot=32, interleaved=True),
    dict(d=64, bits=4, n_seq=3, n_kv=8, g=3, n_new=65, start=[0, 63, 129], new_lens=[65, 0, 17], dtype="fp32", rot=16),
    dict(d=64, bits=3, n_seq=4, n_kv=2, g=2, n_new=2, start=[9, 62, 63, 0], new_lens=[2, 1, 0, -3], interleaved=True, rot=48),
    dict(d=256, bits=2.5, n_seq=2, n_kv=4, g=2, n_new=140, start=[3, 100], new_lens=[500, 139], dtype="fp32", rot=96),
    dict(d=256, bits=3, n_seq=2, n_kv=1, g=8, n_new=3, start=[126, 0], dtype="fp32"),
    dict(d=128, bits=3, n_seq=2, n_kv=8, g=2, n_new=100, start=[100, 10], pages=2),                 # past what the table reaches
    dict(d=128, bits=3, n_seq=2, n_kv=1, g=2, n_new=3, start=[127, 10], pages=2),
    dict(d=128, bits=3, n_seq=2, n_kv=8, g=2, n_new=90, start=[0, 64], rope_pos=[1000, 4050], n_pos=4096),   # positions of their own, past the table
    dict(d=128, bits=3, n_seq=2, n_kv=2, g=2, n_new=2, start=[0, 64], rope_pos=[-5, 4095], n_pos=4096),
    dict(d=128, bits=4, n_seq=2, n_kv=8, g=2, n_new=130, start=[7, 0], new_lens=[130, 65], v_bits=4, v_group=32),
    dict(d=64, bits=2, n_seq=2, n_kv=2, g=2, n_new=1, start=[7, 0], v_bits=2, v_group=16),
    dict(d=128, bits=3, n_seq=1, n_kv=3, g=1, n_new=400, start=[77], with_q=False)])
def test_shapes(kw):
    a = Setup(**kw)
    a.append()
    a.check()


@pytest.mark.parametrize("d,bits,n_new", [(128, 3, 1), (128, 2.5, 300), (64, 4, 3), (256, 2, 90)])
def test_without_rotation_the_bytes_are_those_of_the_separate_calls(d, bits, n_new):
    for v_bits, group in ((0, 0), (3, 32)):
        a = Setup(d, bits, 2, 8, 1, n_new, [5, 100], rot=0, v_bits=v_bits, v_group=group)
        a.append()
        want = torch.full_like(a.k_pool, FILL)
        binding.octopus_encode_paged(a.cb, a.k_dev, a.signs_dev, want, a.n_pages, a.block_dev, a.start_dev)
        torch.cuda.synchronize()
        assert torch.equal(a.k_pool, want)
        if v_bits:
            want = torch.full_like(a.v_pool, FILL)
            binding.octopus_encode_values_paged(a.v_dev, v_bits, group, want, a.n_kv, a.block_dev, a.start_dev)
            torch.cuda.synchronize()
            assert torch.equal(a.v_pool, want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_prompt_at_once_and_token_by_token_give_the_same_bytes(interleaved):
    a = Setup(128, 3, 1, 8, 2, 150, None, interleaved=interleaved)
    a.append()
    b = Setup(128, 3, 1, 8, 2, 150, None, interleaved=interleaved)
    for t in range(150):
        out = torch.empty_like(b.q_out[:, t:t + 1])
        b.append(slice(t, t + 1), start_pos=ints([t]), q=b.q_dev[:, t:t + 1], q_out=out)
        b.q_out[:, t:t + 1] = out
    assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool) and torch.equal(a.q_out, b.q_out)


def read(a, n_tok, start=None, lens=None, dtype=torch.float32, keys=True, values=True):
    shape = (a.n_seq, n_tok, a.n_kv, a.d)
    k = torch.full(shape, 9.0, dtype=dtype, device=DEV) if keys else None
    v = torch.full(shape, 9.0, dtype=dtype, device=DEV) if values else None
    v_pool = a.v_pool if a.v_bits else a.v_pool.view(torch.bfloat16)
    binding.octopus_read_paged(a.cb, a.signs_dev, a.k_pool, v_pool, a.n_pages, a.block_dev, k, v, start_pos=ints(start), lens=ints(lens),
                               v_bits=a.v_bits, v_group=a.v_group)
    torch.cuda.synchronize()
    return k, v


def check_read(a, n_tok, start, lens, k, v):
    gran = a.cb.plan.granules
    recs = a.k_pool.cpu().numpy().reshape(a.n_pages, a.n_kv, gran, 64, 16)
    rows = a.v_pool.cpu().numpy()
    half = 0.0 if (k if k is not None else v).dtype == torch.float32 else 2.0 ** -8
    for s in range(a.n_seq):
        first = 0 if start is None else max(0, start[s])
        n = max(0, min(n_tok if lens is None else lens[s], n_tok, a.reach - first))
        slots = first + np.arange(n)
        page, off = a.block[s, slots // 64], slots % 64
        for h in range(a.n_kv):
            if k is not None:
                got = k[s, :, h].double().cpu().numpy()
                assert np.all(got[n:] == 9.0)
                if n:
                    rec = recs[page, h, :, off].reshape(n, gran * 16)[:, :a.cb.plan.record_bytes]
                    want = oracle.reconstruct(a.plan, rec, a.signs[h])
                    norm = np.linalg.norm(want, axis=-1, keepdims=True)
                    tol = (np.log2(a.d) + 6) * 2.0 ** -24 * norm + half * np.abs(want)
                    assert np.all(np.abs(got[:n] - want) <= tol)
            if v is not None:
                got = v[s, :, h].double().cpu().numpy()
                assert np.all(got[n:] == 9.0)
                if n and a.v_bits:
                    want = oracle.vq_decode(np.ascontiguousarray(rows[page, h, off]), a.d, a.v_bits, a.v_group)
                    assert np.all(np.abs(got[:n] - want) <= (2.0 ** -24 + half) * np.abs(want) + 2.0 ** -24 * np.max(np.abs(want)))
                elif n:
                    bits = np.ascontiguousarray(rows[page, h, off]).view(np.uint16).astype(np.uint32) << 16
                    assert np.array_equal(got[:n], bits.view(np.float32).astype(np.float64))


@pytest.mark.parametrize("bits", [1, 1.5, 2, 2.5, 3, 4])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_read_every_width(d, bits):
    v_bits = int(bits) if bits in (2, 3, 4) else 0
    a = Setup(d, bits, 2, 2, 1, 200, None, v_bits=v_bits, v_group=16 if v_bits else 0, with_q=False)
    a.append()
    for dtype in (torch.float32, torch.bfloat16):
        check_read(a, 200, None, None, *read(a, 200, dtype=dtype))


@pytest.mark.parametrize("n_tok,start,lens", [(1, [63, 64], None), (70, [60, 0], [3, 0]), (300, [0, 190], [300, 7]), (64, [64, 128], [-1, 1000])])
def test_read_ranges_and_what_is_left_alone(n_tok, start, lens):
    a = Setup(128, 3, 2, 2, 1, 200, None, with_q=False)
    a.append()
    check_read(a, n_tok, start, lens, *read(a, n_tok, start, lens))
    k, _ = read(a, n_tok, start, lens, values=False)
    check_read(a, n_tok, start, lens, k, None)
    _, v = read(a, n_tok, start, lens, keys=False, dtype=torch.bfloat16)
    check_read(a, n_tok, start, lens, None, v)


def test_nothing_to_append_or_read():
    s = Setup(128, 3, 2, 2, 2, 4, [3, 60])
    empty = s.k_dev[:, :0].contiguous()
    binding.octopus_append_paged(s.cb, empty, empty, s.signs_dev, s.k_pool, s.v_pool.view(torch.bfloat16), s.n_pages, s.block_dev, start_pos=s.start_dev)
    s.append(new_lens=ints([0, -3]))
    assert bool((s.k_pool == FILL).all()) and bool((s.v_pool == FILL).all()) and bool((s.q_out == 7.0).all())
    out = torch.full((2, 4, 2, 128), 5.0, device=DEV)
    binding.octopus_read_paged(s.cb, s.signs_dev, s.k_pool, s.v_pool.view(torch.bfloat16), s.n_pages, s.block_dev, out[:, :0].contiguous(), None)
    binding.octopus_read_paged(s.cb, s.signs_dev, s.k_pool, s.v_pool.view(torch.bfloat16), s.n_pages, s.block_dev, out, out.clone(), lens=ints([0, -1]))
    torch.cuda.synchronize()
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("n_new", [1, 70])
def test_page_ids_outside_the_pool_are_clamped(n_new):
    a, b = (Setup(128, 3, 2, 2, 2, n_new, [3, 60], pages=3, seed=1) for _ in range(2))
    for s, ids in ((a, (0, a.n_pages - 1)), (b, (-2 ** 31, 2 ** 31 - 1))):
        s.block[:] = np.asarray([[3, 4, ids[0]], [5, 6, ids[1]]])[:, ::-1]
        s.block_dev = ints(s.block)
        s.append()
    assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool) and torch.equal(a.q_out, b.q_out)
    out = [torch.zeros((2, n_new, 2, 128), device=DEV) for _ in range(4)]
    for s, k, v in ((a, *out[:2]), (b, *out[2:])):
        binding.octopus_read_paged(s.cb, s.signs_dev, s.k_pool, s.v_pool.view(torch.bfloat16), s.n_pages, s.block_dev, k, v, start_pos=s.start_dev)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]) and float(out[0].abs().sum()) > 0


@pytest.mark.parametrize("n_new", [1, 130])
def test_keys_that_are_no_numbers_are_encoded_as_by_the_separate_call(n_new):
    s = Setup(128, 3, 2, 2, 2, n_new, [5, 64], rot=0)
    s.k_dev[0, 0, 0, 3], s.k_dev[1, n_new - 1, 1, 100], s.k_dev[1, 0, 0] = float("nan"), float("inf"), 0.0
    pool = torch.full_like(s.k_pool, FILL)
    binding.octopus_encode_paged(s.cb, s.k_dev.contiguous(), s.signs_dev, pool, s.n_pages, s.block_dev, s.start_dev)
    s.append()
    assert torch.equal(s.k_pool, pool)


def test_appending_on_another_stream():
    s, t = (Setup(128, 3, 2, 2, 2, 200, [5, 64], seed=2) for _ in range(2))
    s.append()
    stream, kept = torch.cuda.Stream(), t.qkv.clone()
    t.qkv.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        big = torch.ones(4096, 4096, device=DEV)
        for _ in range(4):
            big = big @ big * 1e-4
        t.qkv.copy_(kept)
        t.append(stream=stream)
    assert torch.equal(s.k_pool, t.k_pool) and torch.equal(s.v_pool, t.v_pool) and torch.equal(s.q_out, t.q_out)


@pytest.mark.parametrize("v_bits,v_group", [(0, 0), (3, 16)])
def test_reading_keys_or_values_alone(v_bits, v_group):
    s = Setup(128, 3, 2, 2, 1, 70, [5, 64], v_bits=v_bits, v_group=v_group)
    s.append()
    v_pool = s.v_pool if v_bits else s.v_pool.view(torch.bfloat16)
    both, alone = [torch.zeros((2, 70, 2, 128), device=DEV) for _ in range(2)], [torch.zeros((2, 70, 2, 128), device=DEV) for _ in range(2)]
    args = dict(start_pos=s.start_dev, v_bits=v_bits, v_group=v_group)
    binding.octopus_read_paged(s.cb, s.signs_dev, s.k_pool, v_pool, s.n_pages, s.block_dev, *both, **args)
    binding.octopus_read_paged(s.cb, s.signs_dev, s.k_pool, None, s.n_pages, s.block_dev, alone[0], None, **args)
    binding.octopus_read_paged(s.cb, None, None, v_pool, s.n_pages, s.block_dev, None, alone[1], **args)
    torch.cuda.synchronize()
    assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1]) and float(both[0].abs().min(dim=-1).values.max()) > 0


def test_queries_rotated_in_place_and_without_rotation():
    s = Setup(128, 3, 2, 2, 4, 50, [5, 64], new_lens=[50, 20])
    s.append()
    own = s.q_dev.contiguous()
    s.append(q=own, q_out=own)                                 # the rows are the call's own to overwrite
    assert torch.equal(own[0], s.q_out[0]) and torch.equal(own[1, :20], s.q_out[1, :20]) and torch.equal(own[1, 20:], s.q_dev[1, 20:])
    plain = torch.full_like(s.q_out, 7.0)
    s.append(rope=None, rope_pos=None, q_out=plain)
    assert torch.equal(plain[0], s.q_dev[0]) and bool((plain[1, 20:] == 7.0).all())

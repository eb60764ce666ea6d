"""A server's loop out of the calls that surround it, as they would be used: a system prompt appended once with the rotation by
position, sequences that go on from it with tokens of their own, the shared-prefix attention of every step over what was appended, and
the cache read back as values.  The attention is checked in 64 bits over the keys and values that reading gives, the keys themselves
against rotated ones; a captured step gives the eager one's bits.

Tolerances, by arithmetic.  Attention: a score is off by (2 d + 40) 2^-23 scale |q| |k| (the kernel's operands have 22 bits; the read
keys are off by log2 d + 6 roundings), an output by twice that and 2^-16, of the largest value; queries in fp32.  Keys: the codec's own
error, 11 % of a key's norm on average at 3 bits; 30 % bounds each."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, sign_bits_dev  # noqa: E402
from test_gpu_append import ints, rope_table, turned  # noqa: E402


class Server:
    def __init__(self, d, bits, n_seq, n_kv, g, prefix, pages, seed=0):
        rng = np.random.default_rng(seed)
        self.d, self.n_seq, self.n_kv, self.g, self.prefix = d, n_seq, n_kv, g, prefix
        self.cb = binding.octopus_build_codebooks(d, bits)
        self.signs = sign_bits_dev(rng.integers(0, 2, size=(n_kv, d)).astype(np.int8) * 2 - 1)
        self.prefix_pages = -(-prefix // 64)
        self.n_pages = self.prefix_pages + n_seq * pages + 2
        ids = rng.permutation(self.n_pages)
        self.prefix_table = ints(ids[:self.prefix_pages])
        self.table = ints(ids[self.prefix_pages:self.prefix_pages + n_seq * pages].reshape(n_seq, pages))
        self.k_pool = torch.zeros(binding.octopus_paged_pool_bytes(self.cb, self.n_pages, n_kv), dtype=torch.uint8, device=DEV)
        self.v_pool = torch.full((self.n_pages, n_kv, 64, d), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.max_len = 64 * pages
        self.cos_sin = rope_table(prefix + self.max_len, d)
        self.rope = torch.from_numpy(self.cos_sin).to(DEV)
        self.start, self.lens, self.pos = ints([0] * n_seq), ints([0] * n_seq), ints([prefix] * n_seq)
        self.prefix_len = ints([prefix])
        self.ws = torch.empty(binding.octopus_attn_prefix_workspace(self.cb, n_seq, n_kv * g, n_kv, 4, prefix, self.max_len), dtype=torch.uint8,
                              device=DEV)
        self.scale = d ** -0.5

    def prompt(self, qkv):
        """the prefix's tokens, [1, prefix, (g + 2) heads, d]"""
        _, k, v = qkv.split([self.n_kv * self.g, self.n_kv, self.n_kv], dim=2)
        binding.octopus_append_paged(self.cb, k, v, self.signs, self.k_pool, self.v_pool, self.n_pages, self.prefix_table.view(1, -1), rope=self.rope)

    def step(self, qkv, q_rot, out, new, n_new):
        """every sequence's next tokens (new[s] of them at most count): appended, and attended to"""
        q, k, v = qkv.split([self.n_kv * self.g, self.n_kv, self.n_kv], dim=2)
        binding.octopus_append_paged(self.cb, k, v, self.signs, self.k_pool, self.v_pool, self.n_pages, self.table, start_pos=self.start,
                                     new_lens=new, rope=self.rope, rope_pos=self.pos, q=q, q_out=q_rot)
        self.start.add_(new)
        self.pos.add_(new)
        binding.octopus_attn_decode_paged_prefix(self.cb, q_rot, self.signs, self.k_pool, self.v_pool, self.prefix_table, self.prefix_len,
                                                 self.prefix, self.table, self.start, self.max_len, self.scale, out, self.ws, q_lens=new,
                                                 causal=n_new > 1)

    def read(self, table, n):
        k = torch.empty((table.shape[0], n, self.n_kv, self.d), dtype=torch.float32, device=DEV)
        v = torch.empty_like(k)
        binding.octopus_read_paged(self.cb, self.signs, self.k_pool, self.v_pool, self.n_pages, table, k, v)
        return k.double().cpu().numpy(), v.double().cpu().numpy()


def attention(q, k, v, scale):
    """q [heads, d], k and v [tokens, kv, d] in 64 bits"""
    g = q.shape[0] // k.shape[1]
    out, big = np.zeros_like(q), np.zeros(q.shape[0])
    for h in range(q.shape[0]):
        s = scale * (k[:, h // g] @ q[h])
        p = np.exp(s - s.max())
        out[h] = p @ v[:, h // g] / p.sum()
        big[h] = np.max(np.abs(v[:, h // g])) * (2.0 ** -16 + 2 * (2 * len(q[h]) + 40) * 2.0 ** -23 * abs(scale) * np.linalg.norm(q[h]) *
                                                  np.max(np.linalg.norm(k[:, h // g], axis=-1)))
    return out, big


@pytest.mark.parametrize("d,bits,n_seq,n_kv,g,prefix,steps", [
    (128, 3, 3, 2, 4, 333, [70, 1, 3, 1]),
    (64, 4, 5, 3, 1, 64, [1, 4, 64]),
    (256, 2.5, 2, 1, 2, 131, [20, 2])])
def test_prompt_steps_attention_and_reading(d, bits, n_seq, n_kv, g, prefix, steps):
    rng = np.random.default_rng(d + prefix)
    srv = Server(d, bits, n_seq, n_kv, g, prefix, -(-sum(steps) // 64), seed=prefix)
    rows = lambda b, n: rng.standard_normal((b, n, (g + 2) * n_kv, d)).astype(np.float32)  # noqa: E731
    first = rows(1, prefix)
    srv.prompt(torch.from_numpy(first).to(DEV))
    all_k = [[] for _ in range(n_seq)]
    total = np.zeros(n_seq, dtype=int)
    for n in steps:
        counts = [max(0, n - s) for s in range(n_seq)]                   # a padded batch
        qkv = rows(n_seq, n)
        q_rot = torch.zeros((n_seq, n, n_kv * g, d), dtype=torch.float32, device=DEV)
        out = torch.full_like(q_rot, 5.0)
        srv.ws = torch.empty(binding.octopus_attn_prefix_workspace(srv.cb, n_seq, n_kv * g, n_kv, n, prefix, srv.max_len), dtype=torch.uint8, device=DEV)
        srv.step(torch.from_numpy(qkv).to(DEV), q_rot, out, ints(counts), n)
        shared_k, shared_v = srv.read(srv.prefix_table.view(1, -1), prefix)
        own_k, own_v = srv.read(srv.table, int(total.max()) + n)
        q_rot, out = q_rot.double().cpu().numpy(), out.double().cpu().numpy()
        for s in range(n_seq):
            pos = prefix + total[s] + np.arange(counts[s])
            keys = turned(qkv[s, :counts[s], g * n_kv:(g + 1) * n_kv], srv.cos_sin, pos, False)
            queries = turned(qkv[s, :counts[s], :g * n_kv], srv.cos_sin, pos, False)
            got = own_k[s, total[s]:total[s] + counts[s]]
            assert np.all(np.linalg.norm(got - keys, axis=-1) <= (0.3 if bits >= 2.5 else 0.6) * np.linalg.norm(keys, axis=-1))
            assert np.all(np.abs(q_rot[s, :counts[s]] - queries) <= 6 * 2.0 ** -24 * np.max(np.abs(queries), initial=0.0))
            for i in range(n):
                if i >= counts[s]:
                    assert np.all(out[s, i] == 5.0)
                    continue
                seen = total[s] + i + 1
                k = np.concatenate([shared_k[0], own_k[s, :seen]])
                v = np.concatenate([shared_v[0], own_v[s, :seen]])
                want, tol = attention(q_rot[s, i], k, v, srv.scale)
                assert np.all(np.abs(out[s, i] - want) <= tol[:, None]), (n, s, i, np.max(np.abs(out[s, i] - want) / tol[:, None]))
        total += counts


def test_steps_captured_and_replayed_with_one_workspace():
    """Two graphs, of steps of one token and of four, that share the workspace; each replayed several times in turn, with eager work and
    synchronisations between the replays: the eager loop's bits."""
    d, n_seq, n_kv, g, prefix = 128, 3, 2, 4, 500
    rng = np.random.default_rng(77)
    plan = [1, 4, 1, 1, 4, 4, 1, 4]
    first = torch.from_numpy(rng.standard_normal((1, prefix, (g + 2) * n_kv, d)).astype(np.float32)).to(DEV, torch.bfloat16)
    inputs = [torch.from_numpy(rng.standard_normal((n_seq, n, (g + 2) * n_kv, d)).astype(np.float32)).to(DEV, torch.bfloat16) for n in plan]
    counts = [ints([n, max(1, n - 2), n]) for n in plan]

    def buffers(n):
        q_rot = torch.zeros((n_seq, n, n_kv * g, d), dtype=torch.bfloat16, device=DEV)
        return torch.zeros((n_seq, n, (g + 2) * n_kv, d), dtype=torch.bfloat16, device=DEV), q_rot, torch.zeros(q_rot.shape, device=DEV), ints([0] * n_seq)

    eager, want = Server(d, 3, n_seq, n_kv, g, prefix, 1, seed=5), []
    eager.prompt(first)
    buf = {n: buffers(n) for n in (1, 4)}
    for n, x, c in zip(plan, inputs, counts):
        buf[n][0].copy_(x), buf[n][3].copy_(c), buf[n][2].fill_(9.0)
        eager.step(*buf[n], n)
        torch.cuda.synchronize()
        want.append(buf[n][2].clone())

    srv = Server(d, 3, n_seq, n_kv, g, prefix, 1, seed=5)
    srv.prompt(first)
    graphs = {}
    for n in (1, 4):
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n]):
            srv.step(*buf[n], n)
    for t, (n, x, c) in enumerate(zip(plan, inputs, counts)):
        buf[n][0].copy_(x), buf[n][3].copy_(c), buf[n][2].fill_(9.0)
        srv.ws.fill_(0xFF)                                               # (scratch: nothing of it outlives a call)
        torch.cuda.synchronize()
        graphs[n].replay()
        torch.cuda.synchronize()
        assert torch.equal(buf[n][2], want[t]), t
    assert torch.equal(srv.k_pool, eager.k_pool) and torch.equal(srv.start, eager.start)
    assert torch.equal(srv.v_pool.view(torch.int16), eager.v_pool.view(torch.int16))


def test_pages_behind_four_gibibytes():
    """The same steps with their pages at a pool's end, whose offsets pass 32 bits in either pool, and at its beginning."""
    d, n_seq, n_kv, g, prefix = 256, 2, 8, 2, 130
    rng = np.random.default_rng(3)
    rows = lambda b, n: torch.from_numpy(rng.standard_normal((b, n, (g + 2) * n_kv, d)).astype(np.float32)).to(DEV, torch.bfloat16)  # noqa: E731
    first, new, got = rows(1, prefix), rows(n_seq, 4), []
    for n_pages in (0, 90_000):
        srv = Server(d, 4, n_seq, n_kv, g, prefix, 1, seed=1)
        if n_pages:
            shift = n_pages - srv.n_pages
            srv.n_pages, srv.prefix_table, srv.table = n_pages, srv.prefix_table + shift, srv.table + shift
            srv.k_pool = torch.empty(binding.octopus_paged_pool_bytes(srv.cb, n_pages, n_kv), dtype=torch.uint8, device=DEV)
            srv.v_pool = torch.empty((n_pages, n_kv, 64, d), dtype=torch.bfloat16, device=DEV)
            assert srv.k_pool.numel() > 2 ** 32 and int(srv.table.min()) * (srv.k_pool.numel() // n_pages) > 2 ** 32
        srv.prompt(first)
        q_rot = torch.empty((n_seq, 4, n_kv * g, d), dtype=torch.bfloat16, device=DEV)
        out = torch.empty(q_rot.shape, device=DEV)
        srv.step(new, q_rot, out, ints([4, 4]), 4)
        got.append((out, *srv.read(srv.table, 4), *srv.read(srv.prefix_table.view(1, -1), prefix)))
    assert torch.equal(got[0][0], got[1][0]) and bool(torch.isfinite(got[0][0]).all())
    for a, b in zip(got[0][1:], got[1][1:]):
        assert np.array_equal(a, b)

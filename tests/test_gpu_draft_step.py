"""A server's steps with drafts, put together: pages for the next tokens with forks and trims (octopus_pages_update, octopus_pages_copy), the
tokens appended by positions on several axes (octopus_append_paged_axes), attention over the pages (octopus_attn_decode_paged_prefix, causal), drafts verified
(octopus_verify_drafts), and the pages moved together now and then (octopus_pages_compact, octopus_pages_rename).

The attention's results go by lengths and contents alone, and a prompt appended at once has the bytes of one appended bit by bit: so every step's are
equal, bit for bit, to those over pages of the test's own, into which each sequence's whole history has been appended at once and which nothing shares.
The tokens are equal to the definition's (tests/verify_model.py), the pages to the sequential model's (tests/pages_model.py)."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding, synth
from pages_model import Pages, ceil
from verify_model import verify

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV, sign_bits_dev  # noqa: E402
from test_gpu_append import rope_table  # noqa: E402

N_SEQ, N_KV, N_QH, D, N_DRAFT, VOCAB, N_AXES, PER, N_PAGES, LAYERS = 6, 2, 4, 128, 4, 300, 3, 8, 60, 2
N_NEW = N_DRAFT + 1


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def pages_for(cb, n_pages):
    k = torch.zeros((LAYERS, n_pages, binding.octopus_paged_pool_bytes(cb, 1, N_KV)), dtype=torch.uint8, device=DEV)
    return k, torch.zeros((LAYERS, n_pages, N_KV, 64, D), dtype=torch.bfloat16, device=DEV)


class Step:
    """The buffers of a server's step, and the step."""

    def __init__(self):
        self.cb = binding.octopus_build_codebooks(D, 3)
        self.signs = sign_bits_dev(synth.sign_vectors(5, N_KV, D))
        self.rope = torch.from_numpy(rope_table(2000, D)).to(DEV)
        self.axis = bytes([0] * 16 + [1] * 24 + [2] * 24)
        self.refs, self.table = torch.zeros(N_PAGES, dtype=torch.int32, device=DEV), torch.zeros((N_SEQ, PER), dtype=torch.int32, device=DEV)
        self.k_pools, self.v_pools = pages_for(self.cb, N_PAGES)
        self.pools = binding.page_pools([*self.k_pools, *self.v_pools])
        self.moves, self.map = torch.zeros(2 + N_PAGES, dtype=torch.int32, device=DEV), torch.zeros(N_PAGES, dtype=torch.int32, device=DEV)
        self.ws_pages = torch.empty(binding.octopus_pages_workspace(N_PAGES, N_SEQ, PER), dtype=torch.uint8, device=DEV)
        self.ws_attn = torch.empty(binding.octopus_attn_prefix_workspace(self.cb, N_SEQ, N_QH, N_KV, N_NEW, 0, PER * 64), dtype=torch.uint8, device=DEV)
        self.ws_verify = torch.empty(binding.octopus_verify_workspace(N_SEQ, N_DRAFT, VOCAB), dtype=torch.uint8, device=DEV)
        # what the step goes by, set before it, and what it leaves
        self.lens, self.keep, self.new, self.source = (torch.zeros(N_SEQ, dtype=torch.int32, device=DEV) for _ in range(4))
        self.qkv = torch.zeros((LAYERS, N_SEQ, N_NEW, N_QH + 2 * N_KV, D), dtype=torch.bfloat16, device=DEV)
        self.pos = torch.zeros((N_AXES, N_SEQ, N_NEW), dtype=torch.int32, device=DEV)
        self.target = torch.zeros((N_SEQ, N_NEW, VOCAB), dtype=torch.float32, device=DEV)
        self.draft = torch.zeros((N_SEQ, N_DRAFT, VOCAB), dtype=torch.float32, device=DEV)
        self.x, self.u = torch.zeros((N_SEQ, N_DRAFT), dtype=torch.int32, device=DEV), torch.zeros((N_SEQ, N_NEW), dtype=torch.float32, device=DEV)
        self.q_rot = torch.zeros((LAYERS, N_SEQ, N_NEW, N_QH, D), dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros((LAYERS, N_SEQ, N_NEW, N_QH, D), dtype=torch.float32, device=DEV)
        self.tokens, self.accepted = torch.zeros((N_SEQ, N_NEW), dtype=torch.int32, device=DEV), torch.zeros(N_SEQ, dtype=torch.int32, device=DEV)

    def set(self, **values):
        for name, value in values.items():
            getattr(self, name).copy_(value if isinstance(value, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(value)))

    def append(self, layer, pools, table, qkv, pos, start, q_out):
        q, k, v = qkv.split([N_QH, N_KV, N_KV], dim=2)
        binding.octopus_append_paged_axes(self.cb, k, v, self.signs, pools[0][layer], pools[1][layer], pools[0].shape[1], table, self.rope, self.axis,
                                          pos.permute(1, 2, 0), start_pos=start, q=q, q_out=q_out)

    def attend(self, layer, pools, table, q, lens, out):
        binding.octopus_attn_decode_paged_prefix(self.cb, q, self.signs, pools[0][layer], pools[1][layer], None, None, 0, table, lens, PER * 64, D ** -0.5, out,
                                                 self.ws_attn, causal=True)

    def run(self):
        binding.octopus_pages_update(self.refs, self.table, self.lens, self.new, self.moves, self.ws_pages, source=self.source, keep_lens=self.keep)
        binding.octopus_pages_copy(self.pools, self.moves)
        for layer in range(LAYERS):
            self.append(layer, (self.k_pools, self.v_pools), self.table, self.qkv[layer], self.pos, self.keep, self.q_rot[layer])
            self.attend(layer, (self.k_pools, self.v_pools), self.table, self.q_rot[layer], self.lens, self.out[layer])
        binding.octopus_verify_drafts(self.target, self.draft, self.x, self.u, self.tokens, self.accepted, self.ws_verify)

    def compact(self):
        binding.octopus_pages_compact(self.refs, self.map, self.moves, self.ws_pages)
        binding.octopus_pages_copy(self.pools, self.moves)
        binding.octopus_pages_rename(self.map, self.table, self.lens)

    def state(self):
        return [self.refs, self.table, self.lens, self.moves[:2], self.k_pools, self.v_pools, self.q_rot, self.out, self.tokens, self.accepted]


class Server:
    """What is asked of the steps, and each slot's history on the host."""

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.keep = np.zeros(N_SEQ, dtype=np.int32)
        self.history = [(torch.zeros((LAYERS, 0, N_QH + 2 * N_KV, D), dtype=torch.bfloat16, device=DEV), np.zeros((N_AXES, 0), dtype=np.int32)) for _ in range(N_SEQ)]

    def next(self, n):
        """Inputs of step n: what of each slot's tokens is kept, whom it goes on from, the new tokens and the drafts' probabilities."""
        rng = self.rng
        source = np.arange(N_SEQ, dtype=np.int32)
        if n % 2:
            source = np.where(rng.random(N_SEQ) < 0.6, source, rng.integers(0, N_SEQ, size=N_SEQ)).astype(np.int32)
        if n == 5:
            source[3] = -1                                       # a sequence ends, another begins there
        keep = np.where(source < 0, 0, self.keep[np.maximum(source, 0)]).astype(np.int32)
        pos = (keep[None, :, None] // np.array([40, 8, 1])[:, None, None] + np.arange(N_NEW) * rng.integers(0, 2, size=(N_AXES, N_SEQ, 1))).astype(np.int32)
        qkv = torch.randn((LAYERS, N_SEQ, N_NEW, N_QH + 2 * N_KV, D), generator=self.g, device=DEV).bfloat16()
        target = torch.softmax(4 * torch.randn((N_SEQ, N_NEW, VOCAB), generator=self.g, device=DEV), -1)
        draft = 0.3 * torch.softmax(4 * torch.randn((N_SEQ, N_DRAFT, VOCAB), generator=self.g, device=DEV), -1) + 0.7 * target[:, :N_DRAFT]
        x = torch.multinomial(draft.reshape(-1, VOCAB).cpu(), 1, generator=torch.Generator().manual_seed(n)).view(N_SEQ, N_DRAFT).int()
        u = rng.random((N_SEQ, N_NEW), dtype=np.float32)
        self.asked = dict(source=source, keep=keep, new=keep + N_NEW, pos=pos, qkv=qkv, target=target, draft=draft, x=x, u=u)
        self.history = [(torch.cat([self.history[s][0][:, :keep[i]], qkv[:, i]], 1), np.concatenate([self.history[s][1][:, :keep[i]], pos[:, i]], 1))
                        for i, s in enumerate(source)]
        return self.asked

    def check(self, step):
        a = self.asked
        want = [verify(a["target"][s].cpu().numpy(), a["draft"][s].cpu().numpy(), a["x"][s].numpy(), a["u"][s], N_DRAFT) for s in range(N_SEQ)]
        assert step.tokens.tolist() == [t for t, _ in want] and step.accepted.tolist() == [n for _, n in want]
        # the whole history at once, in pages that nothing shares
        pools, table = pages_for(step.cb, N_SEQ * PER), torch.arange(N_SEQ * PER, dtype=torch.int32, device=DEV).view(N_SEQ, PER)
        for layer in range(LAYERS):
            for s, (qkv, pos) in enumerate(self.history):
                qkv = qkv[layer][None].contiguous()
                step.append(layer, pools, table[s:s + 1], qkv, ints(pos[:, None]), None, torch.zeros((1, qkv.shape[1], N_QH, D), dtype=torch.bfloat16, device=DEV))
            out = torch.zeros_like(step.out[layer])
            step.attend(layer, pools, table, step.q_rot[layer], ints(a["new"]), out)
            torch.cuda.synchronize()
            assert torch.equal(out, step.out[layer]) and bool(out.abs().sum(-1).gt(0).all())
        self.keep = a["keep"] + 1 + np.array([n for _, n in want], dtype=np.int32)     # (the token after the drafts is the next step's first)
        self.keep = np.minimum(self.keep, a["new"])


def test_steps_with_forks_trims_and_compaction():
    step, server = Step(), Server(1)
    model = Pages(np.zeros(N_PAGES), np.zeros((N_SEQ, PER)), np.zeros(N_SEQ))
    copied = 0
    for n in range(60):
        a = server.next(n)
        step.set(**a)
        step.run()
        torch.cuda.synchronize()
        model.update(a["new"], a["source"], a["keep"])
        copied += len(model.moves)
        assert step.moves[:2].tolist() == [len(model.moves), 0]
        assert np.array_equal(step.table.cpu().numpy(), model.table) and np.array_equal(step.refs.cpu().numpy(), model.refs)
        server.check(step)
        if n % 7 == 6:
            step.compact()
            model.rename(model.compact())
            assert np.array_equal(step.table.cpu().numpy(), model.table) and np.array_equal(step.refs.cpu().numpy(), model.refs)
        model.check()
    assert copied > 20 and max(ceil(int(n)) for n in model.lens) >= 3


def test_a_captured_step():
    """The step captured once and replayed with its inputs changed in place, eager steps of another server between: both leave the same, bit for bit."""
    eager, captured, server = Step(), Step(), Server(2)
    for s in (eager, captured):
        s.run()                                     # (nothing is asked for: no tokens, no pages)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for n in range(8):
        a = server.next(n)
        eager.set(**a)
        captured.set(**a)
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        for x, y in zip(eager.state(), captured.state()):
            assert torch.equal(x, y)
        server.check(captured)

"""GPU tests of octopus_verify_drafts against its definition (tests/verify_model.py): every token and count equal.

Why equal and not nearly: the test of a draft is exact on both sides (a product of two 24-bit numbers in 64 bits).  A drawn token differs only
if the goal u' sum r lies within the sums' rounding, at most vocab 2^-53 of the sum and less than 2^-35 for every vocabulary here, of a border
between two tokens; u' is a multiple of 2^-24, drawn from all of them, so a draw comes that near with a probability of about the number
of borders times 2^-35, under 1e-5 for the largest of these rows and far less for all others together.  Rows of few
dyadic numbers, whose sums are exact, test the borders themselves."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding
from verify_model import verify

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def distributions(rng, shape, dtype, peak=3.0, zeros=0.0):
    x = rng.standard_normal(shape) * peak
    p = np.exp(x - x.max(-1, keepdims=True))
    p[rng.random(shape) < zeros] = 0.0
    p /= np.maximum(p.sum(-1, keepdims=True), 1e-30)
    return torch.from_numpy(p.astype(np.float32)).to(TYPES[dtype])


class Batch:
    def __init__(self, n_seq, n_draft, vocab, dtype="fp32", sampled=True, ragged=False, agree=0.5, zeros=0.0, seed=0):
        rng = np.random.default_rng([seed, n_seq, n_draft, vocab])
        self.target = distributions(rng, (n_seq, n_draft + 1, vocab), dtype, zeros=zeros)
        mix = distributions(rng, (n_seq, n_draft, vocab), dtype, zeros=zeros)
        self.draft = ((1 - agree) * mix.float() + agree * self.target[:, :n_draft].float()).to(TYPES[dtype])
        q = self.draft.float().numpy().astype(np.float64).reshape(-1, vocab)
        at = np.cumsum(q, axis=1)
        self.x = np.minimum((at < rng.random((len(q), 1)) * at[:, -1:]).sum(1), vocab - 1).reshape(n_seq, n_draft).astype(np.int32)
        self.draft = self.draft if sampled else None
        self.u = rng.integers(0, 1 << 24, size=(n_seq, n_draft + 1)).astype(np.float32) * np.float32(2.0 ** -24)
        self.lens = rng.integers(0, n_draft + 1, size=n_seq).astype(np.int32) if ragged else None
        self.n_seq, self.n_draft, self.vocab = n_seq, n_draft, vocab

    def dev(self, t):
        return None if t is None else (t if isinstance(t, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(t))).to(DEV)

    def call(self, target=None, draft=None, ws=None, stream=None, n_draft=None):
        n = self.n_draft
        tokens = torch.full((self.n_seq, n + 1), -7, dtype=torch.int32, device=DEV)
        accepted = torch.full((self.n_seq,), -7, dtype=torch.int32, device=DEV)
        ws = torch.full((binding.octopus_verify_workspace(self.n_seq, n, self.vocab),), 0xFF, dtype=torch.uint8, device=DEV) if ws is None else ws
        binding.octopus_verify_drafts(self.dev(self.target) if target is None else target, self.dev(self.draft) if draft is None else draft,
                                      self.dev(self.x) if n else None, self.dev(self.u), tokens, accepted, ws, draft_lens=self.dev(self.lens), stream=stream)
        torch.cuda.synchronize()
        return tokens.cpu().numpy(), accepted.cpu().numpy()

    def expected(self):
        rows = []
        for s in range(self.n_seq):
            n = self.n_draft if self.lens is None else int(min(max(self.lens[s], 0), self.n_draft))
            rows.append(verify(self.target[s].float().numpy(), None if self.draft is None else self.draft[s].float().numpy(), self.x[s, :n],
                               self.u[s], self.n_draft))
        return np.array([r[0] for r in rows]), np.array([r[1] for r in rows])

    def check(self, **more):
        (tokens, accepted), (want, count) = self.call(**more), self.expected()
        assert np.array_equal(accepted, count), (accepted, count)
        assert np.array_equal(tokens, want), (tokens, want)
        return count


@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 4097, 32000, 50257, 65536, 65537, 128256, 262143, 262144,
                                   300001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("sampled", [True, False])
def test_vocabularies(vocab, dtype, sampled):
    Batch(3, 2, vocab, dtype, sampled, seed=1).check()


@pytest.mark.parametrize("n_seq,n_draft", [(1, 0), (5, 0), (1, 1), (40, 4), (300, 3), (2, 63), (2, 64), (3, 65), (1, 200)])
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("agree", [0.0, 0.9, 1.0])
def test_numbers_of_drafts(n_seq, n_draft, sampled, agree):
    """Drafters that never, often and always agree (drafts of the target's own distribution all stand)."""
    x = Batch(n_seq, n_draft, 130, sampled=sampled, agree=agree, ragged=n_draft > 1)
    count = x.check()
    if agree == 1.0 and sampled:
        assert np.array_equal(count, np.full(n_seq, n_draft) if x.lens is None else x.lens)


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_many_drafts_of_long_rows(sampled, dtype):
    """Rows of two launches: padded batches, drafts past the 64 that a wavefront looks at."""
    Batch(20, 5, 66000, dtype, sampled, ragged=True, agree=0.9, seed=21).check()
    x = Batch(1, 70, 66000, dtype, True, agree=1.0, seed=22)
    x.draft = x.draft if sampled else None
    x.target[0, 66, x.x[0, 66]] = 0.0
    assert x.check().tolist() == [66] or not sampled


@pytest.mark.parametrize("where", [0, 1, 62, 63, 64, 127, 128, 199])
def test_the_first_draft_that_falls_counts(where):
    """Drafts that all stand but for one, and one behind it: before, at and after the 64 that a wavefront looks at."""
    x = Batch(2, 200, 20, agree=1.0)
    x.target[0, where, x.x[0, where]] = 0.0
    x.target[0, 199, x.x[0, 199]] = 0.0
    assert x.check().tolist() == [where, 200]


@pytest.mark.parametrize("sampled", [True, False])
def test_borders_exactly(sampled):
    """Dyadic rows: u q = p does not stand, and a running sum that equals the goal is not past it."""
    p = [0.25, 0.0, 0.125, 0.125, 0.5]
    q = [0.5, 0.25, 0.125, 0.125, 0.0]
    n = 32
    x = Batch(n * 5, 1, 5, sampled=sampled)
    x.target[:] = torch.tensor(p)
    if sampled:
        x.draft[:] = torch.tensor(q)
    x.x = np.repeat(np.arange(5, dtype=np.int32), n)[:, None]
    x.u = np.stack([np.tile(np.arange(n), 5) / n, np.tile(np.arange(n)[::-1], 5) / n], axis=1).astype(np.float32)
    x.check()
    half = np.nextafter(np.float32(0.5), np.float32(0))
    x.u[:n, 0], x.u[n - 1, 0] = 0.5, half
    count = x.check()[:n].tolist()
    assert count == [0] * (n - 1) + [1] or not sampled


@pytest.mark.parametrize("vocab", [5, 1024, 5000, 70000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_random_numbers_at_their_ends(vocab, dtype):
    """0, the largest below 1, and what is none: 1, above, below, infinities, NaN; a token without weight is never drawn."""
    u = [0.0, 1 - 2 ** -24, 1.0, 3.0, -1.0, np.inf, -np.inf, np.nan, 1e-38, 1e-45]
    x = Batch(len(u), 2, vocab, dtype, zeros=0.5, seed=3)
    x.target[:, :, 0] = 0.0
    x.target[:, :, -1] = 0.0
    x.target[:, :, 1] += 0.01
    x.u[:] = np.array(u, dtype=np.float32)[:, None]
    x.check()
    tokens, accepted = x.call()
    last = tokens[np.arange(len(u)), accepted]
    assert np.all(x.target.float().numpy()[np.arange(len(u)), accepted, last] > 0)


@pytest.mark.parametrize("n_seq,vocab", [(64, 700), (4, 66001)])
def test_numbers_that_are_no_probabilities_count_as_zero(n_seq, vocab):
    x = Batch(n_seq, 2, vocab, seed=5)
    rng = np.random.default_rng(0)
    for t in (x.target, x.draft):
        at = torch.from_numpy(rng.random(t.shape) < 0.3)
        t[at] = torch.from_numpy(rng.choice([np.nan, np.inf, -np.inf, -0.5, -0.0, 1e-42], size=int(at.sum())).astype(np.float32))
    x.check()


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("vocab", [2000, 80000])
def test_rows_with_nothing_left(sampled, vocab):
    """A draft that falls though the target is nowhere above the drafter: the token is the target's; an empty row has none."""
    x = Batch(6, 1, vocab, sampled=sampled, seed=6)
    x.target[:, 0] = 0.0
    x.target[0, 0, 77] = 0.25
    x.target[1, 0, 5], x.target[1, 0, vocab - 1] = 0.25, 0.25
    if sampled:
        x.draft[:] = 0.25
        x.x[:2] = [[3], [3]]
    else:
        x.x[:2] = [[77], [5]]
    x.u[:, 0] = 0.5
    x.u[1, 1] = 0.75
    x.check()
    tokens, accepted = x.call()
    assert tokens[0, 0] == 77 and tokens[1, 0] == vocab - 1 and accepted.tolist() == [0] * 6 and np.all(tokens[2:] == -1)


def test_drafts_outside_the_vocabulary_and_counts_out_of_range():
    x = Batch(8, 3, 100, agree=1.0, seed=7)
    x.x[0, 1], x.x[1, 0], x.x[2, 2] = -1, 100, 2 ** 31 - 1
    x.x[3, 0] = -2 ** 31
    x.lens = np.array([3, 3, 3, 3, -4, 99, 0, 2 ** 31 - 1], dtype=np.int32)
    assert x.check().tolist() == [1, 0, 2, 0, 0, 3, 0, 3]
    x.draft = None
    x.check()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 2, 3, 5, 8])
def test_strides_and_alignment(dtype, offset):
    """Rows between other data, at any element: what lies around them has no say; a target that all sequences share."""
    n_seq, n, vocab = 5, 3, 1531
    x = Batch(n_seq, n, vocab, dtype, seed=offset)
    wide = torch.full((n_seq, n + 3, vocab + 29), 1e30, dtype=TYPES[dtype], device=DEV)
    target = wide[:, 1:n + 2, offset:offset + vocab]
    target.copy_(x.target)
    wide = torch.full((n, n_seq, vocab + 17), 1e30, dtype=TYPES[dtype], device=DEV)
    draft = wide[:, :, offset:offset + vocab].transpose(0, 1)
    draft.copy_(x.draft)
    x.check(target=target, draft=draft)
    x.target[:] = x.target[:1].clone()
    x.check(target=x.target[:1].to(DEV).expand(n_seq, -1, -1))


def test_rows_behind_the_last_draft_are_not_looked_at():
    x = Batch(9, 4, 500, ragged=True, seed=8)
    x.lens[0], x.lens[1] = 0, 4
    want = x.call()
    for s, n in enumerate(x.lens):
        x.target[s, n + 1:] = float("nan")
        x.draft[s, n:] = float("nan")
        x.x[s, n:] = -9
    got = x.call()
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    x.check()


def test_targets_of_more_than_4_gib():
    """Offsets past 32 bits, in elements and in bytes."""
    n_seq, vocab = 36, 1 << 26
    target = torch.zeros((n_seq, 1, vocab), dtype=torch.bfloat16, device=DEV)
    at = torch.arange(n_seq, device=DEV) * 1000003 % vocab
    target[torch.arange(n_seq, device=DEV), 0, at] = 0.5
    target[:, 0, vocab - 1] = 0.25
    u = torch.where(torch.arange(n_seq, device=DEV) % 3 == 0, 0.75, 0.5)[:, None].contiguous()
    tokens, accepted = torch.zeros((n_seq, 1), dtype=torch.int32, device=DEV), torch.zeros(n_seq, dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.octopus_verify_workspace(n_seq, 0, vocab), dtype=torch.uint8, device=DEV)
    binding.octopus_verify_drafts(target, None, None, u, tokens, accepted, ws)
    want = torch.where(torch.arange(n_seq, device=DEV) % 3 == 0, vocab - 1, at)
    assert torch.equal(tokens[:, 0].long(), want) and not accepted.any()


def test_tokens_come_out_as_the_targets():
    """60000 sequences of one draft: the first token's counts against the target's distribution, whatever the drafter's; chi-square of 6
    degrees of freedom below its 1 - 1e-5 quantile."""
    rng = np.random.default_rng(11)
    n, vocab = 60000, 7
    p, q = np.float32(rng.dirichlet(np.ones(vocab))), np.float32(rng.dirichlet(np.ones(vocab)))
    for sampled in (True, False):
        x = rng.choice(vocab, size=(n, 1), p=(q / q.sum(dtype=np.float64)).astype(np.float64) / (q / q.sum(dtype=np.float64)).sum()).astype(np.int32)
        u = torch.from_numpy(rng.random((n, 2), dtype=np.float32)).to(DEV)
        tokens, accepted = torch.zeros((n, 2), dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
        ws = torch.empty(binding.octopus_verify_workspace(n, 1, vocab), dtype=torch.uint8, device=DEV)
        target = torch.from_numpy(p).to(DEV).expand(n, 2, vocab)
        draft = torch.from_numpy(q).to(DEV).expand(n, 1, vocab) if sampled else None
        binding.octopus_verify_drafts(target, draft, torch.from_numpy(x).to(DEV), u, tokens, accepted, ws)
        count = np.bincount(tokens[:, 0].cpu().numpy(), minlength=vocab)
        want = n * p / p.sum(dtype=np.float64)
        assert ((count - want) ** 2 / want).sum() < 33.2
        assert 0 < int(accepted.sum()) < n


@pytest.mark.parametrize("vocab", [5000, 66000])
def test_another_stream_and_a_captured_call(vocab):
    x, y = Batch(4, 3, vocab, seed=12), Batch(4, 3, vocab, seed=13)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    want = [b.expected() for b in (x, y)]
    got = x.call(stream=side)
    assert np.array_equal(got[0], want[0][0])
    target, draft, drafts, u = (x.dev(t).clone() for t in (x.target, x.draft, x.x, x.u))
    tokens, accepted = torch.zeros((4, 4), dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    ws = torch.zeros(binding.octopus_verify_workspace(4, 3, vocab), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.octopus_verify_drafts(target, draft, drafts, u, tokens, accepted, ws)
    for replay in range(6):
        b, (t, a) = (x, y)[replay % 2], want[replay % 2]
        for dst, src in ((target, b.target), (draft, b.draft), (drafts, b.x), (u, b.u)):
            dst.copy_(b.dev(src))
        y.call(ws=ws)                        # eager work between, with the same workspace
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(tokens.cpu().numpy(), t) and np.array_equal(accepted.cpu().numpy(), a)

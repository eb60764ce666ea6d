"""GPU tests of octopus_append_paged_axes.

A token's rotation by positions on several axes is one by a row of (cos, sin) pairs of its own: the pairs gathered from the table by
each pair's axis.  So the call is compared, byte for byte, with octopus_append_paged over a table that holds those rows, a position a token; what
that call computes is compared with the oracle's records and with 64 bits here once more, through the helpers of its own tests."""
import numpy as np
import pytest

from paper_2605_21226_amd import binding

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from gpu_util import DEV  # noqa: E402
from test_gpu_append import FILL, Setup, ints, rope_table  # noqa: E402

N_POS = 900


def axis_map(pairs, n_axes, kind, seed=0):
    if kind == "runs":
        return np.minimum(np.arange(pairs) * n_axes // pairs, n_axes - 1).astype(np.uint8)
    if kind == "turns":
        return (np.arange(pairs) % n_axes).astype(np.uint8)
    return np.random.default_rng(seed).integers(0, n_axes, size=pairs).astype(np.uint8)


def gathered(table, axis, pos):
    """Rows of (cos, sin) of tokens at pos [..., n_axes] (positions outside the table read as the nearest inside)."""
    p = np.clip(pos, 0, len(table) - 1)
    return np.stack([table[p[..., a], i] for i, a in enumerate(axis)], axis=-2)


class Axes(Setup):
    def __init__(self, *args, n_axes=3, kind="runs", pos=None, rot=None, seed=0, **more):
        super().__init__(*args, rot=rot, seed=seed, **more)
        rng = np.random.default_rng(1000 + seed)
        self.of_axes = rope_table(N_POS, self.d if rot is None else rot)
        self.axis = axis_map(self.of_axes.shape[1], n_axes, kind, seed)
        self.pos = rng.integers(0, N_POS, size=(self.n_seq, self.n_new, n_axes)).astype(np.int32) if pos is None else pos
        self.pos_dev = ints(self.pos)
        # the same as one table with a row a token
        self.table = gathered(self.of_axes, self.axis, self.pos).reshape(self.n_seq * self.n_new, -1, 2)
        self.rope = torch.from_numpy(np.ascontiguousarray(self.table)).to(DEV)
        self.rope_pos = np.arange(self.n_seq) * self.n_new

    def append_axes(self, pos=None, part=slice(None), **more):
        v_pool = self.v_pool if self.v_bits else self.v_pool.view(torch.bfloat16)
        args = dict(start_pos=self.start_dev, new_lens=self.lens_dev, rope_interleaved=self.interleaved, q=self.q_dev, q_out=self.q_out,
                    v_bits=self.v_bits, v_group=self.v_group)
        args.update(more)
        binding.octopus_append_paged_axes(self.cb, self.k_dev[:, part], self.v_dev[:, part], self.signs_dev, self.k_pool, v_pool, self.n_pages,
                                          self.block_dev, torch.from_numpy(self.of_axes).to(DEV), self.axis.tobytes(),
                                          self.pos_dev if pos is None else pos, **args)
        torch.cuda.synchronize()

    def taken(self):
        """What the calls wrote, and everything as it was before."""
        got = [x.clone() for x in (self.k_pool, self.v_pool) + (() if self.q_out is None else (self.q_out,))]
        self.k_pool.fill_(FILL)
        self.v_pool.fill_(FILL)
        if self.q_out is not None:
            self.q_out.fill_(7.0)
        return got

    def compare(self, **more):
        self.append_axes(**more)
        got = self.taken()
        self.append()
        for x, y in zip(got, (self.k_pool, self.v_pool, self.q_out)):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("bits", [1, 1.5, 2, 2.5, 3, 4])
@pytest.mark.parametrize("n_new", [1, 700])
def test_every_plan(d, bits, n_new):
    """One token a sequence and prompts (which have kernels of their own), ragged starts, all channels, a run of pairs an axis."""
    x = Axes(d, bits, 2, 2, 2, n_new, [5, 77], seed=int(10 * bits))
    x.append_axes()
    x.check()
    x.compare()


@pytest.mark.parametrize("kind", ["runs", "turns", "random"])
@pytest.mark.parametrize("n_axes", [1, 2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot,n_new,dtype", [(64, 32, 3, "fp32"), (128, 128, 130, "bf16"), (128, 48, 1, "bf16"), (256, 256, 65, "fp32"),
                                               (256, 16, 300, "bf16")])
def test_maps_and_widths(kind, n_axes, interleaved, d, rot, n_new, dtype):
    Axes(d, 3, 3, 1, 3, n_new, [0, 64, 31], n_axes=n_axes, kind=kind, rot=rot, interleaved=interleaved, dtype=dtype, seed=n_axes).compare()


@pytest.mark.parametrize("n_new", [1, 400])
def test_one_position_on_all_axes_is_the_call_of_one_axis(n_new):
    """Text between images: every byte that of octopus_append_paged at that position."""
    start = [3, 130, 64]
    at = np.repeat((np.asarray(start)[:, None] + np.arange(n_new))[..., None], 3, axis=2).astype(np.int32)
    x = Axes(128, 3, 3, 2, 4, n_new, start, pos=at)
    x.append_axes()
    got = x.taken()
    x.append(rope=torch.from_numpy(x.of_axes).to(DEV), rope_pos=None)
    for a, b in zip(got, (x.k_pool, x.v_pool, x.q_out)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("n_new", [1, 250])
@pytest.mark.parametrize("layout", ["axis first", "gaps", "no token stride", "no sequence stride", "no axis stride"])
def test_strides_of_positions(n_new, layout):
    rng = np.random.default_rng(3)
    n_seq, n_axes = 4, 3
    pos = rng.integers(0, N_POS, size=(n_seq, n_new, n_axes)).astype(np.int32)
    if layout == "axis first":
        dev = ints(pos.transpose(2, 0, 1)).permute(1, 2, 0)
    elif layout == "gaps":
        room = torch.full((n_seq, n_new, 2, 7), -9, dtype=torch.int32, device=DEV)
        room[:, :, 1, :2 * n_axes:2] = ints(pos)
        dev = room[:, :, 1, :2 * n_axes:2]
    else:
        axis = ("no sequence stride", "no token stride", "no axis stride").index(layout)
        pos = np.broadcast_to(pos.take([0], axis=axis), pos.shape)
        dev = ints(pos.take([0], axis=axis)).expand(*pos.shape)
        assert dev.stride()[axis] == 0 or pos.shape[axis] == 1
    x = Axes(128, 2, n_seq, 2, 2, n_new, [0, 1, 63, 64], pos=np.ascontiguousarray(pos))
    x.compare(pos=dev)


@pytest.mark.parametrize("n_new,new_lens", [(1, [1, 0, 1, -5]), (70, [70, 0, 3, 64]), (200, [500, 1, 0, 199])])
def test_padded_batches_look_at_no_position_behind_the_counted_tokens(n_new, new_lens):
    """Positions of tokens that do not count may not be there at all: the last sequence's lie at the very end of the array, which holds as many as count."""
    x = Axes(128, 3, 4, 2, 2, n_new, [0, 5, 63, 10], new_lens=new_lens)
    x.append_axes()
    x.check()
    x.compare()
    count = [max(0, min(n, n_new)) for n in new_lens]
    junk = x.pos_dev.clone()
    for s, n in enumerate(count):
        junk[s, n:] = torch.iinfo(torch.int32).min
    x.compare(pos=junk)


@pytest.mark.parametrize("n_new", [1, 90])
def test_positions_outside_the_table_are_read_as_the_nearest_inside(n_new):
    pos = np.random.default_rng(9).choice([-2 ** 31, -1, 0, N_POS - 1, N_POS, 2 ** 31 - 1], size=(3, n_new, 4)).astype(np.int32)
    Axes(64, 3, 3, 2, 1, n_new, [0, 9, 64], n_axes=4, kind="turns", pos=pos).compare()


@pytest.mark.parametrize("v_bits,v_group", [(2, 16), (3, 32), (4, 16)])
@pytest.mark.parametrize("n_new", [1, 77])
def test_quantised_values(v_bits, v_group, n_new):
    Axes(128, 3, 2, 3, 1, n_new, [61, 0], v_bits=v_bits, v_group=v_group).compare()


def test_tokens_past_the_table_and_calls_without_queries():
    Axes(128, 3, 2, 2, 1, 200, [100, 0], pages=3).compare()
    x = Axes(128, 3, 2, 2, 1, 70, [100, 0], with_q=False)
    x.append_axes()
    got = x.taken()
    x.append()
    assert torch.equal(got[0], x.k_pool) and torch.equal(got[1], x.v_pool)


def test_a_prompt_at_once_and_token_by_token():
    x = Axes(128, 3, 2, 2, 2, 96, [40, 0], kind="turns")
    x.append_axes()
    k, v, q = x.taken()
    for t in range(96):
        part = slice(t, t + 1)
        q_out = torch.zeros_like(x.q_out[:, part])
        x.append_axes(pos=x.pos_dev[:, part], part=part, start_pos=x.start_dev + t, q=x.q_dev[:, part], q_out=q_out)
        assert torch.equal(q_out, q[:, part])
    assert torch.equal(x.k_pool, k) and torch.equal(x.v_pool, v)


@pytest.mark.parametrize("n_new", [1, 130])
def test_queries_in_place(n_new):
    x = Axes(128, 3, 2, 2, 4, n_new, [0, 7])
    x.append_axes()
    q = x.q_dev.contiguous()
    x.append_axes(q=q, q_out=q)
    assert torch.equal(q, x.q_out)


@pytest.mark.parametrize("n_new", [1, 70])
def test_positions_far_apart(n_new):
    """Axes 2^30 numbers apart, sequences 2^29: offsets past 32 bits, in elements and in bytes."""
    far = torch.empty(2 ** 31 + 2 ** 29 + 1000, dtype=torch.int32, device=DEV)
    x = Axes(64, 3, 2, 1, 2, n_new, [0, 30])
    pos = far.as_strided((2, n_new, 3), (2 ** 29, 1, 2 ** 30))
    pos.copy_(x.pos_dev)
    x.compare(pos=pos)


def test_another_stream():
    x = Axes(128, 3, 2, 2, 2, 300, [7, 0])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    x.append_axes(stream=side)
    got = x.taken()
    x.append()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, (x.k_pool, x.v_pool, x.q_out)))

"""Host-side checks, without a GPU, of octopus_append_paged_axes: what it refuses, and what the Python entry point refuses before the
library is asked."""
import ctypes

import pytest

from paper_2605_21226_amd import binding
from test_serve_host import APPEND, EINVAL, EUNSUPPORTED, FAKE, OFF4, OFF8, OK, books, broken_books, lib, refuses, unbuilt_books  # noqa: F401

AXES = bytes(i % 3 for i in range(64))


def rope(**changes):
    f = {**dict(table=FAKE, n_pos=100, pos=OFF4, stride_seq=24, stride_tok=3, stride_axis=1, axis=AXES, n_axes=3, dim=128, interleaved=0), **changes}
    return ctypes.byref(binding.RopeAxes(*[f[n] for n, _ in binding.RopeAxes._fields_]))


def test_refusals(lib):  # noqa: F811
    cb, P = books()
    broken, unbuilt = broken_books(), unbuilt_books()
    good = dict(cb=P, k=FAKE, ks=8192, kt=1024, kh=128, v=FAKE, vs=8192, vt=1024, vh=128, kv_dtype=1, n_seq=2, n_kv=8, n_new=0, new_lens=None,
                rope=rope(), q=FAKE, q_dtype=1, qs=8192, qt=1024, qh=128, n_qh=32, q_out=FAKE, q_out_dtype=1, signs=FAKE, k_pool=FAKE,
                v_pool=FAKE, v_bits=0, v_group=0, n_pages=10, block_table=FAKE, max_pages=4, start_pos=FAKE, stream=None)
    late = AXES[:-1] + bytes([3])
    refuses(lib.octopus_append_paged_axes, APPEND, good, [
        ({}, OK), ({"rope": None}, EINVAL),
        *[({"rope": rope(**k)}, EINVAL) for k in (
            dict(table=None), dict(table=OFF8), dict(n_pos=0), dict(n_pos=-5), dict(n_pos=2 ** 23 + 1), dict(dim=16, n_pos=2 ** 24 + 1), dict(n_pos=2 ** 62), dict(pos=FAKE + 2), dict(dim=0), dict(dim=8),
            dict(dim=24), dict(dim=144), dict(dim=-16), dict(interleaved=2), dict(interleaved=-1), dict(n_axes=0), dict(n_axes=-1), dict(n_axes=5), dict(n_axes=2),
            dict(axis=None), dict(axis=late), dict(stride_seq=-1), dict(stride_tok=-1), dict(stride_tok=2 ** 31), dict(stride_axis=-1))],
        # (pairs past dim / 2 have no axis: nothing there is looked at)
        *[({"rope": rope(**k)}, OK) for k in (dict(axis=late, dim=112), dict(axis=late, n_axes=4), dict(stride_seq=0, stride_tok=0, stride_axis=0),
                                              dict(interleaved=1), dict(pos=None), dict(n_pos=2 ** 23), dict(dim=16, n_pos=2 ** 24), dict(stride_tok=2 ** 31 - 1), dict(dim=16, axis=bytes(8), n_axes=1))],
        *[({name: None}, EINVAL) for name in ("cb", "signs", "k_pool", "v_pool", "block_table", "q_out")],
        *[({name: n}, EINVAL) for name in ("n_seq", "n_kv", "n_pages", "max_pages", "n_qh") for n in (0, -1)],
        ({"n_new": 1, "rope": rope(pos=None)}, EINVAL), ({"k": None, "v": None, "q": None, "rope": rope(pos=None)}, OK),     # (an empty tensor may have no address)
        ({"n_new": -1}, EINVAL), ({"n_qh": 30}, EINVAL), ({"kt": 4}, EINVAL), ({"kv_dtype": 2}, EUNSUPPORTED),
        ({"cb": ctypes.byref(broken)}, EINVAL), ({"cb": ctypes.byref(unbuilt)}, EUNSUPPORTED)])


def test_struct(lib):  # noqa: F811
    assert ctypes.sizeof(binding.RopeAxes) == 8 * 7 + 4 * 3 + 4


def test_what_the_python_call_refuses(monkeypatch):
    torch = pytest.importorskip("torch")
    cb = binding.octopus_build_codebooks(128, 3)

    class Reached(Exception):
        pass

    class Library:
        def octopus_append_paged_axes(self, *_):
            raise Reached
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    n_seq, n_new, n_kv, d = 2, 3, 2, 128
    kv = torch.zeros((n_seq, n_new, n_kv, d), dtype=torch.bfloat16)
    pools = (torch.zeros(4 * n_kv * 64 * 16 * cb.plan.granules, dtype=torch.uint8), torch.zeros((4, n_kv, 64, d), dtype=torch.bfloat16))
    table, turn = torch.zeros((n_seq, 1), dtype=torch.int32), torch.zeros((50, 64, 2))
    pos = torch.zeros((n_seq, n_new, 3), dtype=torch.int32)

    def call(k=kv, v=kv, rope=turn, axis=AXES, pos=pos, **more):
        binding.octopus_append_paged_axes(cb, k, v, torch.zeros((n_kv, d // 8), dtype=torch.uint8), *pools, 4, table, rope, axis, pos, **more)
    for good in (dict(), dict(axis=list(AXES)), dict(pos=pos.permute(2, 0, 1).contiguous().permute(1, 2, 0)), dict(rope=turn[:, :8].contiguous(), axis=AXES[:8]),
                 dict(q=kv, q_out=torch.zeros_like(kv))):
        with pytest.raises(Reached):
            call(**good)
    for bad in (dict(axis=AXES[:-1]), dict(axis=AXES + b"\0"), dict(pos=pos[:1]), dict(pos=pos[:, :2]), dict(pos=pos.long()), dict(pos=pos.float()),
                dict(rope=turn[:, :32]), dict(rope=turn.double()), dict(k=kv[:1], v=kv[:1]), dict(v=kv.float()), dict(q=kv, q_out=torch.zeros_like(kv)[:, :1])):
        with pytest.raises((AssertionError, TypeError)):
            call(**bad)

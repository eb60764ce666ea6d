"""Without a GPU: what the entry points on the pages themselves refuse, their workspace, and the sequential model that their GPU tests go by."""
import ctypes

import numpy as np
import pytest

from paper_2605_21226_amd import binding
from pages_model import Pages
from test_serve_host import EINVAL, EWORKSPACE, FAKE, OFF4, OFF8, OK, lib, refuses  # noqa: F401

UPDATE = "refs n_pages table max_pages lens n_seq source keep_lens new_lens moves ws ws_bytes stream"
COMPACT = "refs n_pages page_map moves ws ws_bytes stream"
RENAME = "page_map n_pages table n_rows max_pages lens stream"
COPY = "pools n_pools n_pages moves max_moves stream"


def test_workspace(lib):  # noqa: F811
    size = lib.octopus_pages_workspace
    assert size(100, 4, 10) > 0 and size(100, 4, 10) % 256 == 0
    for bad in ((0, 4, 10), (100, 0, 10), (100, 4, 0), (-1, 4, 10), ((1 << 24) + 1, 4, 10), (100, 65536, 10), (100, 4, 2 ** 26), (100, 65535, 16385)):
        assert size(*bad) == 0
    assert size(1 << 24, 65535, 16384) > 4 * 65535 * 16384
    for n in ((1, 1, 1), (5000, 3, 70), (9, 1000, 2)):
        for i in range(3):
            more = list(n)
            more[i] += 1
            assert size(*more) >= size(*n)


def test_update_refusals(lib):  # noqa: F811
    need = lib.octopus_pages_workspace(100, 4, 10)
    good = dict(refs=FAKE, n_pages=100, table=FAKE, max_pages=10, lens=FAKE, n_seq=4, source=None, keep_lens=None, new_lens=FAKE, moves=FAKE, ws=FAKE,
                ws_bytes=need - 1, stream=None)
    refuses(lib.octopus_pages_update, UPDATE, good, [
        ({}, EWORKSPACE), ({"ws": None, "ws_bytes": need}, EWORKSPACE), ({"ws": FAKE + 128, "ws_bytes": need}, EWORKSPACE),
        ({"source": FAKE, "keep_lens": OFF4, "lens": OFF4}, EWORKSPACE),
        *[({name: None}, EINVAL) for name in ("refs", "table", "lens", "new_lens", "moves")],
        *[({name: n}, EINVAL) for name in ("n_pages", "max_pages", "n_seq") for n in (0, -1)],
        ({"n_pages": (1 << 24) + 1}, EINVAL), ({"n_seq": 65536}, EINVAL), ({"max_pages": 2 ** 26}, EINVAL), ({"n_seq": 65535, "max_pages": 16385}, EINVAL),
        ({"refs": OFF8}, EINVAL), *[({name: FAKE + 2}, EINVAL) for name in ("table", "lens", "source", "keep_lens", "new_lens", "moves")]])


def test_compact_and_rename_refusals(lib):  # noqa: F811
    need = lib.octopus_pages_workspace(100, 1, 1)
    good = dict(refs=FAKE, n_pages=100, page_map=FAKE, moves=FAKE, ws=FAKE, ws_bytes=need - 1, stream=None)
    refuses(lib.octopus_pages_compact, COMPACT, good, [
        ({}, EWORKSPACE), ({"ws": None}, EWORKSPACE), ({"ws": FAKE + 64, "ws_bytes": need}, EWORKSPACE),
        *[({name: None}, EINVAL) for name in ("refs", "page_map", "moves")], *[({"n_pages": n}, EINVAL) for n in (0, -1, (1 << 24) + 1)],
        ({"refs": OFF8}, EINVAL), ({"page_map": FAKE + 2}, EINVAL), ({"moves": FAKE + 1}, EINVAL)])
    good = dict(page_map=FAKE, n_pages=100, table=FAKE, n_rows=0, max_pages=10, lens=None, stream=None)
    refuses(lib.octopus_pages_rename, RENAME, good, [
        ({}, EINVAL), *[({"n_rows": 1, **bad}, EINVAL) for bad in (
            {"page_map": None}, {"table": None}, {"n_pages": 0}, {"n_pages": (1 << 24) + 1}, {"max_pages": 0}, {"n_rows": 65536}, {"max_pages": 2 ** 26},
            {"page_map": FAKE + 2}, {"table": FAKE + 2}, {"lens": FAKE + 2}, {"n_rows": 65535, "max_pages": 16385})]])


def test_copy_refusals(lib):  # noqa: F811
    def pools(*each):
        return (binding.Pool * len(each))(*[binding.Pool(*p) for p in each])
    fine = (FAKE, 4096)
    good = dict(pools=pools(fine), n_pools=1, n_pages=100, moves=FAKE, max_moves=0, stream=None)
    refuses(lib.octopus_pages_copy, COPY, good, [
        ({}, OK), ({"pools": pools(*[fine] * 200), "n_pools": 200}, OK), ({"pools": None}, EINVAL), ({"moves": None}, EINVAL), ({"moves": FAKE + 2}, EINVAL),
        *[({"n_pools": n}, EINVAL) for n in (0, -1)], *[({"n_pages": n}, EINVAL) for n in (0, -1, (1 << 24) + 1)], ({"max_moves": -1}, EINVAL),
        *[({"pools": pools(fine, p), "n_pools": 2}, EINVAL) for p in ((None, 4096), (OFF8, 4096), (FAKE, 0), (FAKE, -16), (FAKE, 8), (FAKE, 4104),
                                                                    (FAKE, 1 << 40))]])
    assert ctypes.sizeof(binding.Pool) == 16


def test_what_the_python_calls_refuse(monkeypatch):
    torch = pytest.importorskip("torch")

    class Reached(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            def f(*_):
                raise Reached
            return f
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    ws = torch.zeros(64, dtype=torch.uint8)
    update = dict(refs=ints(50), block_table=ints(3, 5), lens=ints(3), new_lens=ints(3), moves=ints(8), workspace=ws, source=ints(3), keep_lens=ints(3))
    compact = dict(refs=ints(9), page_map=ints(9), moves=ints(10), workspace=ws)
    rename = dict(page_map=ints(9), table=ints(3, 5), lens=ints(3))
    a, b = torch.zeros((10, 4, 16), dtype=torch.uint8), torch.zeros((10, 8), dtype=torch.bfloat16)
    copy = dict(pools=binding.page_pools([a, b]), moves=ints(12), max_moves=5)
    assert [(p.page_bytes) for p in copy["pools"].array] == [64, 16] and binding.page_pools([a.view(-1)], 10).n_pages == 10
    for f, good, bads in (
            (binding.octopus_pages_update, update,
             [{"lens": ints(2)}, {"new_lens": ints(2)}, {"source": ints(2)}, {"keep_lens": ints(2)}, {"moves": ints(7)}, {"refs": ints(50).long()},
              {"refs": ints(100)[::2]}, {"block_table": ints(5, 3).t()}, {"block_table": ints(3, 5).long()}, {"new_lens": torch.zeros(3)}, {"lens": ints(3).long()}]),
            (binding.octopus_pages_compact, compact, [{"page_map": ints(8)}, {"moves": ints(9)}, {"refs": ints(9).long()}, {"page_map": ints(18)[::2]}]),
            (binding.octopus_pages_rename, rename, [{"lens": ints(2)}, {"table": ints(5, 3).t()}, {"page_map": torch.zeros(9)}, {"table": ints(3, 5).long()}]),
            (binding.octopus_pages_copy, copy, [{"moves": ints(11)}, {"moves": ints(24)[::2]}, {"moves": ints(12).long()}])):
        with pytest.raises(Reached):
            f(**good)
        for bad in bads:
            with pytest.raises(AssertionError):
                f(**{**good, **bad})
    for bad in ([a, b[:5]], [a[::2]], [a.transpose(0, 1)]):
        with pytest.raises(AssertionError):
            binding.page_pools(bad)
    with pytest.raises(AssertionError):
        binding.page_pools([a.view(-1)], 7)


def test_model():
    """The model itself, on a case that can be followed by hand."""
    x = Pages([1, 1, 1, 0, 0, 0], [[0, 1, 9], [2, 9, 9], [9, 9, 9]], [100, 64, 0])
    x.update([101, 65, 101], source=[0, 1, 0])
    # slot 0 keeps pages 0 and 1 and writes into 1; slot 1 gets the first free page, 3 after none was copied; slot 2 shares 0, copies 1 to 4
    assert x.table.tolist() == [[0, 1, 9], [2, 3, 9], [0, 4, 9]] and x.refs.tolist() == [2, 1, 1, 1, 1, 0] and x.moves == [(1, 4)]
    x.check()
    x.update([101, 0, 101])
    assert x.compact() == [0, 1, 2, 3, 2, 5] and x.moves == [(4, 2)]
    x.rename([0, 1, 2, 3, 2, 5])
    assert x.table[2].tolist() == [0, 2, 9]
    x.check()
    x.update([1000, 0, 101])
    assert x.missing == 0 or x.lens.tolist() == [101, 0, 101]
    assert np.array_equal(x.lens, [192, 0, 101])

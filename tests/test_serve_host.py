"""Host-side checks, without a GPU, of the entry points over pages that surround the attention of a server's step: argument errors are
reported before anything is launched, empty calls do nothing, and the division of a shared-prefix call covers it."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_21226_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = next((c for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")) if c and os.path.exists(c)), None)
FAKE = 0x1000          # never dereferenced: the calls below end before a launch
OFF4, OFF8 = FAKE + 4, FAKE + 8


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_21226_amd import build
        build.build(verbose=False)
    return binding.load()


PREFIX = ("cb q q_dtype n_seq n_qh n_kv n_q q_lens causal signs k_pool v_pool n_pages prefix_table prefix_pages prefix_len max_prefix "
          "block_table max_pages seq_lens max_len scale out ws ws_bytes stream")
APPEND = ("cb k ks kt kh v vs vt vh kv_dtype n_seq n_kv n_new new_lens rope q q_dtype qs qt qh n_qh q_out q_out_dtype signs k_pool v_pool "
          "v_bits v_group n_pages block_table max_pages start_pos stream")
READ = ("cb signs k_pool v_pool v_bits v_group n_pages block_table max_pages n_seq n_kv start_pos n_tok lens k_out v_out out_dtype stream")


def refuses(f, order, good, bad):
    """Each (changes, code): the call that is good but for the changes returns the code."""
    for changes, code in bad:
        assert set(changes) <= set(good), changes
        values = {**good, **changes}
        assert f(*[values[name] for name in order.split()]) == code, changes


def books(d=128, bits=3):
    cb = binding.octopus_build_codebooks(d, bits)
    return cb, ctypes.byref(cb)


def broken_books():
    cb = binding.octopus_build_codebooks(128, 3)
    cb.plan.record_bytes = 57
    return cb


def unbuilt_books():
    return binding.octopus_build_codebooks_pair(64, 3, 3)


EINVAL, EUNSUPPORTED, EWORKSPACE, OK = binding.EINVAL, binding.EUNSUPPORTED, binding.EWORKSPACE, binding.OK


def test_prefix_attention_refusals(lib):
    cb, P = books()
    broken, unbuilt = broken_books(), unbuilt_books()
    size = binding.octopus_attn_prefix_workspace(cb, 3, 32, 8, 2, 4096, 1024)
    assert size > 0 and size % 256 == 0
    good = dict(cb=P, q=FAKE, q_dtype=1, n_seq=3, n_qh=32, n_kv=8, n_q=2, q_lens=None, causal=0, signs=FAKE, k_pool=FAKE, v_pool=FAKE,
                n_pages=100, prefix_table=FAKE, prefix_pages=64, prefix_len=FAKE, max_prefix=4096, block_table=FAKE, max_pages=16,
                seq_lens=FAKE, max_len=1024, scale=0.1, out=FAKE, ws=0x10000, ws_bytes=size, stream=None)
    refuses(lib.octopus_attn_decode_paged_prefix, PREFIX, good, [
        *[({name: None}, EINVAL) for name in ("cb", "q", "signs", "k_pool", "v_pool", "prefix_table", "prefix_len", "block_table", "seq_lens", "out")],
        *[({name: n}, EINVAL) for name in ("n_seq", "n_qh", "n_kv", "n_q", "n_pages", "prefix_pages", "max_pages") for n in (0, -1)],
        ({"n_qh": 30}, EINVAL), ({"causal": 2}, EINVAL), ({"causal": -1}, EINVAL),
        ({"max_prefix": -1}, EINVAL), ({"max_prefix": 4097}, EINVAL), ({"max_len": -1}, EINVAL), ({"max_len": 1025}, EINVAL),
        ({"max_prefix": 2 ** 31}, EINVAL), ({"max_len": 2 ** 31}, EINVAL), ({"prefix_pages": 2 ** 26}, EINVAL), ({"max_pages": 2 ** 26}, EINVAL),
        ({"n_seq": 2 ** 24 + 1, "n_q": 1, "n_qh": 1, "n_kv": 1}, EINVAL), ({"n_seq": 2 ** 20, "n_q": 16}, EINVAL),
        ({"q": FAKE + 2}, EINVAL), ({"out": FAKE + 2}, EINVAL), ({"k_pool": OFF8}, EINVAL), ({"v_pool": OFF8}, EINVAL),
        ({"q_lens": FAKE + 2}, EINVAL), ({"prefix_len": FAKE + 2}, EINVAL), ({"seq_lens": FAKE + 2}, EINVAL),
        ({"prefix_table": FAKE + 2}, EINVAL), ({"block_table": FAKE + 2}, EINVAL),
        ({"scale": float("nan")}, EINVAL), ({"scale": float("inf")}, EINVAL), ({"q_dtype": 2}, EUNSUPPORTED), ({"q_dtype": -1}, EUNSUPPORTED),
        ({"cb": ctypes.byref(broken)}, EINVAL), ({"cb": ctypes.byref(unbuilt)}, EUNSUPPORTED),
        ({"ws": None}, EWORKSPACE), ({"ws": 0x10080}, EWORKSPACE), ({"ws_bytes": size - 1}, EWORKSPACE), ({"ws_bytes": 0}, EWORKSPACE)])


def test_prefix_workspace_sizes(lib):
    cb, _ = books()
    size = lambda *a: binding.octopus_attn_prefix_workspace(cb, *a)  # noqa: E731
    assert size(3, 30, 8, 1, 64, 64) == 0 and size(0, 32, 8, 1, 64, 64) == 0 and size(3, 32, 8, 1, -1, 64) == 0
    assert binding.octopus_attn_prefix_workspace(unbuilt_books(), 1, 1, 1, 1, 64, 64) == 0
    assert size(1, 1, 1, 1, 0, 0) == 256                       # no tokens: no partial results
    assert size(1, 1, 1, 1, 1, 0) > 256 and size(1, 1, 1, 1, 0, 1) > 256
    one = 8 + 128 * 4                                          # a partial result of a query row
    assert size(64, 32, 8, 1, 8192, 0) >= 64 * 32 * one


def test_append_refusals_and_empty_calls(lib):
    cb, P = books()
    broken, unbuilt, edited = broken_books(), unbuilt_books(), binding.octopus_build_codebooks(128, 3)
    edited.c_xi[0][0] += 0.25
    rope = lambda **k: ctypes.byref(binding.Rope(*[{**dict(table=FAKE, n_pos=100, pos=None, dim=128, interleaved=0), **k}[n]  # noqa: E731
                                                   for n in ("table", "n_pos", "pos", "dim", "interleaved")]))
    good = dict(cb=P, k=FAKE, ks=8192, kt=1024, kh=128, v=FAKE, vs=8192, vt=1024, vh=128, kv_dtype=1, n_seq=2, n_kv=8, n_new=8, new_lens=None,
                rope=rope(), q=FAKE, q_dtype=1, qs=8192, qt=1024, qh=128, n_qh=32, q_out=FAKE, q_out_dtype=1, signs=FAKE, k_pool=FAKE,
                v_pool=FAKE, v_bits=0, v_group=0, n_pages=10, block_table=FAKE, max_pages=4, start_pos=FAKE, stream=None)
    refuses(lib.octopus_append_paged, APPEND, good, [
        *[({name: None}, EINVAL) for name in ("cb", "k", "v", "signs", "k_pool", "v_pool", "block_table", "q_out")],
        *[({name: n}, EINVAL) for name in ("n_seq", "n_kv", "n_pages", "max_pages", "n_qh") for n in (0, -1)],
        ({"n_new": -1}, EINVAL), ({"n_qh": 30}, EINVAL), ({"n_seq": 65536}, EINVAL), ({"n_kv": 65536, "n_qh": 65536}, EINVAL),
        *[({name: n}, EINVAL) for name in ("ks", "kt", "kh", "vs", "vt", "vh", "qs", "qt", "qh") for n in (-8, 4, 1)],
        *[({name: OFF8}, EINVAL) for name in ("k", "v", "q", "q_out", "k_pool", "v_pool")],
        *[({name: FAKE + 2}, EINVAL) for name in ("new_lens", "start_pos", "block_table")],
        *[({name: n}, EUNSUPPORTED) for name in ("kv_dtype", "q_dtype", "q_out_dtype") for n in (2, -1)],
        *[({"v_bits": b, "v_group": g}, EUNSUPPORTED) for b, g in ((1, 16), (5, 16), (8, 32), (-1, 16), (3, 0), (3, 64))],
        *[({"rope": rope(**k)}, EINVAL) for k in (dict(table=None), dict(table=OFF8), dict(n_pos=0), dict(n_pos=-5), dict(pos=FAKE + 2),
                                                  dict(dim=0), dict(dim=8), dict(dim=24), dict(dim=144), dict(dim=-16), dict(interleaved=2))],
        ({"start_pos": None, "n_new": 257}, EINVAL), ({"max_pages": 2 ** 26}, EINVAL), ({"n_new": 2 ** 30}, EINVAL),
        ({"cb": ctypes.byref(broken)}, EINVAL), ({"cb": ctypes.byref(unbuilt)}, EUNSUPPORTED), ({"cb": ctypes.byref(edited)}, EUNSUPPORTED),
        ({"n_new": 0}, OK), ({"n_new": 0, "k": None, "v": None, "q": None}, OK)])      # (an empty tensor may have no address)


def test_read_refusals_and_empty_calls(lib):
    cb, P = books()
    broken, unbuilt = broken_books(), unbuilt_books()
    good = dict(cb=P, signs=FAKE, k_pool=FAKE, v_pool=FAKE, v_bits=0, v_group=0, n_pages=10, block_table=FAKE, max_pages=4, n_seq=2, n_kv=8,
                start_pos=FAKE, n_tok=8, lens=None, k_out=FAKE, v_out=FAKE, out_dtype=1, stream=None)
    refuses(lib.octopus_read_paged, READ, good, [
        *[({name: None}, EINVAL) for name in ("cb", "signs", "k_pool", "v_pool", "block_table")],
        ({"k_out": None, "v_out": None}, EINVAL), ({"k_pool": None, "k_out": FAKE}, EINVAL),
        *[({name: n}, EINVAL) for name in ("n_seq", "n_kv", "n_pages", "max_pages") for n in (0, -1)],
        ({"n_seq": 65536}, EINVAL), ({"n_kv": 65536}, EINVAL), ({"n_tok": -1}, EINVAL), ({"n_tok": 2 ** 30}, EINVAL),
        ({"start_pos": None, "n_tok": 257}, EINVAL), ({"max_pages": 2 ** 26}, EINVAL),
        *[({name: OFF8}, EINVAL) for name in ("k_pool", "v_pool", "k_out", "v_out")],
        *[({name: FAKE + 2}, EINVAL) for name in ("lens", "start_pos", "block_table")],
        ({"out_dtype": 2}, EUNSUPPORTED), *[({"v_bits": b, "v_group": g}, EUNSUPPORTED) for b, g in ((1, 16), (5, 32), (3, 8), (4, 0))],
        ({"cb": ctypes.byref(broken)}, EINVAL), ({"cb": ctypes.byref(unbuilt)}, EUNSUPPORTED),
        ({"n_tok": 0}, OK), ({"n_tok": 0, "k_out": None, "v_out": None}, OK),
        ({"n_tok": 0, "signs": None, "k_pool": None, "k_out": None}, OK)])


def test_structs(lib):
    assert ctypes.sizeof(binding.Rope) == 8 + 8 + 8 + 4 + 4


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if HIPCC is None:
        pytest.skip("hipcc not found")
    exe = str(tmp_path_factory.mktemp("host") / "prefix_shape_driver")
    csrc = os.path.join(ROOT, "paper_2605_21226_amd", "csrc")
    run = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-I" + os.path.join(ROOT, "include"), "-I" + csrc,
                          "-Wno-unused-command-line-argument", os.path.join(csrc, "octopus_host.cpp"), os.path.join(csrc, "octopus_serve_host.cpp"),
                          os.path.join(ROOT, "tests", "host", "prefix_shape_driver.cpp"), "-o", exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stderr[-4000:]
    return exe


CALLS = [(d, bits, *shape) for d, bits in ((64, 4), (128, 3), (256, 2.5)) for shape in (
    (1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 0, 1), (1, 1, 1, 1, 0, 0), (4, 32, 8, 1, 700, 60), (64, 32, 8, 1, 8192, 1500), (16, 32, 8, 1, 65531, 512),
    (8, 24, 24, 5, 3600, 333), (3, 6, 2, 12, 33, 500), (1, 8, 1, 1, 2_000_000, 0), (300, 8, 1, 1, 0, 40), (2, 64, 1, 70, 64, 130_000),
    (1024, 16, 16, 1, 100, 4096), (7, 7, 7, 3, 31, 32), (1, 128, 128, 1, 513, 257))]


def test_the_division_covers_the_call(driver):
    out = subprocess.run([driver, *[str(x) for c in CALLS for x in c]], capture_output=True, text=True, timeout=120, check=True).stdout.splitlines()
    assert len(out) == len(CALLS)
    for (d, bits, n_seq, n_qh, n_kv, n_q, max_prefix, max_len), line in zip(CALLS, out):
        group, waves, p_groups, p_splits, o_groups, o_splits, p_segs, segs, first_own, room = map(int, line.split())
        where = (d, n_seq, n_qh, n_kv, n_q, max_prefix, max_len)
        own_rows = n_q * n_qh // n_kv
        assert group * p_groups >= own_rows * n_seq > group * (p_groups - 1) or max_prefix == 0, where
        assert group * o_groups >= own_rows > group * (o_groups - 1), where
        assert (p_splits > 0) == (max_prefix > 0) and (o_splits > 0) == (max_len > 0) and max(p_splits, o_splits) <= 128, where
        assert p_segs == n_kv * p_groups * p_splits and segs == p_segs + n_seq * n_kv * o_groups * o_splits, where
        rows = n_seq * n_q * n_qh
        assert first_own == rows * p_splits and room >= rows * (p_splits + o_splits) * (segs > 0), where
        # eight dies take the prefix's segments in runs: each segment once
        taken = [seg % 8 * (p_segs // 8) + min(seg % 8, p_segs % 8) + seg // 8 for seg in range(p_segs)]
        assert sorted(taken) == list(range(p_segs)), where
        # ranges of 32-token steps that a length is cut into: all of its steps, in order, no range empty before a full one
        for length in {0, 1, 31, 32, 33, max_prefix // 3, max_prefix, max_len // 2, max_len}:
            for splits, most in ((p_splits, max_prefix), (o_splits, max_len)):
                if length > most or splits == 0:
                    continue
                steps = -(-length // 32)
                per = -(-steps // splits)
                ranges = [(s * per, min((s + 1) * per, steps)) for s in range(splits) if s * per < min((s + 1) * per, steps)]
                assert [t for a, b in ranges for t in range(a, b)] == list(range(steps)) and len(ranges) == (-(-steps // per) if per else 0), where

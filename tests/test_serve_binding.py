"""What the Python entry points over pages refuse before the library is asked: views that a call would write past, or read past, and
pools of another type or size.  Tensors lie on the CPU; no call gets as far as a launch."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2605_21226_amd import binding  # noqa: E402

N_SEQ, N_NEW, N_KV, G, PAGES, N_PAGES = 2, 3, 2, 2, 1, 4


class Reached(Exception):
    """the library was asked"""


@pytest.fixture
def asked(monkeypatch):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_21226_amd import build
        build.build(verbose=False)
    books = {d: binding.octopus_build_codebooks(d, 3) for d in (64, 128)}

    class Library:
        def __getattr__(self, name):
            def f(*_):
                raise Reached
            return f
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: None)
    return books


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def pools(cb, v_bits=0, v_group=0, pages=N_PAGES):
    d = cb.plan.head_dim
    k = torch.zeros(pages * N_KV * 64 * 16 * cb.plan.granules, dtype=torch.uint8)
    row = v_bits * d // 8 + d // v_group * 8 if v_bits else 0
    return k, (torch.zeros((pages, N_KV, 64, row), dtype=torch.uint8) if v_bits else bf16(pages, N_KV, 64, d))


def append(cb, d=128, **changes):
    k_pool, v_pool = pools(cb, changes.get("v_bits", 0), changes.get("v_group", 0))
    args = dict(k=bf16(N_SEQ, N_NEW, N_KV, d), v=bf16(N_SEQ, N_NEW, N_KV, d), signs=torch.zeros((N_KV, d // 8), dtype=torch.uint8), k_pool=k_pool,
                v_pool=v_pool, n_pages=N_PAGES, block_table=torch.zeros((N_SEQ, PAGES), dtype=torch.int32), q=bf16(N_SEQ, N_NEW, N_KV * G, d),
                q_out=bf16(N_SEQ, N_NEW, N_KV * G, d))
    args.update(changes)
    binding.octopus_append_paged(cb, **args)


def read(cb, d=128, **changes):
    k_pool, v_pool = pools(cb, changes.get("v_bits", 0), changes.get("v_group", 0))
    args = dict(signs=torch.zeros((N_KV, d // 8), dtype=torch.uint8), k_pool=k_pool, v_pool=v_pool, n_pages=N_PAGES,
                block_table=torch.zeros((N_SEQ, PAGES), dtype=torch.int32), k_out=bf16(N_SEQ, N_NEW, N_KV, d), v_out=bf16(N_SEQ, N_NEW, N_KV, d))
    args.update(changes)
    binding.octopus_read_paged(cb, **args)


def prefix(cb, d=128, **changes):
    k_pool, v_pool = pools(cb)
    args = dict(q=bf16(N_SEQ, 1, N_KV * G, d), signs=torch.zeros((N_KV, d // 8), dtype=torch.uint8), k_pool=k_pool, v_pool=v_pool, prefix_table=None,
                prefix_len=None, max_prefix=0, block_table=torch.zeros((N_SEQ, PAGES), dtype=torch.int32),
                seq_lens=torch.zeros(N_SEQ, dtype=torch.int32), max_len=64, scale=0.1, out=torch.zeros((N_SEQ, 1, N_KV * G, d)),
                workspace=torch.zeros(4096, dtype=torch.uint8))
    args.update(changes)
    binding.octopus_attn_decode_paged_prefix(cb, **args)


def test_calls_that_fit_reach_the_library(asked):
    cb = asked[128]
    for call, changes in ((append, {}), (append, dict(q=None, q_out=None)), (append, dict(v_bits=3, v_group=32)), (read, {}), (read, dict(k_out=None, k_pool=None)),
                          (read, dict(v_out=None, v_pool=None)), (read, dict(v_bits=4, v_group=16)), (prefix, {}),
                          (append, dict(v_bits=3, v_group=32, v_pool=torch.zeros(N_PAGES * N_KV * 64 * 80, dtype=torch.uint8))),      # a flat pool
                          (append, dict(v_pool=bf16(N_PAGES + 1, N_KV, 64, 128)))):
        with pytest.raises(Reached):
            call(cb, **changes)


@pytest.mark.parametrize("call", [append, read, prefix])
def test_rows_of_another_head_dimension(asked, call):
    with pytest.raises(AssertionError):
        call(asked[64], d=128)
    with pytest.raises(AssertionError):
        call(asked[128], d=64)


@pytest.mark.parametrize("changes", [
    dict(q=bf16(N_SEQ, N_NEW, N_KV * G, 64), q_out=bf16(N_SEQ, N_NEW, N_KV * G, 64)),
    dict(q=bf16(N_SEQ, N_NEW, N_KV * G, 256), q_out=bf16(N_SEQ, N_NEW, N_KV * G, 256)),
    dict(q_out=bf16(N_SEQ, N_NEW, N_KV * G, 64)),
    dict(v_pool=torch.zeros((N_PAGES, N_KV, 64, 128), dtype=torch.float32)),          # bf16 rows are written
    dict(v_pool=torch.zeros((N_PAGES, N_KV, 64, 128), dtype=torch.uint8)),
    dict(v_pool=bf16(N_PAGES - 1, N_KV, 64, 128)),
    dict(k_pool=torch.zeros(N_PAGES * N_KV * 64 * 16 * 4 - 16, dtype=torch.uint8)),
    dict(v_bits=3, v_group=32, v_pool=torch.zeros((N_PAGES, N_KV, 64, 64), dtype=torch.uint8)),
    dict(n_pages=N_PAGES + 1)])
def test_appending_past_a_tensor(asked, changes):
    assert asked[128].plan.granules == 4
    with pytest.raises((AssertionError, TypeError)):
        append(asked[128], **changes)


@pytest.mark.parametrize("changes", [
    dict(k_pool=torch.zeros(N_PAGES * N_KV * 64 * 16 * 4 - 16, dtype=torch.uint8)), dict(v_pool=bf16(N_PAGES + 1, N_KV, 64, 128)),
    dict(v_pool=torch.zeros((N_PAGES, N_KV, 64, 128), dtype=torch.float32)), dict(v_pool=bf16(N_PAGES, N_KV, 128, 64).transpose(2, 3))])
def test_attending_past_a_tensor(asked, changes):
    with pytest.raises((AssertionError, TypeError)):
        prefix(asked[128], **changes)


@pytest.mark.parametrize("changes", [
    dict(k_out=bf16(N_SEQ, N_NEW, N_KV, 64), v_out=bf16(N_SEQ, N_NEW, N_KV, 64)), dict(v_out=bf16(N_SEQ, N_NEW, N_KV, 64)),
    dict(v_pool=torch.zeros((N_PAGES, N_KV, 64, 128), dtype=torch.float32)), dict(v_pool=bf16(N_PAGES - 1, N_KV, 64, 128)),
    dict(v_bits=3, v_group=16), dict(n_pages=N_PAGES + 1)])
def test_reading_past_a_tensor(asked, changes):
    changes = dict(changes)
    if "v_bits" in changes:       # rows of groups of 32 in the pool
        changes["v_pool"] = pools(asked[128], 3, 32)[1]
    with pytest.raises((AssertionError, TypeError)):
        read(asked[128], **changes)

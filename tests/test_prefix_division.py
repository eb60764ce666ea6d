"""On the CPU: the shapes of tests/prefix_shapes.py are divided as their GPU tests need them."""
import subprocess

import pytest

from prefix_shapes import LONG_RANGES, MANY_SEGMENTS
from test_serve_host import driver  # noqa: F401  (the fixture)

GRID = 256                  # workgroups of a launch at most
HELD = 64                   # steps of a wavefront whose page numbers it holds at once


def divide(driver, d, bits, n_seq, n_qh, n_kv, n_q, max_prefix, max_len):  # noqa: F811
    args = [str(x) for x in (d, bits, n_seq, n_qh, n_kv, n_q, max_prefix, max_len)]
    line = subprocess.run([driver, *args], capture_output=True, text=True, timeout=60, check=True).stdout
    _, waves, _, p_splits, _, o_splits, p_segs, segs, _, _ = map(int, line.split())
    return waves, p_splits, o_splits, p_segs, segs


@pytest.mark.parametrize("shape", MANY_SEGMENTS)
def test_workgroups_take_several_segments(driver, shape):  # noqa: F811
    d, bits, n_qh, n_kv, n_q, prefix, lens, _, _ = shape
    _, _, _, p_segs, segs = divide(driver, d, bits, len(lens), n_qh, n_kv, n_q, prefix, max(lens))
    assert segs > GRID and (p_segs > 0) == (prefix > 0)
    if prefix:
        assert p_segs < segs                 # both kinds


def test_some_workgroups_take_three_or_more(driver):  # noqa: F811
    most = 0
    for d, bits, n_qh, n_kv, n_q, prefix, lens, _, _ in MANY_SEGMENTS:
        most = max(most, divide(driver, d, bits, len(lens), n_qh, n_kv, n_q, prefix, max(lens))[4])
    assert most > 2 * GRID


@pytest.mark.parametrize("shape", LONG_RANGES)
def test_ranges_outlast_the_held_page_numbers(driver, shape):  # noqa: F811
    d, bits, n_qh, n_kv, n_q, n_seq, prefix, own, _ = shape
    waves, p_splits, o_splits, _, _ = divide(driver, d, bits, n_seq, n_qh, n_kv, n_q, prefix, own)
    tokens, splits = (own, o_splits) if own > prefix else (prefix, p_splits)
    steps = -(-tokens // 32)
    assert -(-steps // splits) > 2 * HELD * waves      # asked for anew twice

"""Shapes of octopus_attn_decode_paged_prefix whose workgroups take several segments, or segments of more steps than a wavefront holds
page numbers for.  The GPU tests run them; tests/test_prefix_division.py says on the CPU that the library divides them so."""
import numpy as np


def _lens(seed, n, least, most):
    """Ragged lengths with the longest, the shortest and some sequences without a token among them."""
    rng = np.random.default_rng(seed)
    x = rng.integers(least, most + 1, n)
    x[rng.integers(0, n, n // 6)] = least
    x[rng.integers(0, n, 2)] = most
    return [int(t) for t in x]


# head dimension, bits, query heads, KV heads, queries, prefix, own lengths, causal, queries of each sequence that count
MANY_SEGMENTS = [
    (128, 3, 8, 4, 1, 300, _lens(1, 70, 0, 120), False, None),
    (128, 1.5, 32, 4, 6, 70, _lens(2, 30, 6, 90), True, None),
    (128, 3, 16, 4, 20, 0, _lens(3, 26, 0, 100), True, _lens(4, 26, 0, 20)),
    (64, 4, 16, 4, 20, 130, _lens(5, 24, 20, 60), True, _lens(6, 24, 0, 20)),
    (64, 2, 8, 4, 1, 1000, _lens(7, 70, 0, 40), False, None),
    (256, 2.5, 16, 4, 9, 70, _lens(8, 36, 9, 40), True, None),
    (256, 4, 8, 4, 1, 200, _lens(9, 70, 0, 60), False, None)]

# head dimension, bits, query heads, KV heads, queries, sequences, prefix, own tokens, causal
LONG_RANGES = [
    (128, 3, 8, 8, 1, 32, 0, 35_001, False),
    (128, 2.5, 8, 8, 2, 32, 0, 35_011, True),
    (64, 4, 8, 8, 1, 32, 0, 35_001, False),
    (256, 2.5, 8, 8, 2, 32, 0, 17_450, True),
    (128, 3, 16, 1, 1, 510, 35_041, 0, False),
    (256, 3, 8, 1, 1, 510, 17_450, 0, False)]

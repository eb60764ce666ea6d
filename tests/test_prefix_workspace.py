"""Host checks of octopus_attn_prefix_workspace: a larger shape's workspace serves every smaller shape, and none is out of proportion."""
import random

import pytest

from paper_2605_21226_amd import binding


@pytest.fixture(scope="module")
def books():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2605_21226_amd import build
        build.build(verbose=False)
    return {(d, b): binding.octopus_build_codebooks(d, b) for d, b in ((64, 4), (128, 3), (256, 2.5))}


def size(cb, n_seq, g, n_kv, n_q, prefix, own):
    n = binding.octopus_attn_prefix_workspace(cb, n_seq, g * n_kv, n_kv, n_q, prefix, own)
    assert n > 0
    return n


def log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


@pytest.mark.parametrize("d,bits,small,large", [
    (128, 3, (16, 4, 8, 1, 11264, 4096), (16, 4, 8, 1, 15360, 4096)),
    (256, 2.5, (33, 4, 8, 1, 16384, 512), (64, 4, 8, 1, 16384, 512)),
    (128, 3, (64, 4, 8, 1, 8192, 2048), (64, 4, 8, 1, 8192, 3000)),
    (128, 3, (16, 8, 8, 1, 4096, 1056), (16, 8, 8, 1, 4096, 2186)),
    (128, 3, (3, 4, 2, 1, 500, 64), (3, 4, 2, 4, 500, 64))])
def test_shapes_of_a_server(books, d, bits, small, large):
    assert size(books[d, bits], *small) <= size(books[d, bits], *large)


def test_a_larger_shapes_workspace_serves_every_smaller_one(books):
    rng = random.Random(5)
    for _ in range(4000):
        cb = books[rng.choice(list(books))]
        n_kv = rng.choice([1, 2, 3, 8, 24])
        low, high = [], []
        for top in (300, 8, 70, 200_000, 200_000):          # sequences, heads a KV head, queries, prefix, own tokens
            a, b = sorted(log_uniform(rng, 1, top) for _ in range(2))
            a, b = (a, a) if rng.random() < 0.5 else (a, b)
            if top == 200_000 and rng.random() < 0.3:
                a, b = 0, b if rng.random() < 0.5 else 0
            low.append(a)
            high.append(b)
        order = lambda x: (x[0], x[1], n_kv, *x[2:])  # noqa: E731
        assert size(cb, *order(low)) <= size(cb, *order(high)), (cb.plan.head_dim, low, high)


def test_proportions(books):
    """One partial result a row of either kind at least; 2^18 of either kind are the most that ranges add."""
    for (d, _), cb in books.items():
        one = 8 + 4 * d
        for n_seq, g, n_kv, n_q, prefix, own in ((64, 4, 8, 1, 8192, 1500), (300, 8, 8, 70, 200_000, 200_000), (1, 1, 1, 1, 2 ** 30, 0), (1, 1, 1, 1, 1, 1)):
            rows, n = n_seq * g * n_kv * n_q, size(cb, n_seq, g, n_kv, n_q, prefix, own)
            assert rows * ((prefix > 0) + (own > 0)) * one <= n <= 2 * max(rows, 2 ** 18) * one + 1024

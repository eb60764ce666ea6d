"""Operators around a server's pages of compressed keys, as measured cases.

  axes       a step's keys, values and queries into pages, rotated by positions of several axes (frame, row, column of an
             image's or a video's patches); then what the pages hold is read back
  fork       who holds which page: sequences fork from others, drop what was rejected and get pages for their next tokens;
             a page that two of them would write into is copied, in every layer's pools
  turnover   sequences leave and others arrive; in between the pages in use are moved to the front of the pools
  verify     drafted tokens accepted or refused by the target's and the drafter's probabilities, and the token after them

Sizes are those of this repository's workloads (32 query and 8 KV heads of 128, 24 heads of 64, 16 and 8 heads of 256) where one
fits, else generic serving sizes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TILE = 64
BASE = 500000.0      # of the rotation's angles


def _case(name, op, **fields):
    c = {"op": op}
    if op == "axes":
        c.update({"n_q_heads": 32, "n_kv": 8, "d": 128, "bits": 3.0, "dtype": "bf16", "n_new": 1, "start": 0, "ragged": False,
                  "rot": 128, "interleaved": False, "n_axes": 3, "turns": False, "width": 32})
    elif op == "verify":
        c.update({"n_draft": 4, "vocab": 32000, "dtype": "fp32", "sampled": True, "ragged": False, "agree": 0.3})
    else:
        c.update({"n_kv": 8, "d": 128, "bits": 3.0, "layers": 1, "tokens": 1000, "ragged": True})
        c.update({"beams": 1, "alive": 1, "n_new": 1} if op == "fork" else {"retire": 1})
    c.update(fields)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a server's batch in its ordinary step, the sequences with images or videos somewhere before
        _case("axes_batch", "axes", n_seq=64, n_new=1, start=8000, ragged=True),
        # a video's patches as the prompt: 20 frames of 24 x 33
        _case("axes_video", "axes", n_seq=1, n_new=15840, width=33),
        # a padded batch of images in fp32 at 24 heads of 64, two axes in turns over half of the channels, neighbouring pairs
        _case("axes_images_fp32", "axes", n_seq=5, n_q_heads=24, n_kv=24, d=64, bits=4.0, dtype="fp32", n_new=509, start=77, ragged=True,
              rot=32, interleaved=True, n_axes=2, turns=True, width=23),
        # a server's ordinary step: rejected drafts dropped, pages for the next ones, nothing shared
        _case("fork_step", "fork", n_seq=256, tokens=8000, n_new=5),
        # beam search: 16 requests of four beams, two of which live on
        _case("fork_beams", "fork", n_seq=64, beams=4, alive=2, tokens=2000, layers=8),
        # 64 samples of one long prompt
        _case("fork_samples", "fork", n_seq=64, beams=64, alive=1, tokens=65531, layers=16, ragged=False),
        # a batch of chats of all lengths, a few of which end
        _case("turnover_chats", "turnover", n_seq=32, tokens=4000, layers=8, retire=4),
        # many short sequences, 24 heads of 64 at 4 bits, half of them replaced
        _case("turnover_short", "turnover", n_seq=200, n_kv=24, d=64, bits=4.0, tokens=200, layers=2, retire=100),
        # one user's step, four drafted tokens
        _case("verify_one", "verify", n_seq=1),
        # a server's batch, a padded one, probabilities in bf16
        _case("verify_batch", "verify", n_seq=64, n_draft=5, vocab=128256, dtype="bf16", ragged=True),
        # drafts that were looked up in the prompt and have no probabilities
        _case("verify_lookup", "verify", n_seq=8, n_draft=9, vocab=50257, sampled=False, ragged=True, agree=0.8),
        # a large batch
        _case("verify_many", "verify", n_seq=256, n_draft=3, vocab=128256),
    ]


def _log_uniform(rng, lo, hi):
    lo = min(lo, max(1, hi))
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["axes", "axes", "fork", "fork", "turnover", "verify", "verify"])
    if op == "verify":
        n_draft, vocab = rng.choice([1, 2, 3, 5, 8, 13]), _log_uniform(rng, 700, 160000)
        return _case(None, op, n_seq=_log_uniform(rng, 1, min(256, 256 * 4 * 128256 // ((n_draft + 1) * vocab))), n_draft=n_draft, vocab=vocab,
                     dtype=rng.choice(["fp32", "fp32", "bf16"]), sampled=rng.random() < 0.7, ragged=rng.random() < 0.6,
                     agree=rng.choice([0.1, 0.3, 0.8, 2.0]))
    d = rng.choice([64, 128, 128, 256])
    n_kv, bits = rng.choice([1, 2, 4, 8, 8]), rng.choice([1.0, 1.5, 2.0, 2.5, 3.0, 3.0, 4.0])
    if op == "axes":
        n_seq = rng.choice([1, 1, 2, 3, 8, 33, 64])
        n_new = 1 if rng.random() < 0.3 else _log_uniform(rng, 1, 15840 * 8 * 128 // (2 * n_seq * n_kv * d))
        return _case(None, op, n_seq=n_seq, n_q_heads=n_kv * rng.choice([1, 2, 3, 4, 4]), n_kv=n_kv, d=d, bits=bits,
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), n_new=n_new, start=rng.choice([0, _log_uniform(rng, 1, 8000)]),
                     ragged=rng.random() < 0.6, rot=rng.choice([d, d, d // 2, 48]), interleaved=rng.random() < 0.3,
                     n_axes=rng.choice([2, 3, 3, 4]), turns=rng.random() < 0.4, width=_log_uniform(rng, 5, 64))
    layers = rng.choice([1, 2, 5, 8])
    room = 2000000000 // (layers * n_kv * d * 200)             # pages
    if op == "fork":
        beams = rng.choice([1, 1, 2, 3, 4, 8, 17])
        n_seq = beams * _log_uniform(rng, 1, min(256, room // 4) // beams)
        return _case(None, op, n_seq=n_seq, n_kv=n_kv, d=d, bits=bits, layers=layers, beams=beams, alive=rng.randint(1, beams),
                     tokens=_log_uniform(rng, 1, min(65000, TILE * max(1, room // n_seq - 2))), n_new=rng.choice([1, 1, 5, 64, 130]),
                     ragged=rng.random() < 0.7)
    n_seq = _log_uniform(rng, 3, min(200, room // 2))
    return _case(None, op, n_seq=n_seq, n_kv=n_kv, d=d, bits=bits, layers=layers, retire=_log_uniform(rng, 1, n_seq // 2),
                 tokens=_log_uniform(rng, 1, min(8000, TILE * (room // n_seq))), ragged=rng.random() < 0.7)


# ---- the plan of a width, its codebooks, and the sizes that follow ---------------------------------------------------
def _classes(c):
    """[(first triplet, triplets, direction bits, norm bits)]"""
    n_tri = (c["d"] + 2) // 3
    split = lambda b: (1, 1) if b == 1 else (b + 1, b - 1)  # noqa: E731
    twice = int(round(2 * c["bits"]))
    if twice % 2 == 0:
        return [(0, n_tri) + split(twice // 2)]
    first = (n_tri + 1) // 2
    return [(0, first) + split((twice + 1) // 2), (first, n_tri - first) + split((twice - 1) // 2)]


def _stream(n, b):
    g = 8 // math.gcd(b, 8)
    return (n + g - 1) // g * (g * b // 8)


def _record(c):
    return 4 + sum(_stream(2 * n, bd) + _stream(n, bn) for _, n, bd, bn in _classes(c))


def _granules(c):
    return (_record(c) + 15) // 16


def _page_bytes(c):
    """Of a layer's keys and values."""
    return c["n_kv"] * TILE * (16 * _granules(c) + 2 * c["d"])


_BOOKS = {}


def _lloyd_max(density, levels):
    """Lloyd-Max centroids of a density on [0, 1], to the fixed point, from the equal-probability quantiles."""
    n = 1 << 17
    x = (np.arange(n) + 0.5) / n
    f = density(x)
    edge = np.arange(n + 1) / n
    mass = np.concatenate([[0.0], np.cumsum(f) / n])
    mom = np.concatenate([[0.0], np.cumsum(f * x) / n])

    def at(cum, slope, e):     # cumulative at e: a whole number of cells plus the part of one
        i = np.minimum((e * n).astype(np.int64), n - 1)
        return cum[i] + slope[i] * (e - edge[i])
    c = np.interp((np.arange(levels) + 0.5) / levels * mass[-1], mass, edge)
    for _ in range(100000):
        e = np.concatenate([[0.0], 0.5 * (c[1:] + c[:-1]), [1.0]])
        new = np.diff(at(mom, f * x, e)) / np.diff(at(mass, f, e))
        moved = np.abs(new - c).max()
        c = new
        if moved < 1e-12:
            break
    return c


def _book_xi(b):
    if ("xi", b) not in _BOOKS:
        def density(a):
            return ((1 - a) / (1 - 2 * a + 3 * a * a) + a / (2 - 4 * a + 3 * a * a)) / np.sqrt(a * a + (1 - a) ** 2)
        half = _lloyd_max(density, 1 << (b - 1))
        _BOOKS["xi", b] = np.concatenate([-half[::-1], half]).astype(np.float32)
    return _BOOKS["xi", b]


def _book_rho(d, b):
    if ("rho", d, b) not in _BOOKS:
        def density(r):
            g = r * r * (1 - r * r) ** (0.5 * (d - 5))
            return g / g.mean()
        _BOOKS["rho", d, b] = _lloyd_max(density, 1 << b).astype(np.float32)
    return _BOOKS["rho", d, b]


# ---- inputs, from the seed alone ----------------------------------------------------------------------------------
def _gen(seed, *stream):
    g = torch.Generator(device=DEV)
    x = int(seed) & 0x7FFFFFFF
    for s in stream:
        x = (x * 1000003 + int(s) * 7919 + 12345) & 0x7FFFFFFFFFFF
    g.manual_seed(x)
    return g


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _some(c, seed, stream, lo, hi, n):
    """n numbers: hi, or anything in [lo, hi] with hi among them."""
    x = np.full(n, hi, dtype=np.int32)
    if c["ragged"] and hi > lo:
        r = np.random.default_rng([int(seed), stream])
        x = r.integers(lo, hi + 1, size=n).astype(np.int32)
        x[int(r.integers(0, n))] = hi
    return x


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _axis_of(c):
    """The axis of every pair: a run of pairs an axis, the first one (frames) with fewer, or the axes in turns."""
    i, n = np.arange(c["rot"] // 2), c["n_axes"]
    if c["turns"]:
        return i % n
    return np.minimum((i + len(i) // (4 * n)) * n // len(i), n - 1)


def _prepare_axes(c, seed):
    n_seq, n_kv, d, n_new, heads = c["n_seq"], c["n_kv"], c["d"], c["n_new"], c["n_q_heads"]
    st = {"had": _hadamard(d), "books": _device_books(c)}
    r = np.random.default_rng([int(seed), 101])
    s = r.integers(0, 2, size=(n_kv, d)).astype(np.int8) * 2 - 1
    st["sign"] = torch.from_numpy(s).to(DEV).float()
    st["signs"] = torch.from_numpy(np.packbits((s < 0).astype(np.uint8), axis=-1, bitorder="little")).to(DEV)
    # channel scales of real decoders' keys: log-normal, four channels of a head ten times as large
    sig = np.exp(0.5 * r.standard_normal((n_kv, d)))
    np.put_along_axis(sig, np.argsort(r.random((n_kv, d)), axis=1)[:, :4], 10.0, axis=1)
    start = _some(c, seed, 303, 0, c["start"], n_seq)
    st["new_lens"], st["start"] = _ints(_some(c, seed, 304, 0, n_new, n_seq)), _ints(start)
    # one projection's output: queries, keys and values of a token side by side
    qkv = torch.randn((n_seq, n_new, heads + 2 * n_kv, d), generator=_gen(seed, 3), device=DEV)
    qkv[:, :, heads:heads + n_kv].mul_(torch.from_numpy(sig.astype(np.float32)).to(DEV))
    st["q"], st["k"], st["v"] = qkv.to(_dtype(c)).split([heads, n_kv, n_kv], dim=2)
    # positions: some text, then patches by frame, row and column (a last axis counts them), frames of 24 rows
    i = np.arange(n_new)
    patch = np.stack([i // (24 * c["width"]), i // c["width"] % 24, i % c["width"], i % 1000])
    pos = r.integers(0, 4000, size=n_seq)[None, :, None] + patch[[1, 2] if c["n_axes"] == 2 else np.arange(c["n_axes"])][:, None]
    st["pos"] = _ints(pos)                                                                  # [axis, seq, token]
    st["axis"] = bytes(_axis_of(c).astype(np.uint8))
    n_pos = int(pos.max()) + 1
    f = BASE ** (-2.0 * torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64) / c["rot"])
    angle = torch.arange(n_pos, device=DEV, dtype=torch.float64)[:, None] * f
    st["rope"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
    per = (int(start.max()) + n_new + TILE - 1) // TILE
    st["n_pages"] = n_seq * per
    st["table"] = _ints(r.permutation(st["n_pages"]).reshape(n_seq, per))
    st["k_pool"] = torch.zeros((st["n_pages"], n_kv, _granules(c), TILE, 16), dtype=torch.uint8, device=DEV)
    st["v_pool"] = torch.zeros((st["n_pages"], n_kv, TILE, d), dtype=torch.bfloat16, device=DEV)
    st["q_out"] = torch.zeros((n_seq, n_new, heads, d), dtype=_dtype(c), device=DEV)
    st["k_out"] = torch.zeros((n_seq, n_new, n_kv, d), dtype=torch.bfloat16, device=DEV)
    st["v_out"] = torch.zeros_like(st["k_out"])
    if own:
        from paper_2605_21226_amd import binding as lib
        st["lib"], st["cb"] = lib, lib.octopus_build_codebooks(d, c["bits"])
    return st


def _tokens(c, seed):
    """Tokens of each sequence (fork: beams of a request have as many): the same lengths in another order with another seed."""
    each = c.get("beams", 1)
    n = c["n_seq"] // each
    lens = np.linspace(max(1, c["tokens"] // 8) if c["ragged"] else c["tokens"], c["tokens"], n).round().astype(np.int32)[::-1]
    return np.random.default_rng([int(seed), 305]).permutation(lens).repeat(each)


def _prepare_pages(c, seed):
    n_seq, layers, n_kv = c["n_seq"], c["layers"], c["n_kv"]
    r = np.random.default_rng([int(seed), 707])
    lens = _tokens(c, seed)
    pages = -(-lens // TILE)
    grown = -(-(lens + c.get("n_new", 0)) // TILE)
    per = int(grown.max()) + 2
    st = {}
    if c["op"] == "fork":
        # which beams live on, and whom each of the others takes over from (one that lives, of its request)
        order = np.argsort(r.random((n_seq // c["beams"], c["beams"])), axis=1)
        chosen = np.take_along_axis(order, r.integers(0, c["alive"], size=order.shape), axis=1)
        np.put_along_axis(chosen, order[:, :c["alive"]], order[:, :c["alive"]], axis=1)
        source = (chosen + np.arange(0, n_seq, c["beams"])[:, None]).reshape(-1)
        st["source"] = _ints(source) if c["beams"] > 1 else None
        st["keep"], st["new_lens"] = _ints(lens), _ints(lens + c["n_new"])
        if c["beams"] > 16:      # samples of a prompt: nothing but the prompt yet
            pages = np.where(source == np.arange(n_seq), pages, 0)
            lens = np.where(source == np.arange(n_seq), lens, 0)
    n_held = int(pages.sum())
    n_pages = n_held + (int((grown - pages.clip(min=grown - 2)).sum()) + 2 * n_seq if c["op"] == "fork" else n_held // 8 + 2)
    table = np.zeros((n_seq, per), dtype=np.int32)
    held = np.arange(per) < pages[:, None]
    if c["op"] == "fork":        # pages as a server in its midst has them; a turnover's are together at the front
        ids = r.permutation(n_pages)[:n_held]
    else:
        ids = r.permutation(n_held)
    table[held] = ids
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[ids] = 1
    st["refs"], st["table"], st["lens"] = _ints(refs), _ints(table), _ints(lens)
    st["moves"] = torch.zeros(2 + 2 * max(n_seq, n_pages // 2), dtype=torch.int32, device=DEV)
    st["map"] = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    st["k"] = torch.randint(0, 256, (layers, n_pages, n_kv, _granules(c), TILE, 16), generator=_gen(seed, 5), dtype=torch.uint8, device=DEV)
    st["v"] = torch.randint(-30000, 30000, (layers, n_pages, n_kv, TILE, c["d"]), generator=_gen(seed, 6), dtype=torch.int16, device=DEV)
    if own:      # the handles and the workspace of the library
        from paper_2605_21226_amd import binding as lib
        st["lib"] = lib
        st["pools"] = lib.page_pools([*st["k"], *st["v"]])
        st["ws"] = torch.empty(lib.octopus_pages_workspace(n_pages, n_seq, per), dtype=torch.uint8, device=DEV)
    return st


def _prepare_verify(c, seed):
    n_seq, n, vocab = c["n_seq"], c["n_draft"], c["vocab"]
    st = {"target": torch.empty((n_seq, n + 1, vocab), dtype=_dtype(c), device=DEV),
          "draft": torch.empty((n_seq, n, vocab), dtype=_dtype(c), device=DEV) if c["sampled"] else None,
          "x": torch.empty((n_seq, n), dtype=torch.int32, device=DEV)}
    most = max(1, (1 << 25) // ((n + 1) * vocab))
    for at in range(0, n_seq, most):
        some = slice(at, min(at + most, n_seq))
        logits = 3.0 * torch.randn((some.stop - at, n + 1, vocab), generator=_gen(seed, 7, at), device=DEV)
        logits[..., ::509] += 6.0                          # a few likely tokens, a long tail
        st["target"][some] = torch.softmax(logits, -1)
        logits = logits[:, :n] + c["agree"] * torch.randn(logits[:, :n].shape, generator=_gen(seed, 8, at), device=DEV)
        if c["sampled"]:
            st["draft"][some] = torch.softmax(logits, -1)
        noise = torch.rand(logits.shape, generator=_gen(seed, 9, at), device=DEV).clamp_min(1e-20).log().neg_().log_().neg_()
        st["x"][some] = (logits + noise).argmax(-1) if c["sampled"] else logits.argmax(-1)
    st["x_lens"] = _ints(_some(c, seed, 311, 0, n, n_seq))
    st["u"] = torch.rand((n_seq, n + 1), generator=_gen(seed, 10), device=DEV)
    st["tokens"] = torch.zeros((n_seq, n + 1), dtype=torch.int32, device=DEV)
    st["accepted"] = torch.zeros(n_seq, dtype=torch.int32, device=DEV)
    if own:
        from paper_2605_21226_amd import binding as lib
        st["lib"] = lib
        st["ws"] = torch.empty(lib.octopus_verify_workspace(n_seq, n, vocab), dtype=torch.uint8, device=DEV)
    return st


_PREPARE = {"axes": _prepare_axes, "fork": _prepare_pages, "turnover": _prepare_pages, "verify": _prepare_verify}


def prepare(case, seed):
    c = dict(case)
    return dict(_PREPARE[c["op"]](c, seed), c=c)


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(st):
    return (_OWN if own else _PLAIN)[st["c"]["op"]](st)


def _own_axes(st):
    c, lib = st["c"], st["lib"]
    lib.octopus_append_paged_axes(st["cb"], st["k"], st["v"], st["signs"], st["k_pool"], st["v_pool"], st["n_pages"], st["table"],
                                  st["rope"], st["axis"], st["pos"].permute(1, 2, 0), start_pos=st["start"], new_lens=st["new_lens"],
                                  rope_interleaved=c["interleaved"], q=st["q"], q_out=st["q_out"])
    lib.octopus_read_paged(st["cb"], st["signs"], st["k_pool"], st["v_pool"], st["n_pages"], st["table"], st["k_out"], st["v_out"],
                           start_pos=st["start"], lens=st["new_lens"])
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


def _own_fork(st):
    lib = st["lib"]
    lib.octopus_pages_update(st["refs"], st["table"], st["lens"], st["new_lens"], st["moves"], st["ws"], source=st["source"],
                             keep_lens=st["keep"])
    lib.octopus_pages_copy(st["pools"], st["moves"])
    return _held(st)


def _own_turnover(st):
    lib, n = st["lib"], st["c"]["retire"]
    left, none = st["lens"][:n].clone(), st["lens"].new_zeros(n)
    lib.octopus_pages_update(st["refs"], st["table"], st["lens"], torch.cat([st["lens"][n:], none]), st["moves"], st["ws"],
                             source=_shifted(st))
    lib.octopus_pages_compact(st["refs"], st["map"], st["moves"], st["ws"])
    lib.octopus_pages_copy(st["pools"], st["moves"])
    lib.octopus_pages_rename(st["map"], st["table"], st["lens"])
    found = dict(_held(st), compacted=st["moves"].clone())
    lib.octopus_pages_update(st["refs"], st["table"], st["lens"], torch.cat([st["lens"][:-n], left]), st["moves"], st["ws"])
    return found


def _own_verify(st):
    st["lib"].octopus_verify_drafts(st["target"], st["draft"], st["x"], st["u"], st["tokens"], st["accepted"], st["ws"],
                                    draft_lens=st["x_lens"])
    return {"tokens": st["tokens"], "accepted": st["accepted"]}


_OWN = {"axes": _own_axes, "fork": _own_fork, "turnover": _own_turnover, "verify": _own_verify}


def _held(st):
    return {name: st[name] for name in ("table", "lens", "refs", "moves", "map", "k", "v")}


def _shifted(st):
    """The sequences that stay, from the first slot on; then empty slots."""
    s = torch.arange(st["c"]["n_seq"], dtype=torch.int32, device=DEV) + st["c"]["retire"]
    return torch.where(s < st["c"]["n_seq"], s, -1)


# the plain form: elementary torch operations, in 32 bits but for sums and borders of probabilities
def _hadamard(d):
    i = torch.arange(d, device=DEV)
    bits = i[:, None] & i[None, :]
    bits = bits ^ (bits >> 4)
    bits = bits ^ (bits >> 2)
    bits = bits ^ (bits >> 1)
    return (1.0 - 2.0 * (bits & 1).float()) / math.sqrt(d)


def _oct(xi, eta):
    """Oct^-1: points of the square to unit vectors, [..., 3]"""
    r = 1 - xi.abs() - eta.abs()
    a = torch.where(r < 0, torch.where(xi >= 0, 1 - eta.abs(), eta.abs() - 1), xi)
    b = torch.where(r < 0, torch.where(eta >= 0, 1 - xi.abs(), xi.abs() - 1), eta)
    v = torch.stack([a, b, r], dim=-1)
    return v / v.norm(dim=-1, keepdim=True)


def _device_books(c):
    """Per class: centroids, their midpoints, and the unit vector of every pair of direction codes."""
    books = []
    for _, _, bd, bn in _classes(c):
        x, r = torch.from_numpy(_book_xi(bd)).to(DEV), torch.from_numpy(_book_rho(c["d"], bn)).to(DEV)
        books.append((x, 0.5 * (x[1:] + x[:-1]), r, 0.5 * (r[1:] + r[:-1]), _oct(x[:, None], x[None, :])))
    return books


def _through_codes(st, keys):
    """The keys that the codes of keys [..., n_kv, d] define (Alg. 1 and its inverse)."""
    c = st["c"]
    gamma = keys.square().sum(-1, keepdim=True).sqrt()
    u = ((keys / gamma.clamp_min(1e-20)) * st["sign"]) @ st["had"]
    n_tri = (c["d"] + 2) // 3
    t = torch.nn.functional.pad(u, (0, 3 * n_tri - c["d"])).unflatten(-1, (n_tri, 3))
    near = torch.arange(9, device=DEV)
    parts = []
    for (first, n, _, _), (x, mid, r, rho_mid, unit) in zip(_classes(c), st["books"]):
        w = t[..., first:first + n, :]
        p = w / w.abs().sum(-1, keepdim=True).clamp_min(1e-20)
        flat, fold = p[..., :2], 1 - p[..., :2].abs().flip(-1)
        flat = torch.where(p[..., 2:] < 0, torch.where(flat >= 0, fold, -fold), flat)
        j = torch.searchsorted(mid, flat.contiguous())
        jx = (j[..., :1] + torch.div(near, 3, rounding_mode="floor") - 1).clamp(0, len(x) - 1)
        jy = (j[..., 1:] + near % 3 - 1).clamp(0, len(x) - 1)
        best, at = (unit[jx, jy] * w[..., None, :]).sum(-1).max(-1, keepdim=True)
        rho = r[torch.searchsorted(rho_mid, best[..., 0].clamp(0, 1).contiguous())]
        parts.append(rho[..., None] * unit[jx.gather(-1, at)[..., 0], jy.gather(-1, at)[..., 0]])
    back = torch.cat(parts, dim=-2).flatten(-2)[..., :c["d"]] * gamma
    return (back @ st["had"]) * st["sign"]


def _rotate(c, x, cs):
    """x [..., heads, d] by (cos, sin) pairs cs [..., 1, rot / 2, 2]"""
    x = x.float()
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    y = a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]
    y = torch.stack(y, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(y, dim=-1)
    return torch.cat([y, x[..., r:]], dim=-1)


def _plain_axes(st):
    c = st["c"]
    i = torch.arange(c["n_new"], device=DEV)
    slot = st["start"][:, None] + i
    live = i < st["new_lens"][:, None]
    axis = torch.frombuffer(bytearray(st["axis"]), dtype=torch.uint8).to(DEV).long()
    cs = st["rope"][st["pos"][axis].movedim(0, -1).long(), torch.arange(c["rot"] // 2, device=DEV)][:, :, None]
    keep = live[:, :, None, None]
    k = torch.where(keep, _through_codes(st, _rotate(c, st["k"], cs)), 0.0)
    page = st["table"].gather(1, torch.div(slot, TILE, rounding_mode="floor").long())[live].long()
    st["v_pool"][page, :, (slot % TILE)[live].long()] = st["v"].bfloat16()[live]
    return {"q": torch.where(keep, _rotate(c, st["q"], cs), 0.0).to(_dtype(c)), "k": k.bfloat16(),
            "v": torch.where(keep, st["v"].float(), 0.0).bfloat16()}


def _ceil(x):
    return torch.div(x + (TILE - 1), TILE, rounding_mode="floor")


def _add(refs, ids, what):
    refs.scatter_add_(0, ids.reshape(-1).long(), what.reshape(-1).int())


def _plain_update(st, new_lens, source=None, keep=None):
    refs, table, lens = st["refs"], st["table"], st["lens"]
    n_seq, per = table.shape
    slot, j = torch.arange(n_seq, device=DEV), torch.arange(per, device=DEV)
    source = slot if source is None else source.long()
    from_row = source.clamp(0, n_seq - 1)
    have = torch.where((source >= 0) & (source < n_seq), lens[from_row], 0)
    want = new_lens.clamp(0, per * TILE)
    kept = torch.minimum(have, want) if keep is None else torch.minimum(torch.minimum(have, want), keep)
    rows = table[from_row]
    _add(refs, table, -(j < _ceil(lens)[:, None]).int())
    _add(refs, rows, j < _ceil(kept)[:, None])
    # pages that are written into: all but one of those that would write into a page take a copy, and that one too if others read it
    writes = (want > kept) & (kept % TILE != 0)
    at = torch.div(kept, TILE, rounding_mode="floor").clamp(max=per - 1).long()
    page = rows.gather(1, at[:, None])[:, 0].long()
    writers = torch.zeros_like(refs)
    _add(writers, page, writes)
    rank = torch.where(source == slot, slot, n_seq + slot)
    first = torch.full_like(refs, 2 * n_seq).long()
    first.scatter_reduce_(0, page, torch.where(writes, rank, 2 * n_seq), "amin")
    copies = writes & ((refs[page] > writers[page]) | (first[page] != rank))
    need = _ceil(want) - _ceil(kept) + copies
    end = need.cumsum(0)
    free = refs <= 0
    missing = (end[-1] - free.sum()).clamp(min=0)
    enough = missing == 0
    copies, need = copies & enough, torch.where(enough, need, 0)
    begin = need.cumsum(0) - need
    order = free.cumsum(0) - 1
    fresh = torch.zeros_like(refs)
    fresh[torch.where(free, order, refs.numel() - 1)] = torch.where(free, torch.arange(refs.numel(), device=DEV, dtype=torch.int32), 0)
    refs.copy_(torch.where(free & (order < need.sum()), 1, refs))
    _add(refs, page, -copies.int())
    held = torch.where(enough, want, kept)
    nth = begin[:, None] + torch.where(copies[:, None] & (j == at[:, None]), 0, copies[:, None] + j - _ceil(kept)[:, None])
    new = (j >= _ceil(kept)[:, None]) | (copies[:, None] & (j == at[:, None]))
    rows = torch.where(new, fresh[nth.clamp(0, refs.numel() - 1).long()], rows)
    moves = st["moves"]
    pairs = torch.stack([page, fresh[begin.clamp(max=refs.numel() - 1).long()].long()], dim=1)[copies]
    moves[0], moves[1] = copies.sum(), missing
    moves[2:2 + 2 * len(pairs)] = pairs.reshape(-1)
    table.copy_(torch.where(j < _ceil(held)[:, None], rows, table))
    lens.copy_(held)


def _plain_copy(st):
    n = int(st["moves"][0])
    pairs = st["moves"][2:2 + 2 * n].view(n, 2).long()
    st["k"][:, pairs[:, 1]] = st["k"][:, pairs[:, 0]]
    st["v"][:, pairs[:, 1]] = st["v"][:, pairs[:, 0]]


def _plain_fork(st):
    _plain_update(st, st["new_lens"], st["source"], st["keep"])
    _plain_copy(st)
    return _held(st)


def _plain_turnover(st):
    n, refs, moves = st["c"]["retire"], st["refs"], st["moves"]
    left, none = st["lens"][:n].clone(), st["lens"].new_zeros(n)
    _plain_update(st, torch.cat([st["lens"][n:], none]), _shifted(st))
    # the highest page in use to the lowest free one, and so on
    used, i = refs > 0, torch.arange(refs.numel(), device=DEV)
    n_used = used.sum()
    high, low = (used & (i >= n_used)).nonzero()[:, 0].flip(0), (~used & (i < n_used)).nonzero()[:, 0]
    moves[0], moves[1] = len(high), n_used
    moves[2:2 + 2 * len(high)] = torch.stack([high, low], dim=1).reshape(-1)
    st["map"].copy_(i)
    st["map"][high] = low.int()
    refs[low] = refs[high]
    refs[high] = 0
    _plain_copy(st)
    held = torch.arange(st["table"].shape[1], device=DEV) < _ceil(st["lens"])[:, None]
    st["table"].copy_(torch.where(held, st["map"][st["table"].long()], st["table"]))
    found = dict(_held(st), compacted=moves.clone())
    _plain_update(st, torch.cat([st["lens"][:-n], left]))
    return found


def _plain_verify(st):
    n_seq, n, vocab = st["target"].shape[0], st["x"].shape[1], st["target"].shape[2]
    x, u, i = st["x"].long(), st["u"].double(), torch.arange(n, device=DEV)
    p = st["target"][:, :n].gather(2, x[:, :, None])[:, :, 0].double()
    q = st["draft"].gather(2, x[:, :, None])[:, :, 0].double() if st["draft"] is not None else torch.ones_like(p)
    taken = (u[:, :n] * q < p) & (i < st["x_lens"][:, None])
    a = taken.int().cumprod(1).sum(1)
    s, at = torch.arange(n_seq, device=DEV), a.clamp(max=n - 1)
    refused = (a < st["x_lens"])[:, None]
    whole = st["target"][s, a].double()
    if st["draft"] is not None:
        less = st["draft"][s, at].double()
    else:
        less = torch.where(torch.arange(vocab, device=DEV) == x.gather(1, at[:, None]), math.inf, 0.0)
    rest = (whole - torch.where(refused, less, 0.0)).clamp_min(0.0)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, whole)
    upto = rest.cumsum(1)
    token = ((upto > u[:, n:] * upto[:, -1:]) & (rest > 0)).int().argmax(1)
    i = torch.arange(n + 1, device=DEV)
    tokens = torch.where(i < a[:, None], torch.nn.functional.pad(x, (0, 1)), torch.where(i == a[:, None], token[:, None], -1))
    return {"tokens": tokens.int(), "accepted": a.int()}


_PLAIN = {"axes": _plain_axes, "fork": _plain_fork, "turnover": _plain_turnover, "verify": _plain_verify}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    c = dict(case)
    if c["op"] == "verify":
        es = 2 if c["dtype"] == "bf16" else 4
        rows = 2 if c["sampled"] else 1
        return {"bytes": c["n_seq"] * (c["vocab"] * rows * es + c["n_draft"] * (4 + 4 + rows * es) + 4 * (c["n_draft"] + 3)),
                "flops": c["n_seq"] * c["vocab"] * (rows + 2)}
    if c["op"] == "axes":
        d, es, n_kv, heads = c["d"], 2 if c["dtype"] == "bf16" else 4, c["n_kv"], c["n_q_heads"]
        n, n_tri = float(_some(c, 1, 304, 0, c["n_new"], c["n_seq"]).sum()), (d + 2) // 3
        # transform, norm and sign, then per triplet the map, nine candidates of a three-term product, the norm index
        encode = d * math.log2(d) + 3 * d + n_tri * (14 + 54 + 8)
        return {"bytes": n * (n_kv * (2 * d * es + _record(c) + 2 * d + 4 * d) + heads * 2 * d * es + 4 * c["rot"] + 4 * c["n_axes"]),
                "flops": n * (n_kv * encode + (n_kv + heads) * 3 * c["rot"])}
    lens, n_seq = _tokens(c, 1), c["n_seq"]
    pages = -(-lens // TILE)
    if c["op"] == "fork":
        forked = n_seq // c["beams"] * (c["beams"] - c["alive"])
        copied = forked if c["tokens"] % TILE or c["ragged"] else 0
        entries = float(pages.mean()) * forked
    else:
        copied = float(pages.mean()) * c["retire"]
        entries = 3 * float(pages.sum())      # rows that move up, rows that are renamed
    return {"bytes": 2.0 * copied * c["layers"] * _page_bytes(c) + 16.0 * entries + 32 * n_seq, "flops": 0}


# ---- the same in 64 bits, from the definitions -----------------------------------------------------------------------------
def _matrix(d):
    """The Hadamard matrix by doubling."""
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    while h.shape[0] < d:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / math.sqrt(d)


def _direction(x, y):
    z = 1 - abs(x) - abs(y)
    if z < 0:
        x, y = math.copysign(1 - abs(y), x), math.copysign(1 - abs(x), y)
    n = math.sqrt(x * x + y * y + z * z)
    return [x / n, y / n, z / n]


def _exact_keys(c, books, had, sign, k):
    gamma = torch.linalg.vector_norm(k, dim=-1)
    u = (k * sign / gamma.clamp_min(1e-20).unsqueeze(-1)) @ had
    n_tri = (c["d"] + 2) // 3
    full = torch.zeros(u.shape[:-1] + (3 * n_tri,), dtype=torch.float64, device=DEV)
    full[..., :c["d"]] = u
    found = []
    for (first, n, _, _), (cx, cr, units) in zip(_classes(c), books):
        x, y, z = (full[..., 3 * first + a:3 * (first + n):3] for a in range(3))
        l1 = (x.abs() + y.abs() + z.abs()).clamp_min(1e-20)
        up = lambda a: torch.where(a >= 0, 1.0, -1.0)  # noqa: E731
        px, py = x / l1, y / l1
        xi = torch.where(z >= 0, px, up(px) * (1 - py.abs()))
        eta = torch.where(z >= 0, py, up(py) * (1 - px.abs()))
        between = (cx[1:] + cx[:-1]) / 2
        sx, sy = ((v.unsqueeze(-1) > between).sum(-1) for v in (xi, eta))
        best, bx, by = torch.full_like(x, -math.inf), torch.zeros_like(sx), torch.zeros_like(sx)
        for a in (-1, 0, 1):
            for b in (-1, 0, 1):
                jx, jy = (sx + a).clamp(0, len(cx) - 1), (sy + b).clamp(0, len(cx) - 1)
                nx, ny, nz = units[jx, jy].unbind(-1)
                s = x * nx + y * ny + z * nz
                win = s > best
                best, bx, by = torch.where(win, s, best), torch.where(win, jx, bx), torch.where(win, jy, by)
        r = cr[(best.clamp(0, 1).unsqueeze(-1) > (cr[1:] + cr[:-1]) / 2).sum(-1)]
        found.append(r.unsqueeze(-1) * units[bx, by])
    u = torch.cat(found, dim=-2).reshape(gamma.shape + (-1,))[..., :c["d"]]
    return gamma.unsqueeze(-1) * (u @ had) * sign


def _exact_turn(c, x, turn):
    """Each pair as a complex number, times its position's."""
    r = c["rot"]
    y = x.double().clone()
    if c["interleaved"]:
        y[..., :r] = torch.view_as_real(torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn).flatten(-2)
    else:
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def _exact_axes(c, st):
    n_seq, n_new, n_kv, d = c["n_seq"], c["n_new"], c["n_kv"], c["d"]
    books, had, sign = [], _matrix(d), st["sign"].double()
    for _, _, bd, bn in _classes(c):
        x, r = _book_xi(bd).astype(np.float64), _book_rho(d, bn).astype(np.float64)
        units = torch.tensor([[_direction(a, b) for b in x] for a in x], dtype=torch.float64, device=DEV)
        books.append((torch.from_numpy(x).to(DEV), torch.from_numpy(r).to(DEV), units))
    zeros = lambda heads: torch.zeros((n_seq, n_new, heads, d), dtype=torch.float64, device=DEV)  # noqa: E731
    found = {"q": zeros(c["n_q_heads"]), "k": zeros(n_kv), "v": zeros(n_kv)}
    table = torch.view_as_complex(st["rope"].double().contiguous())
    for s in range(n_seq):
        for lo in range(0, int(st["new_lens"][s]), 2048):
            part = slice(lo, min(lo + 2048, int(st["new_lens"][s])))
            turn = torch.stack([table[st["pos"][a, s, part].long(), i] for i, a in enumerate(st["axis"])], dim=-1).unsqueeze(1)
            found["q"][s, part] = _exact_turn(c, st["q"][s, part], turn)
            found["k"][s, part] = _exact_keys(c, books, had, sign, _exact_turn(c, st["k"][s, part], turn))
            found["v"][s, part] = st["v"][s, part].double()
    return found


def _exact_verify(c, st):
    n = c["n_draft"]
    tokens, accepted = torch.full((c["n_seq"], n + 1), -1, dtype=torch.int32), torch.zeros(c["n_seq"], dtype=torch.int32)
    for s in range(c["n_seq"]):
        x, u = [int(t) for t in st["x"][s][:int(st["x_lens"][s])]], [float(v) for v in st["u"][s]]
        a = 0
        for t in x:
            q = float(st["draft"][s, a, t]) if c["sampled"] else 1.0
            if u[a] * q >= float(st["target"][s, a, t]):
                break
            tokens[s, a] = t
            a += 1
        p = st["target"][s, a].cpu().numpy() if c["dtype"] == "fp32" else st["target"][s, a].float().cpu().numpy()
        rest = p.astype(np.float64)
        if a < len(x) and c["sampled"]:
            rest = np.maximum(rest - st["draft"][s, a].float().cpu().numpy().astype(np.float64), 0.0)
        elif a < len(x):
            rest[x[a]] = 0.0
        if not rest.any():
            rest = p.astype(np.float64)
        at = np.nonzero(rest)[0]
        upto = np.cumsum(rest[at].astype(np.longdouble))
        tokens[s, a] = int(at[min(int(np.searchsorted(upto, u[n] * upto[-1], side="right")), len(at) - 1)])
        accepted[s] = a
    return {"tokens": tokens, "accepted": accepted}


def exact(case, seed):
    """None where a pass moves whole numbers and bytes about."""
    c = dict(case)
    if c["op"] in ("fork", "turnover"):
        return None
    return {"axes": _exact_axes, "verify": _exact_verify}[c["op"]](c, prepare(case, seed))

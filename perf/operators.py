"""Operators of a server over pages of compressed keys, as measured cases.

  append   a step's new keys, values and queries as the projection leaves them: keys and queries rotated by position,
           keys encoded into pages, values written (or quantised) into pages; then what the pages hold is read back
  read     tokens of a paged cache as values again
  prefix   attention of sequences that share a long prefix: its pages once for all, each sequence's own pages by itself

Sizes are those of this repository's workloads (32 query and 8 KV heads of 128, 24 heads of 64, 16 and 8 heads of 256)
where one fits, else generic serving sizes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TILE = 64
BASE = 500000.0      # of the rotation's angles


def _case(name, op, n_seq, n_q_heads, n_kv, d, bits, **more):
    c = {"op": op, "n_seq": n_seq, "n_q_heads": n_q_heads, "n_kv": n_kv, "d": d, "bits": bits, "dtype": "bf16", "n_new": 1,
         "start": 0, "ragged": False, "rot": d, "interleaved": False, "v_bits": 0, "v_group": 0, "prefix": 0, "own": 0,
         "causal": False}
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's chat: the token that a step appends, one launch and next to no data
        _case("append_token", "append", 1, 32, 8, 128, 3.0, start=1000),
        # a server's batch in its ordinary step: a token per sequence at ragged positions
        _case("append_batch", "append", 64, 32, 8, 128, 3.0, start=8000, ragged=True),
        # a padded batch of fp32 prompts at 24 heads of 64, half the channels rotated, as neighbouring pairs
        _case("append_padded_fp32", "append", 3, 24, 24, 64, 4.0, dtype="fp32", n_new=509, ragged=True, rot=32, interleaved=True),
        # the prompt of the Llama-shaped workload's prefill in one call
        _case("append_prompt", "append", 1, 32, 8, 128, 3.0, n_new=15877),
        # two prompts whose values are quantised as well
        _case("append_quantised", "append", 2, 32, 8, 128, 3.0, n_new=3001, start=75, v_bits=3, v_group=32),
        # a cached prompt as values, to be moved to another width
        _case("read_prompt", "read", 1, 32, 8, 128, 3.0, n_new=15877),
        # ragged tails of five sequences, fp32, a two-class bit width at head dimension 256, quantised values
        _case("read_ragged_d256", "read", 5, 16, 8, 256, 2.5, dtype="fp32", n_new=777, start=1100, ragged=True, v_bits=4, v_group=16),
        # beam search: four beams of a short prompt
        _case("beams", "prefix", 4, 32, 8, 128, 3.0, prefix=700, own=60),
        # a server's batch behind one system prompt, contexts of their own of all lengths
        _case("system_prompt", "prefix", 64, 32, 8, 128, 3.0, prefix=8192, own=1500, ragged=True),
        # many samples of one long document
        _case("long_prefix", "prefix", 16, 32, 8, 128, 3.0, prefix=65531, own=512),
        # drafts of five tokens verified at once, a padded batch, 24 heads of 64 at 4 bits
        _case("draft_check", "prefix", 8, 24, 24, 64, 4.0, prefix=3600, own=333, n_new=5, causal=True, ragged=True),
        # head dimension 256, two bit widths to a key
        _case("prefix_d256", "prefix", 32, 16, 8, 256, 2.5, prefix=16384, own=200, ragged=True),
    ]


def _log_uniform(rng, lo, hi):
    lo = min(lo, max(1, hi))
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "prefix", "prefix", "prefix"])
    d = rng.choice([64, 128, 128, 256])
    bits = rng.choice([1.0, 1.5, 2.0, 2.5, 3.0, 3.0, 4.0])
    n_kv = rng.choice([1, 2, 4, 8, 8])
    heads = n_kv * rng.choice([1, 2, 3, 4, 4, 8])
    more = {"dtype": "fp32" if rng.random() < 0.25 else "bf16"}
    if op == "prefix":
        n_seq = _log_uniform(rng, 1, 64)
        n_new = rng.choice([1, 1, 1, 2, 5, 17, 70])
        rows = n_seq * n_new * heads
        prefix = _log_uniform(rng, 60, min(65531, 4000000000 // (rows * d), 65531 * 8 * 128 // (n_kv * d)))
        room = min(3000, 800000 // (n_seq * n_kv), 2000000000 // (rows * d))
        return _case(None, op, n_seq, heads, n_kv, d, bits, n_new=n_new, prefix=prefix, own=n_new + _log_uniform(rng, 1, max(1, room)),
                     causal=n_new > 1 or rng.random() < 0.5, ragged=rng.random() < 0.6, **more)
    n_seq = rng.choice([1, 1, 2, 3, 8, 33, 64])
    most = 15877 * 8 * 128 // (n_seq * n_kv * d)
    n_new = 1 if rng.random() < 0.3 else _log_uniform(rng, 1, max(1, most // 2))
    if bits in (2.0, 3.0, 4.0) and rng.random() < 0.4:
        more.update(v_bits=int(bits), v_group=rng.choice([16, 32]))
    more.update(rot=rng.choice([d, d, d // 2, 16]), interleaved=rng.random() < 0.3)
    return _case(None, op, n_seq, heads, n_kv, d, bits, n_new=n_new, start=rng.choice([0, _log_uniform(rng, 1, 8000)]),
                 ragged=rng.random() < 0.6, **more)


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


def _streams(c):
    """[(kind, class, indices, bits, first byte)] of a record, in its order"""
    cl = _classes(c)
    at, found = 4, []
    for kind, per, col in (("dir", 2, 2), ("nrm", 1, 3)):
        for k, x in enumerate(cl):
            found.append((kind, k, per * x[1], x[col], at))
            at += _stream(per * x[1], x[col])
    return found, at


def _granules(c):
    return (_streams(c)[1] + 15) // 16


def _vrow(c):
    return c["v_bits"] * c["d"] // 8 + c["d"] // c["v_group"] * 8 if c["v_bits"] else 2 * c["d"]


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


def _some(c, seed, stream, lo, hi):
    """A number per sequence: hi, or anything in [lo, hi] with hi among them."""
    n = np.full(c["n_seq"], hi, dtype=np.int32)
    if c["ragged"] and hi > lo:
        r = np.random.default_rng([int(seed), stream])
        n = r.integers(lo, hi + 1, size=c["n_seq"]).astype(np.int32)
        n[int(r.integers(0, c["n_seq"]))] = hi
    return n


def _channel_scales(c, seed):
    """Per-channel key scales of real decoders: log-normal, four channels of a head ten times as large."""
    r = np.random.default_rng([int(seed), 202])
    sig = np.exp(0.5 * r.standard_normal((c["n_kv"], c["d"])))
    for h in range(c["n_kv"]):
        sig[h, r.choice(c["d"], size=4, replace=False)] *= 10.0
    return torch.from_numpy(sig.astype(np.float32)).to(DEV)


def _signs(c, seed):
    r = np.random.default_rng([int(seed), 101])
    return r.integers(0, 2, size=(c["n_kv"], c["d"])).astype(np.int8) * 2 - 1


def _table(n_pages, shape, seed, stream):
    r = np.random.default_rng([int(seed), stream])
    return torch.from_numpy(r.permutation(n_pages).astype(np.int32).reshape(shape)).to(DEV)


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def prepare(case, seed):
    c = dict(case)
    n_seq, n_kv, d, n_new = c["n_seq"], c["n_kv"], c["d"], c["n_new"]
    st = {"c": c, "books": _device_books(c), "had": _hadamard(d, torch.float32)}
    s = _signs(c, seed)
    st["sign"] = torch.from_numpy(s).to(DEV).float()
    st["signs"] = torch.from_numpy(np.packbits((s < 0).astype(np.uint8), axis=-1, bitorder="little")).to(DEV)
    sig = _channel_scales(c, seed)
    if c["op"] == "append":
        start = _some(c, seed, 303, 0, c["start"])
        st["new_lens"] = _ints(_some(c, seed, 304, 0, n_new))
        st["start"] = _ints(start)
        per = (int(start.max()) + n_new + TILE - 1) // TILE
        # one projection's output: queries, keys and values of a token side by side
        qkv = torch.randn((n_seq, n_new, c["n_q_heads"] + 2 * n_kv, d), generator=_gen(seed, 3), device=DEV)
        qkv[:, :, c["n_q_heads"]:c["n_q_heads"] + n_kv].mul_(sig)
        qkv = qkv.to(_dtype(c))
        st["q"], st["k"], st["v"] = qkv.split([c["n_q_heads"], n_kv, n_kv], dim=2)
        i = torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64)
        angle = torch.arange(per * TILE, device=DEV, dtype=torch.float64)[:, None] * BASE ** (-2.0 * i / c["rot"])
        st["rope"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
        st["q_out"] = torch.zeros((n_seq, n_new, c["n_q_heads"], d), dtype=_dtype(c), device=DEV)
    else:
        tokens = n_new if c["op"] == "read" else c["own"]
        if c["op"] == "read":
            st["start"] = _ints(_some(c, seed, 303, 0, c["start"]))
            lens = _some(c, seed, 304, 1, n_new)
            tokens = int(st["start"].max()) + n_new
            st["lens"] = _ints(lens)
        per = (tokens + TILE - 1) // TILE
    shared = (c["prefix"] + TILE - 1) // TILE
    st["n_pages"] = n_seq * per + shared
    table = _table(st["n_pages"], (-1,), seed, 707)
    st["prefix_table"], st["table"] = table[:shared].contiguous(), table[shared:].reshape(n_seq, per).contiguous()
    st["k_pool"] = torch.zeros((st["n_pages"], n_kv, _granules(c), TILE, 16), dtype=torch.uint8, device=DEV)
    if c["v_bits"]:
        st["v_pool"] = torch.zeros((st["n_pages"], n_kv, TILE, _vrow(c)), dtype=torch.uint8, device=DEV)
    else:
        st["v_pool"] = torch.zeros((st["n_pages"], n_kv, TILE, d), dtype=torch.bfloat16, device=DEV)
    if c["op"] != "append":      # the pages as earlier steps left them
        most = max(1, (1 << 17) // (n_kv * TILE))
        for at in range(0, st["n_pages"], most):
            pages = torch.arange(at, min(at + most, st["n_pages"]), device=DEV)
            tok = pages.repeat_interleave(TILE)
            off = torch.arange(TILE, device=DEV).repeat(len(pages))
            keys = torch.randn((len(tok), n_kv, d), generator=_gen(seed, 5, at), device=DEV).mul_(sig)
            st["k_pool"][tok, :, :, off] = _pack(c, *_encode(st, keys)).view(len(tok), n_kv, -1, 16)
            v = torch.randn((len(tok), n_kv, d), generator=_gen(seed, 6, at), device=DEV)
            st["v_pool"][tok, :, off] = _pack_values(c, *_quantise(c, v)) if c["v_bits"] else v.bfloat16()
    if c["op"] == "read":
        st["k_out"] = torch.zeros((n_seq, n_new, n_kv, d), dtype=_dtype(c), device=DEV)
        st["v_out"] = torch.zeros_like(st["k_out"])
    if c["op"] == "prefix":
        st["q"] = torch.randn((n_seq, n_new, c["n_q_heads"], d), generator=_gen(seed, 7), device=DEV).to(_dtype(c))
        q_lens = _some(c, seed, 305, 1, n_new)
        own_lens = np.maximum(_some(c, seed, 306, 1, c["own"]), q_lens if c["causal"] else 0)
        st["q_lens"], st["lens"], st["prefix"] = _ints(q_lens), _ints(own_lens), _ints([c["prefix"]])
        st["out"] = torch.zeros((n_seq, n_new, c["n_q_heads"], d), dtype=torch.float32, device=DEV)
    if own:      # the handle and the workspace of the library
        from paper_2605_21226_amd import binding as lib
        st["lib"], st["cb"] = lib, lib.octopus_build_codebooks(d, c["bits"])
        if c["op"] == "prefix":
            st["ws"] = torch.empty(lib.octopus_attn_prefix_workspace(st["cb"], n_seq, c["n_q_heads"], n_kv, n_new, c["prefix"],
                                                                     c["own"]), dtype=torch.uint8, device=DEV)
        if c["op"] == "append":
            st["k_out"] = torch.zeros((n_seq, n_new, n_kv, d), dtype=torch.bfloat16, device=DEV)
            st["v_out"] = torch.zeros_like(st["k_out"])
    return st


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _PLAIN[st["c"]["op"]](st)


def _run_own(st):
    c, lib, cb = st["c"], st["lib"], st["cb"]
    if c["op"] == "append":
        lib.octopus_append_paged(cb, st["k"], st["v"], st["signs"], st["k_pool"], st["v_pool"], st["n_pages"], st["table"],
                                 start_pos=st["start"], new_lens=st["new_lens"], rope=st["rope"],
                                 rope_interleaved=c["interleaved"], q=st["q"], q_out=st["q_out"], v_bits=c["v_bits"],
                                 v_group=c["v_group"])
        lib.octopus_read_paged(cb, st["signs"], st["k_pool"], st["v_pool"], st["n_pages"], st["table"], st["k_out"], st["v_out"],
                               start_pos=st["start"], lens=st["new_lens"], v_bits=c["v_bits"], v_group=c["v_group"])
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    if c["op"] == "read":
        lib.octopus_read_paged(cb, st["signs"], st["k_pool"], st["v_pool"], st["n_pages"], st["table"], st["k_out"], st["v_out"],
                               start_pos=st["start"], lens=st["lens"], v_bits=c["v_bits"], v_group=c["v_group"])
        return {"k": st["k_out"], "v": st["v_out"]}
    lib.octopus_attn_decode_paged_prefix(cb, st["q"], st["signs"], st["k_pool"], st["v_pool"], st["prefix_table"], st["prefix"],
                                         c["prefix"], st["table"], st["lens"], c["own"], 1.0 / math.sqrt(c["d"]), st["out"],
                                         st["ws"], q_lens=st["q_lens"], causal=c["causal"])
    return {"out": st["out"]}


# the plain form: elementary torch operations in 32 bits
def _hadamard(d, dtype):
    i = torch.arange(d, device=DEV)
    bits = i[:, None] & i[None, :]
    for k in (1, 2, 4):
        bits = bits ^ (bits >> k)
    return (1.0 - 2.0 * (bits & 1).to(dtype)) / math.sqrt(d)


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


def _encode(st, keys):
    """Alg. 1 on keys [..., n_kv, d]: norms, and per class the direction codes [..., triplets, 2] and the norm codes."""
    c = st["c"]
    k = keys.float()
    gamma = k.square().sum(-1).sqrt()
    u = ((k / gamma.clamp_min(1e-20)[..., None]) * st["sign"]) @ st["had"]
    n_tri = (c["d"] + 2) // 3
    t = torch.nn.functional.pad(u, (0, 3 * n_tri - c["d"])).unflatten(-1, (n_tri, 3))
    near = torch.arange(9, device=DEV)
    codes = []
    for (first, n, bd, _), (x, mid, _, rho_mid, unit) in zip(_classes(c), st["books"]):
        w = t[..., first:first + n, :]
        p = w / w.abs().sum(-1, keepdim=True).clamp_min(1e-20)
        flat, fold = p[..., :2], 1 - p[..., :2].abs().flip(-1)
        flat = torch.where(p[..., 2:] < 0, torch.where(flat >= 0, fold, -fold), flat)
        j = torch.searchsorted(mid, flat.contiguous())
        jx = (j[..., :1] + torch.div(near, 3, rounding_mode="floor") - 1).clamp(0, len(x) - 1)
        jy = (j[..., 1:] + near % 3 - 1).clamp(0, len(x) - 1)
        score = (unit[jx, jy] * w[..., None, :]).sum(-1)
        best, at = score.max(-1, keepdim=True)
        codes.append((torch.cat([jx.gather(-1, at), jy.gather(-1, at)], dim=-1),
                      torch.searchsorted(rho_mid, best[..., 0].clamp(0, 1).contiguous())))
    return gamma, codes


def _decode(st, gamma, codes):
    """gamma u^ in the rotated basis, [..., n_kv, d]"""
    parts = [(r[nrm][..., None] * unit[xy[..., 0], xy[..., 1]]) for (xy, nrm), (_, _, r, _, unit) in zip(codes, st["books"])]
    return torch.cat(parts, dim=-2).flatten(-2)[..., :st["c"]["d"]] * gamma[..., None]


def _back(st, rotated):
    return (rotated @ st["had"]) * st["sign"]


def _to_bytes(codes, bits, n_bytes):
    b = ((codes[..., None] >> torch.arange(bits, device=DEV)) & 1).flatten(-2).to(torch.uint8)
    b = torch.nn.functional.pad(b, (0, 8 * n_bytes - b.shape[-1])).unflatten(-1, (n_bytes, 8))
    return (b << torch.arange(8, device=DEV, dtype=torch.uint8)).sum(-1, dtype=torch.uint8)


def _from_bytes(data, n, bits):
    b = (data[..., None] >> torch.arange(8, device=DEV, dtype=torch.uint8)) & 1
    b = b.flatten(-2)[..., :n * bits].unflatten(-1, (n, bits))
    return (b << torch.arange(bits, device=DEV, dtype=torch.uint8)).sum(-1, dtype=torch.uint8)


def _pack(c, gamma, codes):
    """Records, padded to whole granules: uint8 [..., n_kv, 16 granules]"""
    parts = [gamma.float()[..., None].contiguous().view(torch.uint8)]
    for kind, k, n, b, _ in _streams(c)[0]:
        parts.append(_to_bytes(codes[k][0].flatten(-2) if kind == "dir" else codes[k][1], b, _stream(n, b)))
    rec = torch.cat(parts, dim=-1)
    return torch.nn.functional.pad(rec, (0, 16 * _granules(c) - rec.shape[-1]))


def _unpack(c, rec):
    gamma = rec[..., :4].contiguous().view(torch.float32)[..., 0]
    codes = [[None, None] for _ in _classes(c)]
    for kind, k, n, b, at in _streams(c)[0]:
        x = _from_bytes(rec[..., at:at + _stream(n, b)], n, b).int()
        codes[k][0 if kind == "dir" else 1] = x.unflatten(-1, (-1, 2)) if kind == "dir" else x
    return gamma, codes


def _quantise(c, v):
    g = v.float().unflatten(-1, (-1, c["v_group"]))
    lo, hi = g.amin(-1), g.amax(-1)
    scale = (hi - lo) / torch.full_like(hi, float((1 << c["v_bits"]) - 1))
    code = ((g - lo[..., None]) / torch.where(scale > 0, scale, 1.0)[..., None]).round().clamp(0, (1 << c["v_bits"]) - 1)
    return scale, lo, code.int()


def _values_of(scale, lo, code):
    return (lo[..., None] + scale[..., None] * code).flatten(-2)


def _pack_values(c, scale, lo, code):
    meta = torch.stack([scale, lo], dim=-1).flatten(-2).contiguous().view(torch.uint8)
    return torch.cat([_to_bytes(code.flatten(-2), c["v_bits"], c["v_bits"] * c["d"] // 8), meta], dim=-1)


def _unpack_values(c, row):
    n = c["v_bits"] * c["d"] // 8
    meta = row[..., n:].contiguous().view(torch.float32).unflatten(-1, (-1, 2))
    return meta[..., 0], meta[..., 1], _from_bytes(row[..., :n], c["d"], c["v_bits"]).unflatten(-1, (-1, c["v_group"]))


def _rotate(c, x, cs):
    """x [..., heads, d] by (cos, sin) pairs cs [..., 1, rot / 2, 2]"""
    x = x.float()
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    y = a * cs[..., 0] - b * cs[..., 1], a * cs[..., 1] + b * cs[..., 0]
    y = torch.stack(y, dim=-1).flatten(-2) if c["interleaved"] else torch.cat(y, dim=-1)
    return torch.cat([y, x[..., r:]], dim=-1)


def _plain_append(st):
    c = st["c"]
    i = torch.arange(c["n_new"], device=DEV)
    pos = st["start"][:, None] + i
    live = i < st["new_lens"][:, None]
    cs = st["rope"][pos][:, :, None]
    gamma, codes = _encode(st, _rotate(c, st["k"], cs))
    page, off = st["table"].gather(1, torch.div(pos, TILE, rounding_mode="floor").long())[live].long(), (pos % TILE)[live].long()
    st["k_pool"][page, :, :, off] = _pack(c, gamma, codes)[live].unflatten(-1, (-1, 16))
    if c["v_bits"]:
        parts = _quantise(c, st["v"])
        st["v_pool"][page, :, off] = _pack_values(c, *parts)[live]
        v = _values_of(*parts)
    else:
        v = st["v"].bfloat16()
        st["v_pool"][page, :, off] = v[live]
    keep = live[:, :, None, None]
    k = torch.where(keep, _back(st, _decode(st, gamma, codes)), 0.0)
    return {"q": torch.where(keep, _rotate(c, st["q"], cs), 0.0).to(_dtype(c)), "k": k.bfloat16(),
            "v": torch.where(keep, v.float(), 0.0).bfloat16()}


def _plain_read(st):
    c = st["c"]
    i = torch.arange(c["n_new"], device=DEV)
    pos = st["start"][:, None] + i
    page, off = st["table"].gather(1, torch.div(pos, TILE, rounding_mode="floor").long()).long(), (pos % TILE).long()
    k = _back(st, _decode(st, *_unpack(c, st["k_pool"][page, :, :, off].flatten(-2))))
    v = st["v_pool"][page, :, off]
    v = _values_of(*_unpack_values(c, v)) if c["v_bits"] else v.float()
    keep = (i < st["lens"][:, None])[:, :, None, None]
    return {"k": torch.where(keep, k, 0.0).to(_dtype(c)), "v": torch.where(keep, v, 0.0).to(_dtype(c))}


def _pages(st, table):
    """Keys (in the rotated basis) and values of whole pages, [..., n_kv, tokens, d]"""
    rec = st["k_pool"][table.long()].movedim(-4, -5).movedim(-2, -3).flatten(-2)      # [..., n_kv, page, 64, bytes] after the moves
    keys = _decode(st, *_unpack(st["c"], rec.flatten(-3, -2)))
    v = st["v_pool"][table.long()].movedim(-3, -4).flatten(-3, -2)
    return keys, v.float()


def _plain_prefix(st):
    c = st["c"]
    n_seq, n_q, n_kv, d = c["n_seq"], c["n_new"], c["n_kv"], c["d"]
    group = c["n_q_heads"] // n_kv
    q = st["q"].float().unflatten(2, (n_kv, group))                                       # [seq, q, kv, g, d]
    q = (q * st["sign"][:, None]) @ st["had"] * (1.0 / math.sqrt(d))
    k, v = _pages(st, st["prefix_table"])
    k, v = k[:, :c["prefix"]], v[:, :c["prefix"]]
    rows = q.permute(2, 0, 1, 3, 4).reshape(n_kv, -1, d)                                  # [kv, seq q g, d]
    shared = rows @ k.transpose(1, 2).contiguous()
    k_own, v_own = _pages(st, st["table"])                                                # [seq, kv, tokens, d]
    rows = q.permute(0, 2, 1, 3, 4).reshape(n_seq, n_kv, -1, d)                           # [seq, kv, q g, d]
    mine = rows @ k_own.transpose(2, 3).contiguous()
    t, i = torch.arange(k_own.shape[2], device=DEV), torch.arange(n_q, device=DEV).repeat_interleave(group)
    seen = st["lens"][:, None] - (st["q_lens"][:, None] - 1 - i if c["causal"] else 0 * i)    # [seq, q g]
    mine = torch.where(t < seen[:, None, :, None], mine, -math.inf)
    shared = shared.view(n_kv, n_seq, n_q * group, -1).transpose(0, 1)                    # [seq, kv, q g, prefix]
    top = torch.maximum(shared.amax(-1, keepdim=True), mine.amax(-1, keepdim=True))
    a, b = (shared - top).exp(), (mine - top).exp()
    out = (a.transpose(0, 1).reshape(n_kv, n_seq * n_q * group, -1) @ v).view(n_kv, n_seq, -1, d).transpose(0, 1) + b @ v_own
    out = out / (a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True))
    out = out.view(n_seq, n_kv, n_q, group, d).transpose(1, 2).reshape(n_seq, n_q, -1, d)
    return {"out": torch.where((torch.arange(n_q, device=DEV) < st["q_lens"][:, None])[:, :, None, None], out, 0.0)}


_PLAIN = {"append": _plain_append, "read": _plain_read, "prefix": _plain_prefix}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    c = dict(case)
    d, es, n_kv, heads = c["d"], 2 if c["dtype"] == "bf16" else 4, c["n_kv"], c["n_q_heads"]
    rec, vrow = _streams(c)[1], _vrow(c)
    n_tri = (d + 2) // 3
    if c["op"] == "append":
        n = float(_some(c, 1, 304, 0, c["n_new"]).sum())
        # transform, norm and sign, then per triplet the map, nine candidates of a three-term product, the norm index
        encode = d * math.log2(d) + 3 * d + n_tri * (14 + 54 + 8)
        return {"bytes": n * (n_kv * (2 * d * es + rec + vrow + 4 * d) + heads * 2 * d * es + 4 * c["rot"]),
                "flops": n * (n_kv * encode + (n_kv + heads) * 3 * c["rot"])}
    if c["op"] == "read":
        n = float(_some(c, 1, 304, 1, c["n_new"]).sum()) * n_kv
        return {"bytes": n * (rec + vrow + 2 * d * es), "flops": n * (d * math.log2(d) + 5 * d)}
    q = _some(c, 1, 305, 1, c["n_new"]).astype(np.float64)
    mine = np.maximum(_some(c, 1, 306, 1, c["own"]), q if c["causal"] else 0)
    seen = mine - (q - 1) / 2 if c["causal"] else mine
    return {"bytes": (c["prefix"] + mine.sum()) * n_kv * (rec + vrow) + q.sum() * heads * d * (es + 4),
            "flops": float((q * (c["prefix"] + seen)).sum()) * heads * 4 * d}


# ---- the same in 64 bits, from the definitions -----------------------------------------------------------------------------
def _matrix(d):
    """The Hadamard matrix by doubling."""
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    while h.shape[0] < d:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / math.sqrt(d)


def _fields(rec, at, n, b):
    """n fields of b bits of byte strings, the first at byte `at`, lowest bits first."""
    bit = 8 * at + b * torch.arange(n, device=DEV)
    wide = torch.nn.functional.pad(rec, (0, 2)).long()
    byte = torch.div(bit, 8, rounding_mode="floor")
    word = wide[..., byte] + 256 * wide[..., byte + 1]
    return torch.remainder(torch.div(word, 2 ** torch.remainder(bit, 8), rounding_mode="floor"), 1 << b)


def _direction(x, y):
    z = 1 - abs(x) - abs(y)
    if z < 0:
        x, y = math.copysign(1 - abs(y), x), math.copysign(1 - abs(x), y)
    n = math.sqrt(x * x + y * y + z * z)
    return [x / n, y / n, z / n]


def _exact_books(c):
    found = []
    for _, _, bd, bn in _classes(c):
        x, r = _book_xi(bd).astype(np.float64), _book_rho(c["d"], bn).astype(np.float64)
        units = torch.tensor([[_direction(a, b) for b in x] for a in x], dtype=torch.float64, device=DEV)
        found.append((torch.from_numpy(x).to(DEV), torch.from_numpy(r).to(DEV), units))
    return found


def _exact_keys(c, books, had, sign, gamma, parts):
    """Keys from norms and per class (xi, eta, rho) codes."""
    u = []
    for (jx, jy, jr), (_, r, units) in zip(parts, books):
        u.append(r[jr].unsqueeze(-1) * units[jx, jy])
    u = torch.cat(u, dim=-2).reshape(gamma.shape + (-1,))[..., :c["d"]]
    return gamma.unsqueeze(-1) * (u @ had) * sign


def _exact_read(c, books, had, sign, rec):
    gamma = rec[..., :4].contiguous().view(torch.float32).squeeze(-1).double()
    parts = [[None, None, None] for _ in books]
    for kind, k, n, b, at in _streams(c)[0]:
        f = _fields(rec, at, n, b)
        if kind == "dir":
            parts[k][0], parts[k][1] = f[..., 0::2], f[..., 1::2]
        else:
            parts[k][2] = f
    return _exact_keys(c, books, had, sign, gamma, parts)


def _exact_value(c, row):
    n = c["v_bits"] * c["d"] // 8
    meta = row[..., n:].contiguous().view(torch.float32).double()
    code = _fields(row, 0, c["d"], c["v_bits"]).double()
    each = lambda x: x.repeat_interleave(c["v_group"], dim=-1)  # noqa: E731
    return each(meta[..., 1::2]) + each(meta[..., 0::2]) * code


def _exact_encode(c, books, had, sign, k):
    gamma = torch.linalg.vector_norm(k, dim=-1)
    u = (k * sign / gamma.clamp_min(1e-20).unsqueeze(-1)) @ had
    n_tri = (c["d"] + 2) // 3
    full = torch.zeros(u.shape[:-1] + (3 * n_tri,), dtype=torch.float64, device=DEV)
    full[..., :c["d"]] = u
    parts = []
    for (first, n, bd, bn), (cx, cr, units) in zip(_classes(c), books):
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
        parts.append((bx, by, (best.clamp(0, 1).unsqueeze(-1) > (cr[1:] + cr[:-1]) / 2).sum(-1)))
    return gamma, parts


def _exact_turn(c, x, cs):
    """Each pair as a complex number, times the position's."""
    r = c["rot"]
    turn = torch.view_as_complex(cs.double().contiguous())
    y = x.double().clone()
    if c["interleaved"]:
        z = torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def exact(case, seed):
    c = dict(case)
    st = prepare(case, seed)
    n_seq, n_new, n_kv, d, heads = c["n_seq"], c["n_new"], c["n_kv"], c["d"], c["n_q_heads"]
    books, had, sign = _exact_books(c), _matrix(d), st["sign"].double()
    if c["op"] == "append":
        found = {"q": torch.zeros((n_seq, n_new, heads, d), dtype=torch.float64, device=DEV)}
        found["k"] = torch.zeros((n_seq, n_new, n_kv, d), dtype=torch.float64, device=DEV)
        found["v"] = torch.zeros_like(found["k"])
        for s in range(n_seq):
            n, at = int(st["new_lens"][s]), int(st["start"][s])
            cs = st["rope"][at:at + n].unsqueeze(1)
            found["q"][s, :n] = _exact_turn(c, st["q"][s, :n], cs)
            for lo in range(0, n, 2048):
                part = slice(lo, min(lo + 2048, n))
                keys = _exact_turn(c, st["k"][s, part], cs[part])
                found["k"][s, part] = _exact_keys(c, books, had, sign, *_exact_encode(c, books, had, sign, keys))
            v = st["v"][s, :n].double()
            if c["v_bits"]:
                g = v.unflatten(-1, (-1, c["v_group"]))
                lo, hi = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
                # the codec's definition: scale and quotient are fp32 numbers (a quotient next to a half goes by that rounding)
                step = ((hi - lo) / ((1 << c["v_bits"]) - 1)).float().double()
                code = torch.nan_to_num(((g - lo).float().double() / step).float().double()).round()
                v = (lo + step * code).flatten(-2)
            found["v"][s, :n] = v
        return found
    if c["op"] == "read":
        found = {x: torch.zeros((n_seq, n_new, n_kv, d), dtype=torch.float64, device=DEV) for x in ("k", "v")}
        for s in range(n_seq):
            for lo in range(0, int(st["lens"][s]), 4096):
                hi = min(lo + 4096, int(st["lens"][s]))
                pos = int(st["start"][s]) + torch.arange(lo, hi, device=DEV)
                page, off = st["table"][s].long()[pos // TILE], pos % TILE
                rec = st["k_pool"][page, :, :, off].reshape(hi - lo, n_kv, -1)
                found["k"][s, lo:hi] = _exact_read(c, books, had, sign, rec)
                row = st["v_pool"][page, :, off]
                found["v"][s, lo:hi] = _exact_value(c, row) if c["v_bits"] else row.double()
        return found
    group = heads // n_kv
    out = torch.zeros((n_seq, n_new, heads, d), dtype=torch.float64, device=DEV)

    def tokens(pages, h, n):
        rec = st["k_pool"][pages.long(), h].transpose(1, 2).reshape(len(pages) * TILE, -1)[:n]
        return _exact_read(c, books, had, sign[h], rec), st["v_pool"][pages.long(), h].reshape(-1, d)[:n].double()
    for h in range(n_kv):
        k_shared, v_shared = tokens(st["prefix_table"], h, c["prefix"])
        for s in range(n_seq):
            n, m = int(st["q_lens"][s]), int(st["lens"][s])
            k_mine, v_mine = tokens(st["table"][s], h, m)
            q = st["q"][s, :n, h * group:(h + 1) * group].double().reshape(n * group, d)
            score = q @ torch.cat([k_shared, k_mine]).t().contiguous() / math.sqrt(d)
            if c["causal"]:
                last = c["prefix"] + m - n + torch.arange(n, device=DEV).repeat_interleave(group)
                score = score.masked_fill(torch.arange(score.shape[1], device=DEV) > last[:, None], -math.inf)
            out[s, :n, h * group:(h + 1) * group] = (torch.softmax(score, -1) @ torch.cat([v_shared, v_mine])).view(n, group, d)
    return {"out": out}

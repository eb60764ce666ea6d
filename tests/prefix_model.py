"""The arithmetic of the shared-prefix attention on the CPU, with any of its corrections left out: ordinary inputs, their attention in
64 bits, and what the kernel's operands make of it.

Coordinates of keys and queries are two fp16 numbers each, rounded to the nearest; the product of the remainders is left out.  In the
root mean square a term k_i q_i is off by no more than 2^-11 2^-11 / 3 of it for either factor's last bits (a remainder below 2^-11,
rounded by less than 2^-11 of itself, both spread evenly) and as much for the product left out: 2^-22 together, in any direction.
For coordinates of about one, scale sqrt(sum k_i^2 q_i^2) is one and so a score is off by 2^-22. Its fp32 sums round some 30
times, by 2^-25 of sums of two or three: 2^-22 together. Probabilities are three bf16 numbers that make the fp32 one exactly, and
that is an exponential's (2^-23); sums of them round by 2^-23 again. Numerator and denominator take twice the score's part: 2
(2^-22 + 2^-22) + 2 2^-23 < 2^-19 of the output's root mean square, TOLERANCE."""
import numpy as np

import oracle

TOLERANCE = 2.0 ** -19
CASES = [(64, 4), (64, 1.5), (64, 2), (128, 3), (128, 2.5), (128, 4), (128, 1), (256, 2.5), (256, 4), (256, 3)]     # joint tables, two bit widths to a key, none
N_KV, G, PREFIX, OWN = 2, 8, 300, 70


class Inputs:
    """Keys as records [kv, tokens, bytes], values [kv, tokens, d] and queries [1, 1, heads, d]; the prefix's tokens, then the own ones."""

    def __init__(self, d, bits):
        rng = np.random.default_rng(10 * d + int(2 * bits))
        self.d, self.plan, self.scale = d, oracle.make_plan(d, bits), d ** -0.5
        self.signs = rng.integers(0, 2, size=(N_KV, d)).astype(np.int8) * 2 - 1
        keys = rng.standard_normal((N_KV, PREFIX + OWN, d))
        self.rec = np.stack([oracle.encode(self.plan, keys[h], self.signs[h]) for h in range(N_KV)])
        self.v = (rng.standard_normal((N_KV, PREFIX + OWN, d)).astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32)   # bf16
        self.q = rng.standard_normal((1, 1, N_KV * G, d)).astype(np.float32)

    def exact(self):
        out = np.zeros(self.q.shape)
        for h in range(N_KV):
            s = self.scale * (self.q[0, 0, h * G:(h + 1) * G].astype(np.float64) @ oracle.reconstruct(self.plan, self.rec[h], self.signs[h]).T)
            p = np.exp(s - s.max(axis=-1, keepdims=True))
            out[0, 0, h * G:(h + 1) * G] = p @ self.v[h].astype(np.float64) / p.sum(axis=-1, keepdims=True)
        return out


def off(got, want):
    return np.sqrt(np.mean((got - want) ** 2) / np.mean(want ** 2))


def _fp16(x):
    return x.astype(np.float16).astype(np.float64)


def _cut_bf16(x):
    return (x.astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)


def model(x, without=""):
    """The output of Inputs x with the kernel's operands; without: "key" or "query", whose remainders are left out, or "middle" or
    "last", a part of the probabilities."""
    out = np.zeros(x.q.shape)
    for h in range(N_KV):
        k = oracle.reconstruct(x.plan, x.rec[h], x.signs[h])
        gamma = np.linalg.norm(k, axis=-1, keepdims=True)
        k = 256.0 * np.stack([oracle.rotate(row, x.signs[h]) for row in k / gamma])
        q = np.stack([oracle.rotate(row, x.signs[h]) for row in x.q[0, 0, h * G:(h + 1) * G].astype(np.float64)])
        q_size = 2.0 ** np.ceil(np.log2(np.max(np.abs(q), axis=-1, keepdims=True)))
        kh, qh = _fp16(k), _fp16(q / q_size)
        kl, ql = _fp16(k - kh), _fp16(q / q_size - qh)
        if without == "key":
            kl = 0 * kl
        if without == "query":
            ql = 0 * ql
        s = (qh @ kh.T + ql @ kh.T + qh @ kl.T) * gamma.T * q_size * (x.scale / 256.0)
        p = np.exp(s - s.max(axis=-1, keepdims=True)).astype(np.float32).astype(np.float64)
        first = _cut_bf16(p)
        middle = _cut_bf16(p - first)
        last = _cut_bf16(p - first - middle)
        assert np.array_equal(first + middle + last, p)
        parts = first + (0.0 if without == "middle" else middle) + (0.0 if without == "last" else last)
        out[0, 0, h * G:(h + 1) * G] = parts @ x.v[h].astype(np.float64) / p.sum(axis=-1, keepdims=True)
    return out

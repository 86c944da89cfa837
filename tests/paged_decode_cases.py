"""Inputs of the paged decode whose result hangs on the low bits of the softmax weights and of float32 queries.

Two tokens of each case have a weight; the others' logits lie 1200 below.  Keys, values and bfloat16 queries are held
exactly, and so are the logits, so that the float64 result is that of the formula and what is left is the arithmetic
of the softmax and of the sums."""

import numpy as np

U = 2.0 ** -24  # half a step of float32, relative
CLEAR = 90 * U  # what a lost part changes at least: above twice the bound

# Units of U, relative to the values' magnitude of 1, with a logit x of at most 2.4 and w = exp(-x):
#   the exponent: log2(e) rounded 1/2 x 3.5, the product or reference and the difference rounded 2 each (values in
#   [2, 4)), a float32 query's three products 2 x 2.4 x 1.443: 12.7, times ln 2: 9; exp2 off by a step (2), twice
#   where the tokens are in different waves, and their product: 5.  14 of w, which the result feels at most by half
#   (2 w / (1 + w)^2): 7
#   numerator and denominator: three parts, two tokens and the columns added, 8 roundings, and the factors and sums of
#   two merges, 4: 12 each; the division: 5
BOUND = (7 + 24 + 5) * U


def trunc(x, bits):
    """float32 values x cut to their top `bits` significant bits."""
    x = np.asarray(x, dtype=np.float32)
    return (x.view(np.uint32) & np.uint32(0xFFFFFFFF << (24 - bits) & 0xFFFFFFFF)).view(np.float32)


def result(a, v0, v1, w=None):
    """Float64 outputs [heads, d] for logits 0 and -4 a and value rows v0, v1."""
    w = np.exp(-4.0 * np.asarray(a, dtype=np.float64)) if w is None else np.asarray(w, dtype=np.float64)
    return (v0[None] + w[:, None] * v1[None]) / (1.0 + w[:, None])


def heads(G, dtype):
    """Query elements a [G] in (0.08, 0.6) for which cutting the weight exp(-4 a) to 16 bits, and a itself to 16 where
    it is float32, moves (1 - w) / (1 + w) by more than CLEAR."""
    r = np.random.default_rng(G + (100 if dtype == "f32" else 0))
    out = []
    while len(out) < G:
        a = np.float32(r.uniform(0.08, 0.6))
        if dtype == "bf16":
            a = trunc(a, 8)
        ok = all(abs(result([a], np.ones(1), -np.ones(1)) - result([b], np.ones(1), -np.ones(1), w)) > CLEAR
                 for b, w in planted(a, dtype))
        if ok and a not in out:
            out.append(a)
    return np.array(out, dtype=np.float32)


def planted(a, dtype):
    """(a, weights) of computations that lose the last part of the weights, or of the queries."""
    a = np.atleast_1d(np.float32(a))
    yield a, trunc(np.exp(-4.0 * a.astype(np.float64)), 16).astype(np.float64)
    if dtype == "f32":
        yield trunc(a, 16), None


def case(G, d, dtype, n, at):
    """(q [G, d], k [n, d], v [n, d], expected [G, d]), float64, for scale 1; at: the two tokens."""
    r = np.random.default_rng(1000 * G + n)
    a = heads(G, dtype)
    q, k = np.zeros((G, d)), np.zeros((n, d))
    q[:, 0], q[:, 1] = a, 200.0
    k[:, 1] = -6.0
    k[list(at)] = 0.0
    k[at[1], 0] = -4.0
    v = r.choice([-1.0, 1.0], (n, d))
    v[at[0], 5], v[at[1], 5] = 1.0, -1.0
    return q, k, v, result(a, v[at[0]], v[at[1]])

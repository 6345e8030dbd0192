"""Inputs, oracles and rounding bounds shared by the CPU (host stand-in) and GPU tests of the
transformer operators.

Bounds. A rounding to a type is off by at most half a step: H[type] times the value (bf16 2^-8, fp32
2^-24). A sum of n products accumulated in fp32 is off by at most (n + 2) 2^-24 times the sum of the
products' magnitudes, in any order. An activation multiplies an error of its argument by its
largest slope, below 1.2, and its own evaluation (exp2, reciprocal, erf within 4 units in the last
place, on an argument rounded three times) adds below 2^-20 times |argument| + 2^-22; where the
exponential's argument is large its own rounding counts, |argument| 2^-22 more, relative to a value that is
then below the argument itself.
"""
import numpy as np

from oracle import operators as O

H = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}


def to_bf16_bits(a: np.ndarray) -> np.ndarray:
    u = np.ascontiguousarray(a, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def from_bf16_bits(b: np.ndarray) -> np.ndarray:
    return (b.astype(np.uint32) << 16).view(np.float32)


def values(rng, shape, dtype, scale=1.0) -> np.ndarray:
    """float32 array of normals that dtype represents."""
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return from_bf16_bits(to_bf16_bits(a)) if dtype == "bf16" else a


def linear_bound(ref, mag, k, act, out, residual):
    e = (k + 2) * 2.0 ** -24 * mag
    if act != "none":
        e = 1.2 * e + 2.0 ** -20 * mag + 2.0 ** -22
    r = 0.0 if residual is None else np.abs(residual)
    return e + 2.0 ** -24 * (np.abs(ref) + r) + H[out] * (np.abs(ref) + e)


def linear_inputs(m, n, k, dtype, out, bias, residual, seed):
    rng = np.random.default_rng(seed)
    return {"x": values(rng, (m, k), dtype), "w": values(rng, (n, k), dtype, max(k, 1) ** -0.5),
            "bias": rng.standard_normal(n).astype(np.float32) * 0.3 if bias else None,
            "residual": values(rng, (m, n), out) if residual else None}


def rope_bound(ref, x, dtype, pairs, layout, norm_gain=None, dh=None):
    """x: what is rotated (after the norm). A cosine or sine is within 2^-22 (its argument, at most pi / 4,
    rounded to float, a polynomial of five roundings); the products and their sum add 3 2^-24. The norm
    is off by (dh + 8) 2^-24 of each value."""
    P = sum(pairs)
    amp = np.abs(x).astype(np.float64)
    a = amp.copy()
    for j in range(P):
        i0, i1 = (j, j + P) if layout == "half" else (2 * j, 2 * j + 1)
        a[..., i0] = a[..., i1] = amp[..., i0] + amp[..., i1]
    e = a * (2.0 ** -22 + 3 * 2.0 ** -24) + 1e-45
    if norm_gain is not None:
        e = e + a * (dh + 8) * 2.0 ** -24
    return e + H[dtype] * (np.abs(ref) + e)


def attention_bound(ref, mag, top, dtype, dh, keys):
    """A score is off by (dh + 4) 2^-24 of the magnitudes it sums (top), once more for its scaling
    and the exponential; a weight by twice that relatively (numerator and sum), and by half a bf16 step
    where it is rounded for the product with v; the sums over the keys by (keys + 8) 2^-24."""
    w = 2 * (dh + 8) * 2.0 ** -24 * np.maximum(top, 1.0)[..., None] + 2 * (keys + 8) * 2.0 ** -24
    if dtype == "bf16":
        w = w + 2.0 ** -8
    e = w * mag + 1e-38
    return e + H[dtype] * (np.abs(ref) + e)


def seen_keys(n_q, n_k, k_len, window, sinks):
    """bool [k_len]: the keys that any of the n_q queries of a sequence of n_k keys sees."""
    seen = np.zeros(k_len, bool)
    for i in range(n_q):
        seen[:n_k] |= O.visible(i, n_q, n_k, *window, sinks)
    return seen


def check(got, ref, bound, what=""):
    got = np.asarray(got, np.float64)
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} outside, first at {i}: {got[i]} for {ref[i]}, "
                             f"bound {bound[i]}")


# (m, n, k): one row to several tiles of each kernel, sizes on and around the tiles' edges
LINEAR_SHAPES = [(1, 1, 1), (1, 16, 64), (3, 5, 7), (16, 33, 257), (17, 40, 96), (33, 64, 128), (64, 20, 515),
                 (65, 64, 64), (70, 100, 72), (130, 129, 200), (5, 7, 0),
                 (66, 40, 1100)]   # split along k

# tokens, q heads, k heads, dh, pairs, layout, shared
ROPE_SHAPES = [(1, 1, 1, 2, (1,), "half", False), (3, 2, 1, 16, (8,), "half", False), (5, 4, 2, 32, (8, 8), "half", False),
               (7, 3, 3, 24, (4, 4, 4), "half", True), (4, 2, 2, 34, (5, 6, 6), "half", False),
               (6, 5, 1, 64, (10, 11, 11), "adjacent", True), (9, 1, 0, 80, (16, 16), "half", False),
               (2, 40, 8, 128, (64,), "half", False), (3, 2, 2, 256, (128,), "adjacent", False),
               (3, 2, 2, 96, (16,), "adjacent", False), (3, 3, 2, 128, (16, 24, 24), "half", False), (2, 2, 1, 20, (), "half", False)]

# b, sq, sk, hq, hk, dh, (left, right), sinks, q_lengths, k_lengths
ATTENTION_SHAPES = [
    (1, 1, 1, 1, 1, 8, (-1, -1), 0, None, None),
    (2, 3, 5, 2, 1, 16, (-1, 0), 0, None, None),
    (1, 8, 8, 4, 4, 24, (-1, -1), 0, None, None),
    (2, 1, 130, 8, 2, 32, (-1, 0), 0, None, (130, 77)),
    (3, 1, 70, 4, 1, 64, (9, 0), 3, None, (70, 1, 0)),
    (2, 70, 70, 2, 2, 32, (5, 0), 2, (70, 33), (70, 33)),
    (1, 65, 40, 1, 1, 40, (-1, 0), 0, None, None),       # more queries than keys: the first see none
    (1, 20, 150, 3, 1, 128, (30, 2), 70, None, None),
    (1, 17, 66, 2, 2, 80, (0, 0), 0, None, None),        # only its own key
    (1, 5, 64, 2, 1, 256, (-1, -1), 0, None, None),
    (1, 2, 200, 2, 1, 32, (20, 0), 5, None, None),        # most of the cache out of sight, its first keys not
    (2, 2, 700, 2, 1, 16, (600, 0), 3, None, (700, 40)),  # keys split over workgroups, one of them without any
]

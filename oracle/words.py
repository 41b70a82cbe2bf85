"""Words of documents from a topic model's estimates (fp64 numpy oracle).

TEST INFRASTRUCTURE ONLY, like the rest of ``oracle/``: never imported by the product
library, and sharing no code with it.

* ``pack8`` / ``value8``: rows in 8-bit floating point (1 sign, 4 exponent, 3 fraction bits,
  bias 7, no infinities, code 127 is NaN) with a power-of-two scale for each block of 128
  columns: the least exponent e in [-127, 127] whose 448 2^e reaches the block's largest
  finite magnitude, and the nearest of the 8-bit values to x 2^-e, ties to the even code.
* ``scores``: sum over topics of theta phi.
* ``adjusted``: penalties for listed words, biases, masks, every step rounded to fp32.
* ``top``: the k largest scores, ties to the lowest word.
* ``drawn``: the first word whose prefix sum of exp((x - max) / T) exceeds u times the total.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

BLOCK = 128

# value of every non-negative code but NaN (127), ascending
VALUES8 = np.array([m / 512.0 if e == 0 else math.ldexp(1 + m / 8.0, e - 7)
                    for e in range(16) for m in range(8)][:127])


def value8(q: np.ndarray) -> np.ndarray:
    """Values of the codes q."""
    table = np.append(VALUES8, np.nan)
    q = np.asarray(q, np.uint8)
    return np.where(q < 128, 1.0, -1.0) * table[q & 127]


def scale_exponent(amax: float) -> int:
    """Least e in [-127, 127] with amax <= 448 2^e."""
    e = -127
    while e < 127 and Fraction(float(amax)) > 448 * Fraction(2) ** e:
        e += 1
    return e


def _nearest(v: np.ndarray) -> np.ndarray:
    """Codes of the 8-bit values nearest to v >= 0, ties to the even code."""
    hi = np.minimum(np.searchsorted(VALUES8, v), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = VALUES8[hi] - v, v - VALUES8[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def pack8(x: np.ndarray):
    """(codes [rows, blocks * 128] uint8, exponents + 127 [rows, blocks] uint8)."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    q = np.zeros((rows, nb * BLOCK), np.uint8)
    e = np.zeros((rows, nb), np.uint8)
    for i in range(rows):
        for b in range(nb):
            v = x[i, b * BLOCK:(b + 1) * BLOCK]
            finite = np.isfinite(v)
            ex = scale_exponent(np.abs(v[finite]).max()) if finite.any() else -127
            e[i, b] = ex + 127
            with np.errstate(invalid="ignore", over="ignore"):
                y = np.ldexp(v, -ex)
                code = np.where(np.abs(y) <= 448, _nearest(np.minimum(np.abs(np.nan_to_num(y)), 448)),
                                127)
            q[i, b * BLOCK:b * BLOCK + len(v)] = code | np.where(np.signbit(v), 128, 0)
    return q, e


def unpack8(q: np.ndarray, e: np.ndarray) -> np.ndarray:
    """What packed rows stand for, in fp64 [rows, blocks * 128]."""
    return np.ldexp(value8(q), np.repeat(e.astype(np.int64) - 127, BLOCK, axis=1))


def scores(a: np.ndarray, b: np.ndarray) -> np.ndarray:
    """Sums over columns of a [m, k] and b [n, k], in fp64."""
    return np.array([[math.fsum(ai * bj) for bj in b] for ai in a]).reshape(len(a), len(b))


def adjusted(x, listed=None, penalties=None, bias=None, allowed=None) -> np.ndarray:
    """Scores x [rows, V] under the rules, in fp32: listed, a list of word ids per row;
    penalties [rows, 3]; bias [rows, V] and allowed [rows, V] (rows taken from their tables
    already)."""
    f = np.float32
    x = np.array(x, f)
    rows, V = x.shape
    with np.errstate(all="ignore"):
        for i in range(rows):
            if listed is not None:
                counts = {}
                for w in listed[i]:
                    if 0 <= w < V:
                        counts[int(w)] = counts.get(int(w), 0) + 1
                rep, presence, frequency = (f(v) for v in penalties[i])
                for w, c in counts.items():
                    y = f(x[i, w] / rep) if x[i, w] > 0 else f(x[i, w] * rep)
                    x[i, w] = f(y - f(presence + f(frequency * f(c))))
            if bias is not None:
                x[i] = (x[i] + bias[i].astype(f)).astype(f)
            if allowed is not None:
                x[i] = np.where(allowed[i], x[i], f(-np.inf))
    return x


def top(x: np.ndarray, k: int):
    """(words [rows, k], scores [rows, k]): -1 and -inf where none is left."""
    rows, V = x.shape
    word = np.full((rows, k), -1, np.int32)
    value = np.full((rows, k), -np.inf, np.float32)
    for i in range(rows):
        ok = [w for w in range(V) if x[i, w] > -np.inf]
        ok.sort(key=lambda w: (-float(x[i, w]), w))
        n = min(k, len(ok))
        word[i, :n] = ok[:n]
        value[i, :n] = x[i, ok[:n]]
    return word, value


def borders(x: np.ndarray, temperature: float = 1.0):
    """Prefix sums of one row's weights (None: no law)."""
    x = np.asarray(x, np.float64)
    if not len(x) or np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None
    w = np.exp((x - x.max()) / temperature)
    return np.cumsum(w.astype(np.longdouble))


def drawn(x: np.ndarray, u: np.ndarray, temperature: float = 1.0):
    """(words [rows, n], log probabilities [rows, n] fp64, distance of each u to the nearest
    border between two words)."""
    rows, n = u.shape
    word = np.full((rows, n), -1, np.int32)
    logp = np.full((rows, n), np.nan)
    gap = np.full((rows, n), np.inf)
    for i in range(rows):
        c = borders(x[i], temperature)
        if c is None:
            continue
        z = (np.asarray(x[i], np.float64) - np.max(x[i])) / temperature
        log_total = math.log(math.fsum(np.exp(z)))
        positive = np.flatnonzero(np.exp(z) > 0)
        for j in range(n):
            if u[i, j] < 1:
                target = u[i, j] * np.float64(c[-1])  # u times the total, in fp64
                w = int(np.searchsorted(c, np.longdouble(max(target, 0.0)), side="right"))
                w = w if w <= positive[-1] else int(positive[-1])
                inner = np.abs(c[:-1] - target) / c[-1]
                gap[i, j] = inner.min() if u[i, j] > 0 and len(inner) else np.inf
            else:
                w = int(positive[-1])
            word[i, j] = w
            logp[i, j] = z[w] - log_total
    return word, logp, gap

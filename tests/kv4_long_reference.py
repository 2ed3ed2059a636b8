"""Long contexts on the 4-bit paged cache from their definitions, on the CPU in NumPy, 64 bits: what the tests compare with."""
import math

import numpy as np


def seen(n, queries, i, causal, window):
    """(first, one behind the last) of n positions that query i of those at the last `queries` positions sees"""
    pos = n - queries + i
    lo = max(0, pos - window + 1) if window else 0
    return lo, max(lo, min(n, pos + 1) if causal else n)


def weights(old, q, x, k, steps, mids, lse, scale, decay, causal=True, window=0):
    """(weights [kv heads, n], bound) after one call for a sequence: q rotated, x before it was (or q), both [m, heads, d]; k [n, kv heads, d], steps
    and mids [n, kv heads] of the keys; old [kv heads, n]; lse [m, heads].
    bound: products are sums of 128 in steps of 32, of elements c - 8 at most 8 in size: 16 roundings each of sums of 8 step + |mid| times the
    1-norm of q, two products (hi, lo) and the centre's: 40.  q is off by 2^-22 of its largest (two fp16 numbers), and by 16 roundings of the
    1-norm of x over sqrt(d) where it is rotated.  The exponent rounds s and lse four times.  Then a row's weight is off by a factor of
    exp(e), plus 2^-22 (the exponential, 1 ulp, and the product with log2 e), and the sum by 2^-24 for each of its terms."""
    m, heads, d = q.shape
    n, kv = steps.shape
    group = heads // kv
    w = old * decay if decay else np.zeros_like(old)
    bound = np.abs(w) * 2.0 ** -23
    terms = np.zeros_like(old)
    for i in range(m):
        lo, hi = seen(n, m, i, causal, window)
        for j in range(heads):
            y = j // group
            s = scale * k[lo:hi, y] @ q[i, j]
            p = np.exp(s - lse[i, j])
            size = 8 * steps[lo:hi, y] + np.abs(mids[lo:hi, y])
            one = np.abs(q[i, j]).sum()
            turn = 0.0 if x is q else 16 * np.abs(x[i, j]).sum() / math.sqrt(d)
            e = scale * 2.0 ** -24 * size * (40 * one + d * (4 * np.abs(q[i, j]).max() + turn)) + 2.0 ** -22 * (np.abs(s) + abs(lse[i, j]) + 1)
            w[y, lo:hi] += p
            bound[y, lo:hi] += p * np.expm1(e)
            terms[y, lo:hi] += 1
    return w, bound + 2.0 ** -24 * terms * np.abs(w)


def select(w, n, keep, sinks, recent):
    """The kept ones of n positions with weights w [at least n], and -1 behind them."""
    if n <= keep:
        return list(range(n)) + [-1] * (keep - n)
    middle = sorted(range(sinks, n - recent), key=lambda j: (math.isnan(w[j]), 0.0 if math.isnan(w[j]) else -w[j], j))
    return sorted(list(range(sinks)) + middle[:keep - sinks - recent] + list(range(n - recent, n)))

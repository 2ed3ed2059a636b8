"""The 4-bit paged cache and attention over it from their definitions, on the CPU in NumPy: what the tests compare with."""
import math

import numpy as np


def bf16(x):
    """Rounded to bfloat16 (nearest even), as float64."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(np.isnan(x), np.nan, r)


def sylvester(d):
    h = np.ones((1, 1))
    while len(h) < d:
        h = np.block([[h, h], [h, -h]])
    return h / math.sqrt(d)


def butterflies(x):
    """x H / sqrt(d) over the last axis in fp32: strides 1, 2, 4 ... and then the scale, every operation rounded."""
    x = np.asarray(x, np.float32)
    d, w = x.shape[-1], 1
    while w < d:
        y = x.reshape(x.shape[:-1] + (d // (2 * w), 2, w))
        x = np.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).reshape(x.shape)
        w *= 2
    return x * np.float32(d ** -0.5)


def quantize(y, clip):
    """(codes, step, centre) of rows, in fp32 as the header states it."""
    y, clip = np.asarray(y, np.float32), np.float32(clip)
    lo, hi = clip * y.min(-1, keepdims=True), clip * y.max(-1, keepdims=True)
    step = bf16((hi - lo) / np.float32(15)).astype(np.float32)
    mid = bf16(np.float32(0.5) * (hi + lo)).astype(np.float32)
    step = np.where(step < np.float32(2.0 ** -100), np.float32(0), step)
    with np.errstate(divide="ignore"):
        inv = np.where(step == 0, np.float32(0), np.float32(1) / step)
    codes = np.clip(np.rint((y - mid) * inv + np.float32(7.5)), 0, 15).astype(np.int64)
    return codes, step[..., 0], mid[..., 0]


class Pages:
    """The bytes of a cache [pages, page bytes] and where the header says things lie in them, an element at a time."""

    def __init__(self, pages, kv_heads, head_dim, page_size):
        self.h, self.d, self.p = kv_heads, head_dim, page_size
        self.block = page_size * (head_dim + 8)
        self.data = np.zeros((pages, kv_heads * self.block), np.uint8)

    def _value_byte(self, t, e):
        """(byte of a block, shift) of value element e of token t"""
        r, f = divmod(e, self.d // 16)
        half = ((t // 4 * 16 + r) * (self.d // 64) + f // 4) * 4 + t % 4
        return self.p * self.d // 2 + 2 * half + f % 4 // 2, 4 * (f % 2)

    def put(self, slot, head, key, value):
        """key, value: (codes [d], step, centre)"""
        page, t = divmod(int(slot), self.p)
        b = self.data[page, head * self.block:(head + 1) * self.block]
        e = np.arange(self.d)
        row = t * self.d // 2
        b[row:row + self.d // 2] = key[0][0::2] | (key[0][1::2] << 4)
        at = np.array([self._value_byte(t, i) for i in e])
        for byte in np.unique(at[:, 0]):
            b[byte] = sum(int(value[0][i]) << at[i, 1] for i in e[at[:, 0] == byte])
        for i, x in enumerate((key, value)):
            w = b[self.p * (self.d + 4 * i):][4 * t:4 * t + 4]
            w[:] = np.array([x[1], x[2]], np.float32).view(np.uint16)[1::2].copy().view(np.uint8)

    def get(self, slot, head):
        """(key [d], value [d]) as float64"""
        page, t = divmod(int(slot), self.p)
        b = self.data[page, head * self.block:(head + 1) * self.block].astype(np.int64)
        e = np.arange(self.d)
        k = (b[t * self.d // 2 + e // 2] >> (4 * (e % 2))) & 15
        at = np.array([self._value_byte(t, i) for i in e])
        v = (b[at[:, 0]] >> at[:, 1]) & 15
        out = []
        for i, c in enumerate((k, v)):
            w = self.data[page, head * self.block + self.p * (self.d + 4 * i) + 4 * t:][:4].view(np.uint16).astype(np.uint32) << 16
            step, mid = w.view(np.float32).astype(np.float64)
            out.append((c - 7.5) * step + mid)
        return out

    def rows(self, slots):
        """(keys, values) [slots, heads, d]"""
        k, v = np.zeros((2, len(slots), self.h, self.d))
        for i, s in enumerate(slots):
            for j in range(self.h):
                k[i, j], v[i, j] = self.get(s, j)
        return k, v

    def steps(self, slots):
        """steps of the keys [slots, heads]"""
        out = np.zeros((len(slots), self.h))
        for i, s in enumerate(slots):
            page, t = divmod(int(s), self.p)
            for j in range(self.h):
                w = self.data[page, j * self.block + self.p * self.d + 4 * t:][:2].view(np.uint16).astype(np.uint32) << 16
                out[i, j] = w.view(np.float32)[0]
        return out


def attention(q, k, v, steps, scale, causal=True, window=0):
    """(o, log of the sums, bound): q [n, heads, d], k and v [len, kv heads, d], steps of the keys [len, kv heads], the queries at the
    last positions; all float64.
    bound: how far a kernel may be off that rounds q (after a scale by a power of two) and p * step to fp16 (unit roundoff 2^-11) and
    adds up codes that carry 1024 in fp32.  The scores are then off by at most
        e_j = scale * (2^-11 sum_d |q_d| |k_jd| + 16 * 2^-24 * 1024 * step_j sum_d |q_d|)
    (16: the roundings of a sum of 128 in steps of 32 and what takes 1024 off again), so p_j / sum p by a factor of at most
    exp(2 max e), and the result by (exp(2 max e) - 1 + 2^-11 + 2^-16) sum_j p_j |v_j| / sum p (2^-16: fp32 sums and exp)."""
    n, heads, d = q.shape
    length, group = len(k), q.shape[1] // max(1, k.shape[1])
    o, lse, bound = np.zeros((n, heads, d)), np.full((n, heads), -np.inf), np.zeros((n, heads, d))
    for i in range(n):
        pos = length - n + i
        hi = min(length, pos + 1) if causal else length
        lo = max(0, pos - window + 1) if window else 0
        if hi <= lo:
            continue
        for j in range(heads):
            kk, vv, st = k[lo:hi, j // group], v[lo:hi, j // group], steps[lo:hi, j // group]
            s = scale * kk @ q[i, j]
            m = s.max()
            p = np.exp(s - m)
            total = p.sum()
            o[i, j] = p @ vv / total
            lse[i, j] = m + math.log(total)
            e = scale * (2.0 ** -11 * (np.abs(kk) @ np.abs(q[i, j])) + 2.0 ** -10 * st * np.abs(q[i, j]).sum()).max()
            bound[i, j] = (math.expm1(2 * e) + 2.0 ** -11 + 2.0 ** -16) * (p @ np.abs(vv)) / total
    return o, lse, bound

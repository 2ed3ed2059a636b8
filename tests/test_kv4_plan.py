"""CPU-only: how attention over the 4-bit cache is laid out.  Whatever the lengths, the chunks of a row tile cover the keys that its
rows see."""
import ctypes as C
import random

import pytest

from paper_2504_13989_amd import binding


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def plan_of(L, lens, counts, heads, kv, d, dtype, causal, window, page=64, max_len=None, decode=False, units=256):
    cache = binding.RqKv4(1 << 20, 1 << 20, kv, d, page)
    p = binding.RqKv4Plan()
    rc = L.rq_kv4_attention_plan(C.byref(cache), dtype, sum(counts), heads, len(lens), int(decode), int(causal), window,
                                 max(lens) if max_len is None else max_len, units, C.byref(p))
    assert rc == binding.RQ_OK
    return p


def keys_of(n, m, base, rows, group, causal, window):
    """The first key and the one behind the last that some row of a row tile sees: m queries at the end of n positions, rows base ... of
    m * group."""
    first, last = n - m + base // group, n - m + (min(base + rows, m * group) - 1) // group
    lo = max(0, first - window + 1) if window else 0
    return lo, (min(n, last + 1) if causal else n)


def check(p, lens, counts, group, causal, window):
    if p.chunks == 1:
        return
    for n, m in zip(lens, counts):
        for base in range(0, m * group, p.rows):
            lo, hi = keys_of(n, m, base, p.rows, group, causal, window)
            assert hi <= lo or lo // 64 * 64 + p.chunk * p.chunks >= hi, (n, m, base, lo, hi, p.chunk, p.chunks)


@pytest.mark.parametrize("lens,counts,heads,kv,d,dtype,window", [
    ([16384], [4096], 4, 1, 128, binding.RQ_BF16, 4096),
    ([8192], [1024], 16, 4, 128, binding.RQ_F16, 4096),
    ([16384], [2000], 8, 2, 128, binding.RQ_BF16, 4096),
    ([5253, 4814], [4814, 3000], 2, 2, 64, binding.RQ_BF16, 4096),
    ([11184, 3230], [3230, 900], 4, 1, 128, binding.RQ_F16, 4096),
])
def test_chunks_cover_the_keys_behind_a_query_that_is_not_causal(L, lens, counts, heads, kv, d, dtype, window):
    p = plan_of(L, lens, counts, heads, kv, d, dtype, False, window)
    assert p.many and p.chunks > 1
    check(p, lens, counts, heads // kv, False, window)


def test_chunks_cover_all_keys(L):
    rng, seen = random.Random(1), {}
    for _ in range(8000):
        kv, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 5, 8, 40))
        d, dtype, causal = rng.choice((64, 128)), rng.choice((binding.RQ_BF16, binding.RQ_F16)), rng.random() < 0.5
        window = rng.choice((0, 1, 60, 1000, 4096, rng.randrange(1, 20000)))
        lens = [int(2 ** rng.uniform(0, 15)) for _ in range(rng.choice((1, 1, 2, 5)))]
        counts = [max(1, int(n * rng.uniform(0, 1.2))) for n in lens]
        p = plan_of(L, lens, counts, kv * group, kv, d, dtype, causal, window, units=rng.choice((64, 256, 304)))
        assert p.rows in (4, 8, 16, 128, 256) and p.tiles >= sum(-(-m * group // p.rows) for m in counts)
        check(p, lens, counts, group, causal, window)
        key = (p.many, p.chunks > 1, causal, window > 0)
        seen[key] = seen.get(key, 0) + 1
    for causal in (True, False):                     # all of these were among them
        for windowed in (True, False):
            assert seen[1, True, causal, windowed] >= 10 and seen[1, False, causal, windowed] >= 10


def test_plan_refuses(L):
    cache, p = binding.RqKv4(1 << 20, 4, 2, 128, 16), binding.RqKv4Plan()
    ok = dict(dtype=0, tokens=3, heads=4, batch=3, decode=1, causal=1, window=0, max_len=32, units=256)
    ask = lambda **kw: L.rq_kv4_attention_plan(C.byref(cache), *{**ok, **kw}.values(), C.byref(p))  # noqa: E731
    assert ask() == binding.RQ_OK and not p.many and p.chunks == 1
    for bad in (dict(dtype=binding.RQ_F32), dict(tokens=0), dict(tokens=-1), dict(tokens=4), dict(heads=3), dict(heads=0), dict(batch=0, tokens=0),
                dict(causal=2), dict(window=-1), dict(max_len=-1), dict(units=-1)):
        assert ask(**bad) == binding.RQ_ERR_ARG, bad
    assert L.rq_kv4_attention_plan(C.byref(cache), *ok.values(), None) == binding.RQ_ERR_ARG


@pytest.mark.parametrize("window", [4096, 4097, 1 << 30, (1 << 31) - 1])
def test_a_window_over_all_positions_is_none(L, window):
    """as the plan shows, which takes two groups of waves without a window and one with"""
    plans = [plan_of(L, [4096], [4096], 8, 8, 64, binding.RQ_BF16, True, w) for w in (0, window, 4095)]
    assert bytes(plans[0]) == bytes(plans[1]) and plans[0].groups == 2 and plans[2].groups == 1

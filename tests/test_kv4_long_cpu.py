"""CPU-only: argument checks of the 4-bit cache's calls for long contexts."""
import ctypes as C
import random

import pytest

from paper_2504_13989_amd import binding
from paper_2504_13989_amd.pages import PagePool
from test_kv4_cpu import BAD_CACHES, cache

ARG, OK = binding.RQ_ERR_ARG, binding.RQ_OK


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def test_attention_weights_refuses(L):
    def weigh(h=None, c=None, Q=64, dtype=0, tokens=3, heads=4, q=(512, 128), lse=64, table=64, batch=3, width=2, lens=64, start=None, scale=0.1,
              causal=1, window=0, max_len=32, decay=1.0, w=64, strides=(64, 32), ws=None, ws_bytes=0):
        return L.rq_kv4_attention_weights(h, c if c is not None else cache(), Q, dtype, tokens, heads, *q, lse, table, batch, width, lens, start, scale,
                                          causal, window, max_len, decay, w, *strides, ws, ws_bytes, None)

    for bad in BAD_CACHES:
        assert weigh(c=cache(**bad)) == ARG, bad
    for bad in (dict(Q=None), dict(Q=65), dict(lse=None), dict(lse=66), dict(dtype=binding.RQ_F32), dict(dtype=9), dict(tokens=-1), dict(tokens=1 << 25),
                dict(heads=0), dict(heads=3), dict(heads=2 * 257), dict(q=(-1, 128)), dict(q=(512, -1)), dict(table=None), dict(table=66), dict(batch=-1),
                dict(width=-1), dict(lens=None), dict(lens=66), dict(start=66), dict(tokens=4), dict(scale=0.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(causal=2), dict(window=-1), dict(max_len=-1), dict(max_len=33), dict(decay=-0.5), dict(decay=1.5),
                dict(decay=float("nan")), dict(w=None), dict(w=66), dict(strides=(-64, 32)), dict(strides=(64, -32)), dict(strides=(64, 31)),
                dict(strides=(63, 32)), dict(strides=(32, 64)), dict(strides=(0, 32)), dict(strides=(1 << 62, 32)),
                dict(batch=1 << 10, tokens=1 << 10, width=1 << 26, max_len=1 << 30, strides=(1 << 31, 1 << 30))):
        assert weigh(**bad) == ARG, bad
    assert weigh(h=binding.hadamard_build(64)._h) == ARG
    assert weigh(tokens=0, batch=0, Q=None, lse=None, lens=None, table=None, w=None) == OK
    assert weigh(max_len=0, Q=None, lse=None, lens=None, table=None, w=None) == OK
    for bad in (dict(tokens=-1), dict(heads=3), dict(batch=-1), dict(window=-1), dict(max_len=-1), dict(max_len=0)):
        a = dict(tokens=3, heads=4, batch=3, decode=0, window=0, max_len=32)
        a.update(bad)
        assert L.rq_kv4_attention_weights_workspace(cache(), *a.values()) == 0, bad


def test_select_refuses(L):
    def select(w=64, layers=2, batch=3, heads=4, n=50, strides=(600, 200, 50), lens=64, keep=10, sinks=2, recent=3, index=64):
        return L.rq_kv4_select(w, layers, batch, heads, n, *strides, lens, keep, sinks, recent, index, None)

    for bad in (dict(w=None), dict(w=66), dict(layers=-1), dict(layers=1 << 17), dict(batch=-1), dict(batch=1 << 21), dict(heads=0), dict(heads=1025),
                dict(n=-1), dict(n=(1 << 30) + 1), dict(strides=(-1, 200, 50)), dict(strides=(600, -1, 50)), dict(strides=(600, 200, -1)), dict(lens=None),
                dict(lens=66), dict(keep=-1), dict(keep=4), dict(keep=(1 << 30) + 1), dict(sinks=-1), dict(recent=-1), dict(sinks=1 << 62),
                dict(index=None), dict(index=66), dict(layers=1 << 16, batch=1 << 15, heads=1)):
        assert select(**bad) == ARG, bad
    assert select(layers=0, w=None, lens=None, index=None) == select(batch=0, w=None, lens=None, index=None) == OK
    assert select(keep=0, sinks=0, recent=0, w=None, lens=None, index=None) == OK


def test_evict_refuses(L):
    def evict(c=None, layers=2, stride=4 * 2 * 16 * 136, index=64, keep=20, table=64, batch=3, width=2, new=None, new_width=0, w=64, n=40,
              strides=(240, 80, 40)):
        return L.rq_kv4_evict(c if c is not None else cache(), layers, stride, index, keep, table, batch, width, new, new_width, w, n, *strides, None)

    for bad in BAD_CACHES:
        assert evict(c=cache(**bad)) == ARG, bad
    for bad in (dict(layers=-1), dict(layers=1 << 17), dict(stride=4 * 2 * 16 * 136 - 16), dict(stride=4 * 2 * 16 * 136 + 8), dict(index=None), dict(index=66),
                dict(keep=-1), dict(keep=33), dict(keep=20, width=1), dict(table=None), dict(table=66), dict(batch=-1), dict(batch=1 << 21), dict(width=-1),
                dict(new=64, new_width=1), dict(new=64, new_width=-1), dict(new=66, new_width=2), dict(w=66), dict(n=19), dict(n=1 << 31),
                dict(strides=(-240, 80, 40)), dict(strides=(240, -80, 40)), dict(strides=(240, 80, -40)), dict(strides=(239, 80, 40)),
                dict(strides=(240, 79, 40)), dict(strides=(240, 80, 39)), dict(strides=(0, 80, 40))):
        assert evict(**bad) == ARG, bad
    assert evict(layers=0, index=None, table=None) == evict(batch=0, index=None, table=None) == OK
    assert evict(keep=0, index=None, table=None, w=None, n=0) == OK


def test_prefix_attention_refuses(L):
    ok = dict(h=None, c=cache(), Q=64, dtype=0, tokens=3, heads=4, q=(512, 128), ptable=64, groups=2, pwidth=3, plens=64, gstart=64, table=64, batch=3, width=2,
              lens=64, start=None, scale=0.1, causal=1, window=0, max_prefix=48, max_len=32, out=4096, o=(512, 128), lse=None, ws=None, ws_bytes=0)

    def attend(**kw):
        a = {**ok, **kw}
        return L.rq_kv4_prefix_attention(a["h"], a["c"], a["Q"], a["dtype"], a["tokens"], a["heads"], *a["q"], a["ptable"], a["groups"], a["pwidth"], a["plens"],
                                         a["gstart"], a["table"], a["batch"], a["width"], a["lens"], a["start"], a["scale"], a["causal"], a["window"],
                                         a["max_prefix"], a["max_len"], a["out"], *a["o"], a["lse"], a["ws"], a["ws_bytes"], None)

    for bad in BAD_CACHES:
        assert attend(c=cache(**bad)) == ARG, bad
    for bad in (dict(Q=None), dict(Q=65), dict(out=None), dict(out=65), dict(dtype=binding.RQ_F32), dict(dtype=9), dict(tokens=-1), dict(tokens=1 << 25),
                dict(heads=0), dict(heads=3), dict(heads=2 * 257), dict(q=(-1, 128)), dict(o=(512, -1)), dict(o=(100, 128)), dict(o=(512, 127)),
                dict(ptable=None), dict(ptable=66), dict(groups=0), dict(groups=-1), dict(groups=1 << 21), dict(pwidth=-1), dict(plens=None), dict(plens=66),
                dict(gstart=None), dict(gstart=66), dict(table=None), dict(table=66), dict(batch=-1), dict(batch=0), dict(width=-1), dict(lens=None),
                dict(lens=66), dict(start=66), dict(tokens=4), dict(scale=0.0), dict(scale=float("nan")), dict(causal=2), dict(window=-1), dict(max_prefix=-1),
                dict(max_prefix=49), dict(max_len=-1), dict(max_len=33), dict(pwidth=1 << 27, max_prefix=1 << 30), dict(lse=66)):
        assert attend(**bad) == ARG, bad
    assert attend(h=binding.hadamard_build(64)._h) == ARG
    assert attend(tokens=0, batch=0, groups=0, Q=None, out=None, lens=None, table=None, ptable=None, plens=None, gstart=None) == OK


def prefix_plan(L, units=256, **kw):
    a = dict(dtype=0, tokens=3, heads=4, groups=1, batch=3, decode=1, window=0, max_prefix=4096, max_len=64)
    a.update(kw)
    p = binding.RqKv4PrefixPlan()
    rc = L.rq_kv4_prefix_attention_plan(cache(kv_heads=a.pop("kv", 2), head_dim=a.pop("d", 128)), *a.values(), units, C.byref(p))
    return p if rc == OK else rc


def test_prefix_plan_refuses(L):
    assert prefix_plan(L).separate == 0 and prefix_plan(L, max_prefix=500).separate == 1
    for bad in (dict(dtype=1), dict(tokens=0), dict(tokens=4), dict(heads=3), dict(groups=0), dict(groups=1 << 21), dict(batch=0, tokens=0), dict(window=-1),
                dict(max_prefix=-1), dict(max_len=-1), dict(max_prefix=1 << 30), dict(units=-1)):
        assert prefix_plan(L, **bad) == ARG, bad
        if "units" not in bad and "dtype" not in bad:
            a = dict(tokens=3, heads=4, groups=1, batch=3, decode=1, window=0, max_prefix=4096, max_len=64)
            a.update(bad)
            if a["tokens"] != 4:
                assert L.rq_kv4_prefix_attention_workspace(cache(), *a.values()) == 0, bad


def test_prefix_chunks_cover_all_keys(L):
    rng, seen = random.Random(2), {}
    for _ in range(6000):
        kv, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 5, 8, 40))
        batch = int(2 ** rng.uniform(0, 8))
        counts = rng.choice((1, 1, 3, 50, 700))
        a = dict(kv=kv, heads=kv * group, d=rng.choice((64, 128)), dtype=rng.choice((0, 2)), tokens=batch * counts, batch=batch, groups=min(batch, rng.choice((1, 1, 2, 9))),
                 decode=int(counts == 1), window=rng.choice((0, 0, 0, 100)), max_prefix=int(2 ** rng.uniform(0, 17)), max_len=int(2 ** rng.uniform(0, 13)))
        p = prefix_plan(L, units=rng.choice((64, 256, 304)), **a)
        assert p.own_rows in (4, 8, 16, 128)
        if p.separate:
            assert p.waves in (4, 8) and not p.many and not p.own_many
        else:
            assert a["window"] in (0, 100) and (a["window"] == 0 or a["max_prefix"] + a["max_len"] <= 100) and p.shared_rows in (4, 8, 16, 128)
            assert p.shared_chunk % 64 == p.own_chunk % 64 == 0
            assert p.shared_chunk * p.shared_chunks >= a["max_prefix"] and p.own_chunk * p.own_chunks >= a["max_len"]
            assert p.shared_chunk * (p.shared_chunks - 1) < a["max_prefix"] + 64 and p.own_chunk * (p.own_chunks - 1) < a["max_len"] + 64
        key = (p.separate, p.many, p.own_many, p.shared_chunks > 1)
        seen[key] = seen.get(key, 0) + 1
    assert all(seen.get(k, 0) >= 10 for k in ((1, 0, 0, False), (0, 0, 0, True), (0, 1, 0, True), (0, 1, 1, False))), seen


def test_common_pages():
    pool = PagePool(40, 16)
    pool.add("a")
    pool.extend("a", 50)
    assert pool.common_pages(["a"]) == 3 and pool.common_pages([]) == 0
    pool.fork("a", "b")
    assert pool.common_pages("ab") == 3            # the fourth is not full
    pool.extend("a", 1)
    pool.extend("b", 30)
    assert pool.common_pages(["a", "b"]) == pool.common_pages(["b", "a"]) == 3
    pool.fork("b", "c")
    assert pool.common_pages("bc") == 5 and pool.common_pages("abc") == 3
    pool.truncate("c", 20)
    assert pool.common_pages("bc") == 1
    pool.add("d")
    assert pool.common_pages("ad") == 0
    pool.extend("d", 64)
    assert pool.common_pages("ad") == 0


def test_select_refuses_sums_that_leave_64_bits(L):
    for sinks, recent in ((1 << 62, 1 << 62), ((1 << 63) - 1, 1), (1, (1 << 63) - 1), ((1 << 63) - 1, (1 << 63) - 1), (8, 3), (0, 11)):
        assert L.rq_kv4_select(64, 2, 3, 4, 50, 600, 200, 50, 64, 10, sinks, recent, 64, None) == ARG, (sinks, recent)


def test_prefix_attention_refuses_sums_that_leave_64_bits(L):
    for most in ((1 << 63) - 1, (1 << 63) - 32, (1 << 62) + 1, (1 << 30) - 63, 1 << 30):
        assert prefix_plan(L, max_prefix=most, max_len=64) == ARG, most
        assert L.rq_kv4_prefix_attention_workspace(cache(), 3, 4, 1, 3, 1, 0, most, 64) == 0, most
        assert L.rq_kv4_prefix_attention(None, cache(), 64, 0, 3, 4, 512, 128, 64, 1, (1 << 31) - 1, 64, 64, 64, 3, 4, 64, None, 0.1, 1, 0, most, 64,
                                         4096, 512, 128, None, None, 0, None) == ARG, most
    assert prefix_plan(L, max_prefix=(1 << 30) - 64, max_len=64).shared_chunks > 0


def test_shared_pages():
    pool = PagePool(40, 16)
    pool.add("a")
    assert pool.shared_pages("a") == 0
    pool.extend("a", 50)
    assert pool.shared_pages("a") == 0
    pool.fork("a", "b")
    pool.fork("b", "c")
    assert [pool.shared_pages(s) for s in "abc"] == [4, 4, 4]
    pool.extend("b", 20)                           # its fourth page is its own then, and so is the fifth
    assert [pool.shared_pages(s) for s in "abc"] == [4, 3, 4]
    pool.truncate("c", 20)
    assert [pool.shared_pages(s) for s in "abc"] == [3, 3, 2]
    pool.free("a")
    assert [pool.shared_pages(s) for s in "bc"] == [2, 2]
    pool.compact()
    assert [pool.shared_pages(s) for s in "bc"] == [2, 2]
    pool.free("c")
    assert pool.shared_pages("b") == 0
    with pytest.raises(KeyError):
        pool.shared_pages("c")

"""CPU-only: the 4-bit paged cache's argument checks, the layout the tests' reference reads, and the page pool."""
import ctypes as C
import random

import numpy as np
import pytest

import kv4_reference as ref
from paper_2504_13989_amd import binding
from paper_2504_13989_amd.pages import PagePool

ARG = binding.RQ_ERR_ARG


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def cache(**kw):
    c = dict(data=1 << 20, pages=4, kv_heads=2, head_dim=128, page_size=16)
    c.update(kw)
    return C.byref(binding.RqKv4(c["data"], c["pages"], c["kv_heads"], c["head_dim"], c["page_size"]))


BAD_CACHES = [dict(data=0), dict(data=(1 << 20) + 8), dict(pages=-1), dict(pages=1 << 31), dict(kv_heads=0), dict(kv_heads=1025),
              dict(head_dim=96), dict(head_dim=256), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=-16)]


def test_page_bytes(L):
    assert L.rq_kv4_page_bytes(8, 128, 64) == 8 * 64 * 136
    assert L.rq_kv4_page_bytes(3, 64, 16) == 3 * 16 * 72
    for bad in ((0, 128, 64), (8, 96, 64), (8, 128, 24), (8, 128, 512), (1 << 30, 128, 64)):
        assert L.rq_kv4_page_bytes(*bad) == 0
        with pytest.raises(binding.RotqError):
            binding.kv4_page_bytes(*bad)


def append(L, h=None, c=None, K=64, V=64, dtype=0, tokens=3, strides=(256, 128, 256, 128), slots=64, clip=1.0):
    return L.rq_kv4_append(h, c if c is not None else cache(), K, V, dtype, tokens, *strides, slots, clip, None)


def test_append_refuses(L):
    assert append(L, c=C.POINTER(binding.RqKv4)()) == ARG
    for bad in BAD_CACHES:
        assert append(L, c=cache(**bad)) == ARG, bad
    for bad in (dict(K=None), dict(V=None), dict(slots=None), dict(K=63), dict(V=63), dict(slots=60), dict(K=66, dtype=1), dict(dtype=3),
                dict(tokens=-1), dict(clip=0.0), dict(clip=1.5), dict(clip=float("nan")), dict(strides=(-1, 128, 256, 128)),
                dict(strides=(256, 128, 256, -128))):
        assert append(L, **bad) == ARG, bad
    other, block = binding.hadamard_build(64), binding.hadamard_build(384)
    assert append(L, h=other._h) == ARG and append(L, h=block._h) == ARG      # not the heads' rotation
    assert append(L, tokens=0, K=None, V=None, slots=None) == binding.RQ_OK


def test_read_refuses(L):
    def read(h=None, c=None, slots=64, rows=3, K=64, V=64, dtype=0):
        return L.rq_kv4_read(h, c if c is not None else cache(), slots, rows, K, V, dtype, None)

    for bad in BAD_CACHES:
        assert read(c=cache(**bad)) == ARG, bad
    for bad in (dict(slots=None), dict(slots=68), dict(rows=-1), dict(K=None), dict(V=None), dict(K=72), dict(V=68), dict(dtype=7)):
        assert read(**bad) == ARG, bad
    assert read(h=binding.hadamard_build(64)._h) == ARG
    assert read(rows=0, slots=None, K=None, V=None) == binding.RQ_OK


def test_copy_pages_refuses(L):
    def copy(c=None, layers=2, stride=4 * 2 * 16 * 136, src=64, dst=64, pairs=1):
        return L.rq_kv4_copy_pages(c if c is not None else cache(), layers, stride, src, dst, pairs, None)

    for bad in BAD_CACHES:
        assert copy(c=cache(**bad)) == ARG, bad
    for bad in (dict(layers=-1), dict(layers=1 << 20), dict(stride=4 * 2 * 16 * 136 - 16), dict(stride=4 * 2 * 16 * 136 + 8), dict(src=None),
                dict(dst=None), dict(src=66), dict(dst=62), dict(pairs=-1), dict(pairs=1 << 31)):
        assert copy(**bad) == ARG, bad
    assert copy(pairs=0, src=None, dst=None) == binding.RQ_OK and copy(layers=0) == binding.RQ_OK


def test_attention_refuses(L):
    def attend(h=None, c=None, Q=64, dtype=0, tokens=3, heads=4, q=(512, 128), table=64, batch=3, width=2, lens=64, start=None, scale=0.1,
               causal=1, window=0, max_len=32, out=4096, o=(512, 128), lse=None, ws=None, ws_bytes=0):
        return L.rq_kv4_attention(h, c if c is not None else cache(), Q, dtype, tokens, heads, *q, table, batch, width, lens, start, scale, causal,
                                  window, max_len, out, *o, lse, ws, ws_bytes, None)

    for bad in BAD_CACHES:
        assert attend(c=cache(**bad)) == ARG, bad
    for bad in (dict(Q=None), dict(Q=65), dict(out=None), dict(out=65), dict(dtype=binding.RQ_F32), dict(dtype=9), dict(tokens=-1),
                dict(tokens=1 << 25), dict(heads=0), dict(heads=3), dict(heads=2 * 257), dict(q=(-1, 128)), dict(o=(512, -1)), dict(table=None),
                dict(table=66), dict(batch=-1), dict(batch=0), dict(width=-1), dict(lens=None), dict(lens=66), dict(start=66),
                dict(tokens=4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(causal=2),
                dict(window=-1), dict(max_len=-1), dict(max_len=33), dict(lse=66)):
        assert attend(**bad) == ARG, bad
    assert attend(h=binding.hadamard_build(64)._h) == ARG
    assert attend(tokens=0, batch=0, Q=None, out=None, lens=None, table=None) == binding.RQ_OK
    for bad in (dict(tokens=-1), dict(heads=3), dict(batch=-1), dict(window=-1), dict(max_len=-1)):
        a = dict(tokens=3, heads=4, batch=3, decode=1, window=0, max_len=32)
        a.update(bad)
        assert L.rq_kv4_attention_workspace(cache(), *a.values()) == 0, bad


def test_a_closed_rotation_is_refused():
    h = binding.hadamard_build(128)
    assert binding._rotation(None) == 0 and binding._rotation(h) == h._p
    h.close()
    with pytest.raises(binding.RotqError):
        binding._rotation(h)


def test_cache_object():
    import torch
    c = binding.KV4Cache(torch.zeros((3, 5, 2 * 16 * 136), dtype=torch.uint8), 2, 128, 16)
    assert (c.layers, c.pages) == (3, 5) and c.layer(2).data.data_ptr() == c.data[2].data_ptr() and c.layer(0).layers == 1
    assert c.layer(1).layer(0).data.shape == (5, 2 * 16 * 136)
    with pytest.raises(IndexError):
        c.layer(3)
    with pytest.raises(ValueError):
        binding.KV4Cache(c.data, 2, 64, 16)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_reference_layout_is_one_to_one(d, page):
    """every nibble of a block belongs to one element, and what is put comes back"""
    rng = np.random.default_rng(0)
    c = ref.Pages(3, 2, d, page)
    rows = {}
    for slot in rng.permutation(3 * page):
        for head in range(2):
            rows[slot, head] = [(rng.integers(0, 16, d), 2.0 ** rng.integers(-3, 3), float(rng.integers(-8, 8))) for _ in range(2)]
            c.put(slot, head, *rows[slot, head])
    for (slot, head), (k, v) in rows.items():
        for got, (codes, step, mid) in zip(c.get(slot, head), (k, v)):
            assert np.array_equal(got, (codes - 7.5) * step + mid)
    assert np.array_equal(c.steps([0, 5])[:, 1], [rows[0, 1][0][1], rows[5, 1][0][1]])


def test_reference_rotation_is_the_sylvester_matrix():
    x = np.random.default_rng(1).standard_normal((7, 64))
    assert np.allclose(ref.butterflies(x), x @ ref.sylvester(64), atol=1e-6)
    h = binding.hadamard_build(64)
    assert np.array_equal(np.sign(ref.sylvester(64)), h.dense())


# ---- the pool

def test_pool_hands_out_slots_and_frees():
    pool = PagePool(4, 16)
    pool.add("a")
    slots, copies = pool.extend("a", 20)
    assert slots == list(range(20)) and copies == [] and pool.free_pages == 2 and pool.length("a") == 20
    assert pool.extend("a", 0) == ([], [])
    pool.truncate("a", 16)
    assert pool.free_pages == 3 and pool.table("a") == [0]
    pool.free("a")
    assert pool.free_pages == 4
    for call in (lambda: pool.table("a"), lambda: pool.free("a"), lambda: pool.extend("a", 1)):
        with pytest.raises(KeyError):
            call()


def test_pool_refuses():
    with pytest.raises(ValueError):
        PagePool(-1, 16)
    pool = PagePool(2, 16)
    pool.add(1)
    with pytest.raises(ValueError):
        pool.add(1)
    with pytest.raises(ValueError):
        pool.extend(1, -1)
    with pytest.raises(MemoryError):
        pool.extend(1, 33)
    assert pool.length(1) == 0 and pool.free_pages == 2
    pool.extend(1, 32)
    with pytest.raises(ValueError):
        pool.truncate(1, 33)
    with pytest.raises(ValueError):
        pool.fork(1, 1)


def test_pool_copies_a_shared_page_before_it_is_written():
    pool = PagePool(6, 16)
    pool.add("a")
    pool.extend("a", 20)
    pool.fork("a", "b")
    assert pool.free_pages == 4 and pool.table("b") == pool.table("a") == [0, 1]
    slots, copies = pool.extend("b", 2)
    assert copies == [(1, 2)] and slots == [2 * 16 + 4, 2 * 16 + 5] and pool.table("b") == [0, 2]
    assert pool.extend("a", 1) == ([16 + 4], [])                    # its own again
    pool.free("a")
    assert pool.table("b") == [0, 2] and pool.free_pages == 4
    pool.add("c")
    pool.extend("c", 16)
    pool.fork("c", "d")
    assert pool.extend("d", 1)[1] == []                             # a full page needs no copy


def test_pool_against_a_model():
    """random work: every sequence's tokens stay where its table says, through forks, frees and compactions"""
    rng, P = random.Random(3), 16
    pool, mem, truth, n = PagePool(24, P), {}, {}, 0

    def copy(pairs):
        read, written = {s for s, _ in pairs}, [d for _, d in pairs]
        assert not read & set(written) and len(set(written)) == len(written)
        for s, d in pairs:
            for i in range(P):
                mem.pop(d * P + i, None)
                if s * P + i in mem:
                    mem[d * P + i] = mem[s * P + i]

    for _ in range(3000):
        seqs = list(truth)
        do = rng.choice(("add", "extend", "extend", "extend", "fork", "free", "truncate", "compact"))
        if do == "add" or not seqs:
            n += 1
            pool.add(n)
            truth[n] = []
        elif do == "extend":
            s, k = rng.choice(seqs), rng.randrange(1, 30)
            try:
                slots, pairs = pool.extend(s, k)
            except MemoryError:
                continue
            copy(pairs)
            for x in slots:
                mem[x] = (s, len(truth[s]), rng.random())
                truth[s].append(mem[x])
        elif do == "fork":
            n += 1
            s = rng.choice(seqs)
            pool.fork(s, n)
            truth[n] = list(truth[s])
        elif do == "free":
            s = rng.choice(seqs)
            pool.free(s)
            del truth[s]
        elif do == "truncate":
            s = rng.choice(seqs)
            k = rng.randrange(len(truth[s]) + 1)
            pool.truncate(s, k)
            del truth[s][k:]
        else:
            copy(pool.compact())
            held = {p for s in truth for p in pool.table(s)}
            assert held == set(range(len(held)))
        held = {p for s in truth for p in pool.table(s)}
        assert pool.free_pages == 24 - len(held)
        for s, rows in truth.items():
            t = pool.table(s)
            assert pool.length(s) == len(rows) and len(t) == -(-len(rows) // P)
            assert [mem[t[i // P] * P + i % P] for i in range(len(rows))] == rows


@pytest.mark.parametrize("o", [(0, 128), (512, 0), (512, 127), (100, 128), (0, 0)])
def test_attention_refuses_results_that_overlap(L, o):
    assert L.rq_kv4_attention(None, cache(), 64, 0, 3, 4, 512, 128, 64, 3, 2, 64, None, 0.1, 1, 0, 32, 4096, *o, None, None, 0, None) == ARG


def test_pairs_of_consecutive_extends_make_one_copy():
    """A server's step: every sequence gets room, then one copy of all pairs, all pages read before any is written, then the tokens.  Pairs name no
    page in both places, and every sequence keeps its tokens."""
    rng, P = random.Random(5), 16
    pool, mem, truth, n = PagePool(80, P), {}, {0: []}, 0
    pool.add(0)
    joined = 0
    for step in range(400):
        tokens, pairs = [], []
        for s in rng.sample(sorted(truth), len(truth)):
            k = rng.choice((0, 1, 1, 1, 7, 20))
            try:
                slots, copies = pool.extend(s, k)
            except MemoryError:
                continue
            tokens += [(x, s, (s, len(truth[s]) + i, step)) for i, x in enumerate(slots)]
            truth[s] = truth[s] + [(s, len(truth[s]) + i, step) for i in range(len(slots))]
            pairs += copies
        src, dst = [a for a, _ in pairs], [b for _, b in pairs]
        assert not set(src) & set(dst) and len(set(dst)) == len(dst)
        joined = max(joined, len(pairs))
        old = dict(mem)
        for a, b in pairs:
            for i in range(P):
                if a * P + i in old:
                    mem[b * P + i] = old[a * P + i]
        for x, _, value in tokens:
            mem[x] = value
        for s, rows in truth.items():
            t = pool.table(s)
            assert [mem[t[i // P] * P + i % P] for i in range(len(rows))] == rows
        s = rng.choice(sorted(truth))
        if len(truth) < 6:
            n += 1
            pool.fork(s, n)
            truth[n] = list(truth[s])
        elif rng.random() < 0.5:
            pool.free(s)
            del truth[s]
        else:
            k = rng.randrange(len(truth[s]) + 1)
            pool.truncate(s, k)
            truth[s] = truth[s][:k]
    assert joined > 1

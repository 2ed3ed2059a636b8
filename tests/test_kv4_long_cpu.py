"""CPU-only: argument checks of the 4-bit cache's calls for long contexts."""
import ctypes as C

import pytest

from paper_2504_13989_amd import binding
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
                dict(strides=(63, 32)), dict(strides=(32, 64)), dict(strides=(0, 32)), dict(strides=(1 << 62, 32))):
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

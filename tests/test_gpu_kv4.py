"""GPU: the 4-bit paged cache against its definition (tests/kv4_reference.py, NumPy, 64 bits)."""
import itertools
import math

import numpy as np
import pytest

import kv4_reference as ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402
from paper_2504_13989_amd import binding  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U_OUT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}      # unit roundoff


def rows(rng, n, heads, d, dtype, scale=1.0):
    """token rows with a strong channel and some large tokens, as a device tensor and as the float64 values it holds"""
    x = rng.standard_normal((n, heads, d)) * scale
    x[:, :, rng.integers(0, d)] *= 8
    x *= rng.uniform(0.5, 2, (n, heads, 1))
    t = torch.tensor(x, dtype=torch.float32).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def reference_of(cache):
    c = ref.Pages(0, cache.kv_heads, cache.head_dim, cache.page_size)
    c.data = cache.data.cpu().numpy()
    return c


# ---- append

@pytest.mark.parametrize("d,page", [(64, 16), (128, 16), (128, 64), (64, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rotate", [False, True])
def test_append_writes_the_bytes_of_the_definition(d, page, dtype, rotate):
    rng = np.random.default_rng(d + page)
    heads, tokens, pages = 3, 37, 6
    k, kx = rows(rng, tokens, heads, d, dtype)
    v, vx = rows(rng, tokens, heads, d, dtype)
    slots = rng.permutation(pages * page)[:tokens]
    cache = rq.kv4_cache(pages, heads, d, page)
    want = ref.Pages(pages, heads, d, page)
    rq.kv4_append(rq.hadamard_build(d) if rotate else None, cache, k, v, torch.tensor(slots).cuda(), clip=0.9)
    key = ref.quantize(ref.butterflies(kx) if rotate else kx, 0.9)
    value = ref.quantize(vx, 0.9)
    for i, s in enumerate(slots):
        for h in range(heads):
            want.put(s, h, [x[i, h] for x in key], [x[i, h] for x in value])
    assert np.array_equal(cache.data.cpu().numpy(), want.data)           # all other bytes are as they were


@pytest.mark.parametrize("rotate", [False, True])
def test_appended_rows_are_within_half_a_step_of_the_rows(rotate):
    """clip 1, in 64 bits: half a step, the rounding of the step (2^-9 of 7.5 steps) and of the centre (2^-9), and fp32 arithmetic
    (2^-20 of the row's largest, generously: ten roundings of sums of 128)"""
    rng = np.random.default_rng(5)
    d, heads, tokens = 128, 2, 200
    k, kx = rows(rng, tokens, heads, d, "f32")
    v, vx = rows(rng, tokens, heads, d, "f32")
    cache = rq.kv4_cache(4, heads, d, 64)
    rq.kv4_append(rq.hadamard_build(d) if rotate else None, cache, k, v, torch.arange(tokens).cuda())
    c = reference_of(cache)
    for y, got in zip((kx @ ref.sylvester(d) if rotate else kx, vx), c.rows(range(tokens))):
        span = y.max(-1, keepdims=True) - y.min(-1, keepdims=True)
        mid = abs(y.max(-1, keepdims=True) + y.min(-1, keepdims=True)) / 2
        tol = span / 15 * (1 + 2.0 ** -8) * (0.5 + 7.5 * 2.0 ** -8) + mid * 2.0 ** -8 + 2.0 ** -20 * abs(y).max(-1, keepdims=True)
        assert (abs(got - y) <= tol).all()


@pytest.mark.parametrize("dtype,pad", [("bf16", 8), ("bf16", 1), ("f16", 4), ("f32", 4), ("f32", 1)])
def test_append_takes_slices_of_any_alignment(dtype, pad):
    """the same bytes from a fused projection's output whose rows begin on 16 bytes, or on no such boundary"""
    rng = np.random.default_rng(7)
    d, heads, tokens = 128, 2, 11
    k, _ = rows(rng, tokens, heads, d, dtype)
    v, _ = rows(rng, tokens, heads, d, dtype)
    h, slots = rq.hadamard_build(d), torch.arange(tokens).cuda()
    a, b = rq.kv4_cache(1, heads, d, 16), rq.kv4_cache(1, heads, d, 16)
    rq.kv4_append(h, a, k, v, slots)
    wide = torch.full((tokens, 2 * heads, d + pad), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, :heads, :d], wide[:, heads:, pad:] = k, v
    rq.kv4_append(h, b, wide[:, :heads, :d], wide[:, heads:, pad:], slots)
    assert torch.equal(a.data, b.data)


def test_append_leaves_out_tokens_without_a_slot():
    rng = np.random.default_rng(8)
    k, _ = rows(rng, 9, 2, 64, "bf16")
    cache, some = rq.kv4_cache(2, 2, 64, 16), rq.kv4_cache(2, 2, 64, 16)
    slots = torch.tensor([3, -1, 32, 5, 1 << 40, -(1 << 62), 31, 33, 0]).cuda()
    rq.kv4_append(None, cache, k, k, slots)
    keep = [0, 3, 6, 8]
    rq.kv4_append(None, some, k[keep], k[keep], slots[keep])
    assert torch.equal(cache.data, some.data) and cache.data.any()
    rq.kv4_append(None, cache, k[:0], k[:0], slots[:0])
    assert torch.equal(cache.data, some.data)


def test_append_of_rows_that_are_flat_tiny_huge_or_not_finite():
    d = 128
    x = torch.zeros(8, 1, d)
    x[1] = -3.0                                           # flat
    x[2] = torch.linspace(-1e-37, 1e-37, d)               # a step below 2^-100
    x[3] = torch.linspace(-3e38, 3e38, d)                 # max - min overflows
    x[4] = torch.linspace(-1e37, 1e37, d)
    x[5] = torch.linspace(-1, 1, d)
    x[5, 0, 77] = float("nan")
    x[6] = torch.linspace(-1, 1, d)
    x[6, 0, 3] = float("inf")
    x[7] = torch.linspace(-1, 1, d)
    cache = rq.kv4_cache(1, 1, d, 16)
    rq.kv4_append(None, cache, x.cuda(), x.cuda(), torch.arange(8).cuda())
    for y in reference_of(cache).rows(range(8)):
        y = y[:, 0]
        assert (y[0] == 0).all() and (y[1] == -3).all() and (y[2] == 0).all()
        assert not np.isfinite(y[3]).any() and np.isnan(y[5]).all() and np.isnan(y[6]).all()
        for r in (4, 7):
            want = x[r, 0].double().numpy()
            assert (abs(y[r] - want) <= want[-1] / 15 * 1.1).all()
    # rotated: only the rows with infinities or NaN are lost
    rq.kv4_append(rq.hadamard_build(d), cache, x.cuda(), x.cuda(), torch.arange(8).cuda())
    k = reference_of(cache).rows(range(8))[0][:, 0]
    assert [bool(np.isfinite(r).all()) for r in k] == [True, True, True, False, True, False, False, True]


# ---- read

@pytest.mark.parametrize("d,page,dtype,rotate", [(64, 16, "f32", True), (128, 64, "bf16", True), (128, 32, "f16", False), (64, 128, "bf16", False),
                                                 (128, 16, "f32", True)])
def test_read_gives_the_stored_rows(d, page, dtype, rotate):
    """one rounding to the output's type; rotated keys besides fp32 butterflies: log2(d) + 2 roundings of values up to the row's 1-norm
    over sqrt(d)"""
    rng = np.random.default_rng(d)
    heads, pages = 3, 4
    cache = rq.kv4_cache(pages, heads, d, page)
    k, _ = rows(rng, pages * page, heads, d, "f32")
    v, _ = rows(rng, pages * page, heads, d, "f32")
    rq.kv4_append(None, cache, k, v, torch.arange(pages * page).cuda())
    slots = rng.permutation(pages * page)[:29]
    slots[[4, 9]] = [-1, pages * page]
    gk, gv = rq.kv4_read(rq.hadamard_build(d) if rotate else None, cache, torch.tensor(slots).cuda(), out_dtype=DT[dtype])
    assert gk.shape == gv.shape == (29, heads, d) and gk.dtype == gv.dtype == DT[dtype]
    there = (slots >= 0) & (slots < pages * page)
    wk, wv = reference_of(cache).rows(np.where(there, slots, 0))
    wk, wv = wk * there[:, None, None], wv * there[:, None, None]
    assert np.array_equal(gv.double().cpu().numpy(), torch.tensor(wv).float().to(DT[dtype]).double().numpy())
    if not rotate:
        assert np.array_equal(gk.double().cpu().numpy(), torch.tensor(wk).float().to(DT[dtype]).double().numpy())
    else:
        slop = (math.log2(d) + 2) * 2.0 ** -24 * abs(wk).sum(-1, keepdims=True) / math.sqrt(d)
        wk = wk @ ref.sylvester(d)
        assert (abs(gk.double().cpu().numpy() - wk) <= U_OUT[dtype] * abs(wk) + 2 * slop).all()
    ok, ov = torch.empty_like(gk), torch.empty_like(gv)
    a, b = rq.kv4_read(rq.hadamard_build(d) if rotate else None, cache, torch.tensor(slots).cuda(), out_dtype=DT[dtype], k=ok, v=ov)
    assert a is ok and b is ov and torch.equal(ok, gk) and torch.equal(ov, gv)


# ---- pages

def test_copy_pages_in_all_layers():
    g = torch.Generator(device="cuda").manual_seed(1)
    data = torch.randint(0, 256, (3, 11, 2 * 32 * 136), generator=g, device="cuda", dtype=torch.uint8)
    cache, want = rq.KV4Cache(data, 2, 128, 32), data.clone()
    src, dst = [10, 0, 3, 7, -1, 4, 11], [1, 2, 3, 8, 5, 11, 6]        # 3 -> 3 does nothing; pages that are not there: left out
    rq.kv4_copy_pages(cache, torch.tensor(src, dtype=torch.int32).cuda(), torch.tensor(dst, dtype=torch.int32).cuda())
    for s, d in ((10, 1), (0, 2), (7, 8)):
        want[:, d] = want[:, s]
    assert torch.equal(data, want)
    one = cache.layer(1)
    rq.kv4_copy_pages(one, torch.tensor([9], dtype=torch.int32).cuda(), torch.tensor([0], dtype=torch.int32).cuda())
    want[1, 0] = want[1, 9]
    assert torch.equal(data, want)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    rq.kv4_copy_pages(cache, none, none)
    assert torch.equal(data, want)


@pytest.mark.parametrize("heads,d,page", [(1, 64, 16), (32, 128, 256), (5, 128, 64)])
def test_copy_pages_of_any_size(heads, d, page):
    data = torch.randint(0, 256, (9, heads * page * (d + 8)), device="cuda", dtype=torch.uint8)
    want = data.clone()
    want[[7, 8]] = want[[1, 2]]
    rq.kv4_copy_pages(rq.KV4Cache(data, heads, d, page), torch.tensor([1, 2], dtype=torch.int32).cuda(), torch.tensor([7, 8], dtype=torch.int32).cuda())
    assert torch.equal(data, want)


# ---- attention

class Batch:
    """sequences in a cache of their own: appended keys and values, a table of shuffled pages"""

    def __init__(self, lens, kv_heads, d, page, rotate, seed=0, junk=0xFF, spare=2):
        rng = np.random.default_rng(seed)
        self.rng, self.lens, self.kv, self.d, self.page = rng, lens, kv_heads, d, page
        need = [-(-n // page) for n in lens]
        pages = sum(need) + spare
        self.h = rq.hadamard_build(d) if rotate else None
        self.cache = rq.kv4_cache(pages, kv_heads, d, page)
        self.cache.data.fill_(junk)                       # slots that nothing is appended to: NaN parameters
        order = rng.permutation(pages)
        self.table = np.full((len(lens), max(1, max(need))), -1, np.int32)
        self.slots, at = [], 0
        for i, (n, m) in enumerate(zip(lens, need)):
            self.table[i, :m] = order[at:at + m]
            at += m
            self.slots.append(self.table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page if n else np.zeros(0, np.int64))
        total = sum(lens)
        if total:
            k, _ = rows(rng, total, kv_heads, d, "bf16", 0.7)
            v, _ = rows(rng, total, kv_heads, d, "bf16")
            rq.kv4_append(self.h, self.cache, k, v, torch.tensor(np.concatenate(self.slots)).cuda())
        self.dev_table = torch.tensor(self.table).cuda()
        self.dev_lens = torch.tensor(lens, dtype=torch.int32).cuda()

    def queries(self, counts, heads, dtype, scale=1.0):
        q = torch.tensor(self.rng.standard_normal((sum(counts), heads, self.d)) * scale, dtype=torch.float32).to(DT[dtype])
        start = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32).cuda()
        return q.cuda(), start

    def check(self, q, counts, o, lse=None, scale=None, causal=True, window=0):
        dtype = {v: k for k, v in DT.items()}[q.dtype]
        scale = scale if scale is not None else 1 / math.sqrt(self.d)
        c = reference_of(self.cache)
        qx = q.double().cpu().numpy()
        qx = qx @ ref.sylvester(self.d) if self.h else qx
        got, at = o.double().cpu().numpy(), 0
        for i, n in enumerate(counts):
            k, v = c.rows(self.slots[i])
            w, wl, bound = ref.attention(qx[at:at + n], k, v, c.steps(self.slots[i]), scale, causal, window)
            tol = bound * (1 + U_OUT[dtype]) + U_OUT[dtype] * abs(w)
            g = got[at:at + n]
            assert np.isfinite(g).all()
            assert (abs(g - w) <= tol).all(), (i, n, np.max(abs(g - w) / np.maximum(tol, 1e-30)))
            # all roundings at their worst at once is not what happens: they average out over the elements
            assert np.linalg.norm(g - w) <= 0.25 * np.linalg.norm(bound) + U_OUT[dtype] * np.linalg.norm(w)
            if lse is not None:
                gl = lse[at:at + n].double().cpu().numpy()
                none = np.isinf(wl)
                assert np.array_equal(np.isinf(gl), none)
                # as far off as a score may be: a third of log(1 + bound / sum p |v|) and more
                assert (abs(gl[~none] - wl[~none]) <= 0.05 + 1e-3 * abs(wl[~none])).all()
            at += n


CASES = [  # lens, counts, heads, kv_heads, d, page, rotate, dtype, causal, window
    ([1], [1], 1, 1, 64, 16, False, "bf16", True, 0),
    ([1], [1], 4, 4, 128, 16, True, "f16", True, 0),
    ([15, 16, 17, 63, 64, 65], [1] * 6, 4, 2, 128, 16, True, "bf16", True, 0),
    ([257, 1, 100], [1, 1, 1], 10, 2, 128, 64, True, "f16", True, 0),
    ([300, 31], [1, 1], 32, 1, 64, 32, True, "bf16", True, 0),                    # 32 rows of a kv head: two row tiles
    ([130, 200], [1, 1], 40, 1, 128, 256, False, "f16", True, 0),                 # 40: tiles that end inside a group
    ([129], [129], 2, 1, 128, 16, True, "bf16", True, 0),                         # a prompt
    ([200], [200], 1, 1, 64, 64, False, "f16", True, 0),
    ([150], [70], 4, 2, 128, 32, True, "bf16", True, 0),                          # a chunk of one
    ([150], [70], 4, 2, 128, 32, True, "bf16", False, 0),
    ([333], [300], 1, 1, 128, 64, True, "f16", True, 0),                          # many rows: waves with rows of their own
    ([280], [280], 2, 2, 64, 16, True, "bf16", True, 0),
    ([90, 5, 200, 33], [90, 1, 3, 20], 7, 1, 64, 16, False, "f16", True, 0),      # prompts, chunks and single tokens
    ([90, 5, 200, 33], [90, 1, 3, 20], 6, 3, 128, 16, True, "bf16", True, 40),
    ([260, 100], [200, 77], 2, 1, 128, 64, False, "bf16", True, 1),               # each token sees itself only
    ([260, 100], [200, 77], 4, 4, 64, 64, True, "f16", True, 64),
    ([260, 100], [60, 77], 2, 2, 64, 64, True, "f16", False, 50),
    ([120, 130], [1, 1], 3, 3, 128, 16, True, "bf16", True, 17),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case):
    lens, counts, heads, kv, d, page, rotate, dtype, causal, window = CASES[case]
    b = Batch(lens, kv, d, page, rotate, seed=case)
    q, start = b.queries(counts, heads, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, None if set(counts) == {1} else start, causal=causal, window=window, lse=lse)
    assert o.dtype == q.dtype and o.shape == q.shape
    b.check(q, counts, o, lse, causal=causal, window=window)


@pytest.mark.parametrize("dtype,group", [("bf16", 1), ("f16", 4), ("f16", 24)])
def test_long_sequences_are_split_and_joined(dtype, group):
    lens = [4999, 3, 2048, 0, 1500]
    b = Batch(lens, 1, 64, 32, True, seed=3)
    q, start = b.queries([1] * 5, group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, lse=lse)
    assert binding.lib().rq_kv4_attention_workspace(binding.RqKv4(b.cache.data.data_ptr(), b.cache.pages, 1, 64, 32), 5, group, 5, 1, 0, 4999) > 0
    b.check(q, [1] * 5, o, lse)
    assert torch.equal(o, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens))
    # and as queries of a ragged batch, and with a workspace of the caller's
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    b.check(q, [1] * 5, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, workspace=ws))
    with pytest.raises(rq.RotqError):
        rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, workspace=ws[:64])


def test_chunk_of_a_prompt_behind_a_long_cache():
    b = Batch([3000], 1, 128, 64, True, seed=4)
    q, start = b.queries([130], 2, "bf16")
    lse = torch.empty(q.shape[:2], device="cuda")
    b.check(q, [130], rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, lse=lse), lse)
    b.check(q, [130], rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, window=700, lse=lse), lse, window=700)


def test_rows_that_see_nothing_are_zeros():
    b = Batch([0, 5, 40], 2, 128, 16, True, seed=6)
    for counts in ([3, 9, 0], [1, 1, 1], [100, 90, 80]):           # more queries than positions: the first see nothing
        q, start = b.queries(counts, 4, "bf16")
        o, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
        r = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, out=o, lse=lse)
        assert r is o
        b.check(q, counts, o, lse)
        none = torch.isinf(lse)
        assert none.any() and (lse[none] < 0).all() and (o[none] == 0).all() and (o[~none] != 0).any()


def test_lengths_out_of_range_are_cut():
    b = Batch([32, 30], 1, 64, 16, False, seed=7)
    q, _ = b.queries([1, 1], 2, "f16")
    lens = torch.tensor([1000, -5], dtype=torch.int32).cuda()
    o = rq.kv4_attention(None, b.cache, q, b.dev_table, lens)
    want = rq.kv4_attention(None, b.cache, q, b.dev_table, torch.tensor([32, 0], dtype=torch.int32).cuda())
    assert torch.equal(o, want) and (o[1] == 0).all()
    o = rq.kv4_attention(None, b.cache, q, b.dev_table, b.dev_lens, max_len=20)
    assert torch.equal(o, rq.kv4_attention(None, b.cache, q, b.dev_table, torch.tensor([20, 20], dtype=torch.int32).cuda()))
    # page numbers that are not in the cache read page 0
    odd = torch.tensor([[1 << 30, -7], [0, 0]], dtype=torch.int32).cuda()
    zero = torch.zeros_like(odd)
    assert torch.equal(rq.kv4_attention(None, b.cache, q, odd, b.dev_lens), rq.kv4_attention(None, b.cache, q, zero, b.dev_lens))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_query_does_not_see_does_not_reach_it(bad):
    """keys and values that are not finite at later positions, before the window, and behind the sequence"""
    b = Batch([100], 1, 64, 16, True, seed=9)
    q, start = b.queries([100], 2, "bf16")
    clean = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    row = torch.full((1, 1, 64), bad, device="cuda")
    rq.kv4_append(b.h, b.cache, row, row, torch.tensor(b.slots[0][70:71]).cuda())
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    assert torch.equal(o[:70], clean[:70]) and torch.isnan(o[70:]).all()
    windowed = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, window=10)
    assert torch.isfinite(windowed[80:]).all() and torch.isnan(windowed[70:80]).all() and torch.isfinite(windowed[:70]).all()
    short = rq.kv4_attention(b.h, b.cache, q[:70], b.dev_table, torch.tensor([70], dtype=torch.int32).cuda(), torch.tensor([0, 70], dtype=torch.int32).cuda())
    assert torch.equal(short, clean[:70])


def test_queries_of_any_size_and_queries_that_are_not_finite():
    b = Batch([50], 1, 128, 16, True, seed=10)
    q, start = b.queries([6], 1, "bf16")
    q[0] = 0
    q[1] *= 2.0 ** -120
    q[2] *= 2.0 ** 100
    q[3, 0, 5] = float("nan")
    q[4, 0, 6] = float("inf")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    assert torch.isfinite(o[[0, 1, 2, 5]]).all() and torch.isnan(o[3]).all() and torch.isnan(o[4]).all()
    c = reference_of(b.cache)
    v = c.rows(b.slots[0])[1][:, 0]
    for i in (0, 1):                                      # equal weights over the positions seen
        want = v[:45 + i].mean(0)
        assert (abs(o[i, 0].double().cpu().numpy() - want) <= 2.0 ** -8 * abs(want) + (2.0 ** -11 + 2.0 ** -16) * abs(v[:45 + i]).mean(0)).all()


def test_values_of_very_different_size():
    """steps from 2^-30 to 2^20 in one sequence, in rising and in falling order, and rows without a step"""
    d = 64
    for order in (1, -1):
        x = torch.randn(128, 1, d, generator=torch.Generator().manual_seed(2)) * (2.0 ** torch.linspace(-30, 20, 128))[::1, None, None]
        x = x.flip(0) if order < 0 else x
        x[40:50] = 0.5
        cache = rq.kv4_cache(8, 1, d, 16)
        keys = torch.randn(128, 1, d, generator=torch.Generator().manual_seed(3)).cuda()
        rq.kv4_append(None, cache, keys, x.cuda(), torch.arange(128).cuda())
        table = torch.arange(8, dtype=torch.int32).cuda()[None]
        c = reference_of(cache)
        k, v = c.rows(range(128))
        steps = c.steps(range(128))
        q = torch.randn(128, 1, d, generator=torch.Generator().manual_seed(4)).half().cuda()
        # (fp16 results hold up to 65504: a smaller part of the range)
        for dtype in (torch.bfloat16,):
            qq = q.to(dtype)
            o = rq.kv4_attention(None, cache, qq, table, torch.tensor([128], dtype=torch.int32).cuda(), torch.tensor([0, 128], dtype=torch.int32).cuda())
            w, _, bound = ref.attention(qq.double().cpu().numpy(), k, v, steps, 1 / 8)
            # besides: p * step below 2^-14 of its range is rounded to 2^-24, i.e. 2^-31 of the largest step times its 7.5
            rest = 128 * 8 * 2.0 ** -30 * np.maximum.accumulate(abs(v[:, 0]).max(-1))[:, None, None] / 7.5
            assert (abs(o.double().cpu().numpy() - w) <= bound * 1.01 + 2.0 ** -8 * abs(w) + rest).all()


@pytest.mark.parametrize("pad", [8, 1])
def test_strided_queries_and_results(pad):
    b = Batch([77, 40], 2, 128, 16, True, seed=11)
    q, start = b.queries([5, 3], 4, "f16")
    want = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    wide = torch.zeros(8, 7, 128 + pad, dtype=torch.float16, device="cuda")
    wide[:, 1:5, pad:] = q
    out = torch.full((8, 6, 128 + pad), 7.0, dtype=torch.float16, device="cuda")
    rq.kv4_attention(b.h, b.cache, wide[:, 1:5, pad:], b.dev_table, b.dev_lens, start, out=out[:, 2:, pad:])
    assert torch.equal(out[:, 2:, pad:], want) and (out[:, :2] == 7).all() and (out[:, :, :pad] == 7).all()


def test_scale_and_equal_rows():
    """with a large scale each query finds its own key; heads of a group share keys and values"""
    b = Batch([64], 1, 128, 64, False, seed=12)
    k, v = reference_of(b.cache).rows(b.slots[0])
    q = torch.tensor(k[:, :1] / np.linalg.norm(k[:, :1], axis=-1, keepdims=True) * 8).bfloat16().cuda().expand(64, 3, 128)
    o = rq.kv4_attention(None, b.cache, q, b.dev_table, b.dev_lens, torch.tensor([0, 64], dtype=torch.int32).cuda(), scale=20.0, causal=False)
    assert torch.equal(o[:, 0], o[:, 1]) and torch.equal(o[:, 0], o[:, 2])
    b.check(q[:, :1].contiguous(), [64], o[:, :1], scale=20.0, causal=False)


def test_offsets_beyond_four_gigabytes():
    page_bytes = binding.kv4_page_bytes(8, 128, 256)
    pages = (9 << 30) // page_bytes
    data = torch.empty((pages, page_bytes), dtype=torch.uint8, device="cuda")
    big, small = rq.KV4Cache(data, 8, 128, 256), rq.kv4_cache(2, 8, 128, 256)
    rng = np.random.default_rng(13)
    k, _ = rows(rng, 300, 8, 128, "bf16")
    v, _ = rows(rng, 300, 8, 128, "bf16")
    h, far = rq.hadamard_build(128), [pages - 1, pages // 2 + 1]
    slots = torch.arange(300).cuda()
    rq.kv4_append(h, small, k, v, slots)
    rq.kv4_append(h, big, k, v, torch.tensor(far).cuda()[slots // 256] * 256 + slots % 256)
    assert torch.equal(data[far[0]], small.data[0])
    q = torch.randn(1, 8, 128, device="cuda", dtype=torch.bfloat16)
    n = torch.tensor([300], dtype=torch.int32).cuda()
    a = rq.kv4_attention(h, small, q, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), n)
    assert torch.equal(a, rq.kv4_attention(h, big, q, torch.tensor([far], dtype=torch.int32).cuda(), n))
    rq.kv4_copy_pages(big, torch.tensor([far[0]], dtype=torch.int32).cuda(), torch.tensor([pages - 2], dtype=torch.int32).cuda())
    assert torch.equal(data[pages - 2], small.data[0])
    for x, y in zip(rq.kv4_read(h, big, torch.tensor([(pages - 2) * 256 + 7]).cuda()), rq.kv4_read(h, small, slots[7:8])):
        assert torch.equal(x, y)


# ---- streams and graphs

def test_another_stream():
    b = Batch([500, 30], 2, 128, 16, True, seed=14)
    q, start = b.queries([1, 1], 8, "bf16")
    want = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, stream=s) for _ in range(20)]
    junk = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(20)]     # the current stream's memory is not the call's
    k, v = rq.kv4_read(b.h, b.cache, torch.tensor(b.slots[0]).cuda(), stream=s)
    s.synchronize()
    assert all(torch.equal(o, want) for o in outs) and junk
    wk, wv = rq.kv4_read(b.h, b.cache, torch.tensor(b.slots[0]).cuda())
    assert torch.equal(k, wk) and torch.equal(v, wv)


def test_a_decode_step_in_a_graph():
    b = Batch([900, 64, 17], 2, 128, 16, True, seed=15, spare=4)
    q, _ = b.queries([1, 1, 1], 8, "bf16")
    k, _ = rows(b.rng, 3, 2, 128, "bf16")
    v, _ = rows(b.rng, 3, 2, 128, "bf16")
    slots, out = torch.full((3,), -1).cuda(), torch.empty_like(q)
    lens = b.dev_lens.clone()

    def step():
        rq.kv4_append(b.h, b.cache, k, v, slots)
        rq.kv4_attention(b.h, b.cache, q, b.dev_table, lens, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        slots[0] = int(b.slots[0][899 - i])
        lens[1] = 64 - i
        k.normal_()
        q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        assert torch.equal(got, out)


# ---- refusals of the binding

def test_binding_refuses():
    b = Batch([20, 10], 2, 128, 16, True, seed=16)
    q, start = b.queries([1, 1], 4, "bf16")
    k = torch.randn(2, 2, 128, device="cuda")
    slots = torch.tensor([0, 1]).cuda()

    def bad(kind, f, *a, **kw):
        with pytest.raises(kind):
            f(*a, **kw)

    attend = lambda **kw: rq.kv4_attention(*[kw.pop(n, v) for n, v in (("h", b.h), ("cache", b.cache), ("q", q), ("table", b.dev_table),  # noqa: E731
                                                                       ("lens", b.dev_lens), ("start", None))], **kw)
    for kw in (dict(q=q.cpu()), dict(q=q[:, :, :64]), dict(q=q[:, :3]), dict(q=q.transpose(1, 2)), dict(table=b.dev_table.long()), dict(table=b.dev_table[0]),
               dict(lens=b.dev_lens.long()), dict(lens=b.dev_lens[:1]), dict(start=start[:2]), dict(start=start.cpu()), dict(q=q[:1]),
               dict(out=torch.empty(2, 4, 128, device="cuda")), dict(out=torch.empty(2, 4, 64, device="cuda", dtype=torch.bfloat16)),
               dict(lse=torch.empty(2, 4)), dict(lse=torch.empty(2, 3, device="cuda")), dict(scale=-1.0), dict(window=-1), dict(max_len=-1),
               dict(h=rq.hadamard_build(64)), dict(table=b.dev_table.t().contiguous().t())):
        bad((ValueError, rq.RotqError), attend, **kw)
    bad((TypeError, rq.RotqError), attend, q=q.double())
    bad(rq.RotqError, attend, q=q.float())
    ok = rq.kv4_append
    for args in ((k.cpu(), k, slots), (k, k[:1], slots), (k, k.half(), slots), (k[:, :1], k[:, :1], slots), (k, k, slots[:1]), (k, k, slots.int()),
                 (k, k, slots.cpu()), (k[..., :64], k[..., :64], slots), (k[0], k[0], slots)):
        bad(ValueError, ok, b.h, b.cache, *args)
    bad(rq.RotqError, ok, b.h, b.cache, k, k, slots, clip=0.0)
    layers = rq.kv4_cache(2, 2, 128, 16, layers=2)
    bad(ValueError, ok, b.h, layers, k, k, slots)
    bad(ValueError, rq.kv4_read, b.h, b.cache, slots.int())
    bad(ValueError, rq.kv4_read, b.h, b.cache, slots, k=torch.empty(2, 2, 64, device="cuda"))
    bad(ValueError, rq.kv4_read, b.h, b.cache, slots, out_dtype=torch.float64)
    bad(ValueError, rq.kv4_copy_pages, b.cache, slots, slots)
    bad(ValueError, rq.kv4_copy_pages, b.cache, slots.int(), slots[:1].int())
    for dims in itertools.islice(((2, 64, 16), (2, 128, 32), (3, 128, 16)), 3):
        with pytest.raises(ValueError):
            rq.KV4Cache(b.cache.data, *dims)

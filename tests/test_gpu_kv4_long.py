"""Attention over the 4-bit cache where its work is shared: long sequences, many row tiles, many workgroups."""
import numpy as np
import pytest
import torch

import kv4_reference as ref
import paper_2504_13989_amd as rq
from test_gpu_kv4 import CASES, U_OUT, Batch, reference_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group,dtype", [(128, 1, "bf16"), (128, 8, "f16"), (128, 16, "bf16"), (64, 4, "bf16")])
def test_results_do_not_go_by_the_sums_asked_for(d, group, dtype):
    lens = [7001, 40, 3333, 2600]
    b = Batch(lens, 2, d, 64, True, seed=11)
    q, _ = b.queries([1] * 4, 2 * group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    plain = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens)
    for _ in range(8):
        assert torch.equal(plain, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, lse=lse))
    b.check(q, [1] * 4, plain, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens,counts,kv,group,d,page,window", [
    ([1500], [1500], 8, 2, 64, 64, 0),           # 192 row tiles: two groups of waves, some with one tile of keys, some with 24
    ([700, 300], [700, 300], 16, 2, 64, 16, 0),
    ([300, 64, 1], [300, 64, 1], 28, 3, 64, 32, 100),
    ([1000, 333], [1000, 200], 12, 2, 128, 64, 0),
    ([2100], [2100], 10, 2, 128, 16, 70),        # eight waves
    ([1100, 900], [1100, 700], 24, 2, 64, 64, 0),
])
def test_many_workgroups(dtype, lens, counts, kv, group, d, page, window):
    b = Batch(lens, kv, d, page, True, seed=21)
    q, start = b.queries(counts, kv * group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, window=window, lse=lse)
    b.check(q, counts, o, lse, window=window)


@pytest.mark.parametrize("dtype,first", [("bf16", 0), ("bf16", 1), ("f16", 0)])      # (fp16 has no results of 2^-60 to begin with)
def test_tiles_of_very_different_size(dtype, first):
    """Every other 64 keys have values 2^-60 times the others': the groups that share a row's tiles have ranges of their own."""
    d, page, kv, n = 64, 64, 9, 1450
    b = Batch([n], kv, d, page, False, seed=22)
    v = torch.randn(n, kv, d, device="cuda")
    tile = torch.arange(n, device="cuda") // 64 % 2 == first
    v *= torch.where(tile, 2.0 ** 40, 2.0 ** -20)[:, None, None]
    k = torch.randn(n, kv, d, device="cuda") * 0.5
    rq.kv4_append(None, b.cache, k, v, torch.tensor(b.slots[0]).cuda())
    q, start = b.queries([n], 2 * kv, "bf16")
    if dtype == "bf16":
        b.check(q, [n], rq.kv4_attention(None, b.cache, q, b.dev_table, b.dev_lens, start))
    else:                                         # (results past fp16's range: only values of one size, small ones)
        v = torch.randn(n, kv, d, device="cuda") * torch.where(tile, 1.0, 2.0 ** -60)[:, None, None]
        rq.kv4_append(None, b.cache, k, v, torch.tensor(b.slots[0]).cuda())
        b.check(q.half(), [n], rq.kv4_attention(None, b.cache, q.half(), b.dev_table, b.dev_lens, start))


def test_example():
    """The example's branches against the model without a cache.  A row's 16 levels over 2 max |y| (some 5 deviations for 128 elements) are a third
    of a deviation apart: a rounding of 0.1 deviations, in keys and values; two layers of them, sums of residuals."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "kv4_generate.py")
    spec = importlib.util.spec_from_file_location("kv4_generate", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    far, size = example.main()
    assert size == 2 * 136 and set(far) == {"a", "b", "keys"}
    assert far["keys"] < 0.13 and far["a"] < 0.2 and far["b"] < 0.2


class Wide(Batch):
    """A batch with a table of so many columns, most of them not used, that it is taken for a large one: the kernel for many rows."""

    def __init__(self, *args, columns, **more):
        super().__init__(*args, **more)
        table = torch.full((len(self.lens), columns), -1, dtype=torch.int32, device="cuda")
        table[:, :self.table.shape[1]] = self.dev_table
        self.dev_table = table


MANY = [i for i, c in enumerate(CASES) if sum(c[1]) * c[2] // c[3] // len(c[0]) > 32]


@pytest.mark.parametrize("factor", [1, 64])      # (a row tile and 64 keys a workgroup, and keys in chunks of which most are empty)
@pytest.mark.parametrize("case", MANY)
def test_kernel_for_many_rows(case, factor):
    lens, counts, heads, kv, d, page, rotate, dtype, causal, window = CASES[case]
    tiles = sum(counts) * heads // kv // 16 * kv
    columns = (256 * 256 * 64 // tiles + 64) // page * factor + 64
    b = Wide(lens, kv, d, page, rotate, seed=case, columns=min(columns, (1 << 30) // page))
    q, start = b.queries(counts, heads, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, causal=causal, window=window, lse=lse)
    b.check(q, counts, o, lse, causal=causal, window=window)
    assert torch.equal(o, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, causal=causal, window=window))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens,counts,kv,group,d,page,causal,window", [
    ([1500], [1500], 8, 2, 64, 64, True, 0),      # two groups of waves
    ([700, 300], [700, 300], 16, 2, 64, 16, True, 0),
    ([1000, 333], [1000, 200], 12, 2, 128, 64, False, 0),
    ([2100], [2100], 20, 2, 128, 16, True, 70),   # eight waves
    ([1300], [1300], 32, 2, 64, 64, False, 0),
])
def test_kernel_for_many_rows_and_workgroups(dtype, lens, counts, kv, group, d, page, causal, window):
    """Some tokens of each sequence, the first and the last among them."""
    b = Wide(lens, kv, d, page, True, seed=31, columns=16384 // page)
    q, start = b.queries(counts, kv * group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, causal=causal, window=window, lse=lse)
    c, rng, at = reference_of(b.cache), np.random.default_rng(0), 0
    for i, (n, m) in enumerate(zip(lens, counts)):
        k, v = c.rows(b.slots[i])
        steps = c.steps(b.slots[i])
        for t in {0, m - 1, *rng.integers(0, m, 30).tolist()}:
            seen = n - m + t + 1 if causal else n             # (keys behind a causal query do not count)
            qx = q[at + t:at + t + 1].double().cpu().numpy() @ ref.sylvester(d)
            w, wl, bound = ref.attention(qx, k[:seen], v[:seen], steps[:seen], d ** -0.5, causal, window)
            g = o[at + t:at + t + 1].double().cpu().numpy()
            assert (abs(g - w) <= bound * (1 + U_OUT[dtype]) + U_OUT[dtype] * abs(w)).all(), (i, t)
            assert (abs(lse[at + t].cpu().numpy() - wl[0]) <= 0.05 + 1e-3 * abs(wl[0])).all()
        at += m


def test_kernel_for_many_rows_keeps_to_what_rows_see():
    """Rows that see nothing are zeros, a key or value that is not finite reaches only those that see it."""
    b = Wide([0, 5, 400], 2, 128, 16, True, seed=6, columns=32768)
    counts = [100, 90, 480]                                        # more queries than positions: the first see nothing
    q, start = b.queries(counts, 4, "bf16")
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, lse=lse)
    b.check(q, counts, o, lse)
    none = torch.isinf(lse)
    assert none.any() and (lse[none] < 0).all() and (o[none] == 0).all() and (o[~none] != 0).any()
    k, v = torch.randn(1, 2, 128, device="cuda"), torch.randn(1, 2, 128, device="cuda")
    v[0, 1, 3] = float("inf")
    rq.kv4_append(b.h, b.cache, k, v, torch.tensor([b.slots[2][300]]).cuda())      # position 300, kv head 1
    r = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    first = 190 + 80 + 300                                         # its query sees it first
    assert torch.isfinite(r[:first]).all() and torch.isfinite(r[:, :2]).all() and torch.equal(r[:first], o[:first])
    assert torch.isnan(r[first:, 2:]).all()
    again = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, window=50)
    assert torch.isnan(again[first:first + 50, 2:]).all() and torch.isfinite(again[first + 50:]).all() and torch.isfinite(again[:first]).all()


def test_kernel_for_many_rows_takes_strided_queries():
    b = Wide([300], 2, 64, 32, True, seed=9, columns=65536)
    q, start = b.queries([300], 6, "bf16")
    wide = torch.randn(300, 20, 72, device="cuda").to(torch.bfloat16)
    part = wide[:, 3:15:2, 5:69]                                   # heads two apart, rows that begin anywhere
    part.copy_(q)
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start)
    out = torch.zeros(300, 7, 66, device="cuda").to(torch.bfloat16)
    rq.kv4_attention(b.h, b.cache, part, b.dev_table, b.dev_lens, start, out=out[:, :6, 1:65])
    assert torch.equal(out[:, :6, 1:65], o) and (out[:, 6] == 0).all() and (out[:, :, 0] == 0).all() and (out[:, :, 65] == 0).all()


@pytest.mark.parametrize("d,group,page,dtype,window", [(128, 1, 64, "bf16", 0), (64, 6, 16, "f16", 0), (128, 3, 32, "f16", 40), (64, 13, 64, "bf16", 0)])
def test_many_short_sequences(d, group, page, dtype, window):
    """More row tiles than the chip has room for: a wave each, some with no keys, some with a few tiles of them."""
    lens = np.random.default_rng(3).integers(0, 200, 56).tolist() + [0, 1, 64, 65, 300]
    b = Batch(lens, 14, d, page, True, seed=12)
    q, start = b.queries([1] * len(lens), 14 * group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    o = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, window=window, lse=lse)
    b.check(q, [1] * len(lens), o, lse, window=window)
    assert torch.equal(o, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, start, window=window))

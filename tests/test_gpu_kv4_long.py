"""Attention over the 4-bit cache where its work is shared: long sequences, many row tiles, many workgroups."""
import pytest
import torch

import paper_2504_13989_amd as rq
from test_gpu_kv4 import Batch

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

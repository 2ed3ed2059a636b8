"""GPU: which cached positions are kept, and the kept rows moved together, against their definitions."""
import itertools

import numpy as np
import pytest

import kv4_long_reference as long_ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def check_select(w, lens, keep, sinks=0, recent=0, **kw):
    got = rq.kv4_select(w, ints(lens), keep, sinks, recent, **kw).cpu().numpy()
    x = w.cpu().numpy()
    assert got.shape == w.shape[:-1] + (keep,)
    for at in itertools.product(*map(range, w.shape[:-1])):
        assert got[at].tolist() == long_ref.select(x[at], min(max(lens[at[-2]], 0), w.shape[-1]), keep, sinks, recent), at
    return got


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 1000, 1024, 1025, 4096, 4097, 8192, 9000, 20000, 32768, 33000, 40960, 57344, 57345, 70001])
def test_select(n):
    rng = np.random.default_rng(n)
    w = torch.tensor(np.exp(3 * rng.standard_normal((3, 2, n))), dtype=torch.float32).cuda()
    lens = [n, max(0, n - 3), n // 3]
    for keep in sorted({1, 2, n // 7, n // 2, n - 1, n, n + 5} - {0}):
        check_select(w, lens, keep)
        check_select(w, lens, keep, min(4, keep // 2), keep // 3)


@pytest.mark.parametrize("n", [70, 1500, 5000, 40000])
def test_select_takes_the_lowest_of_equal_ones(n):
    rng = np.random.default_rng(n)
    for values in ([0.0], [1.0, 2.0], [0.0, -0.0, 1.0, -1.0], [float("inf"), float("-inf"), 0.5, float("nan")], [1e-45, 2e-45, 0.0, -1e-45],
                   [3.4e38, -3.4e38, float("nan")]):
        w = torch.tensor(rng.choice(values, (2, 1, n)), dtype=torch.float32).cuda()
        for keep, sinks, recent in ((1, 0, 0), (n // 2, 3, 5), (n - 1, 0, 1), (n // 3, 0, 0), (8, 4, 4)):
            check_select(w, [n, n - 7], keep, sinks, recent)


def test_select_tells_neighbours_apart():
    """numbers one step of fp32 apart, of both signs"""
    u = torch.arange(0x3f800000, 0x3f800000 + 3000, dtype=torch.int32)
    x = u[torch.randperm(3000, generator=torch.Generator().manual_seed(0))].view(torch.float32)
    for y in (x, -x, torch.where(torch.arange(3000) % 2 == 0, x, -x)):
        check_select(y.view(1, 1, -1).cuda(), [3000], 1234)


def test_select_of_layers_strides_and_lengths_out_of_range():
    rng = np.random.default_rng(1)
    buffer = torch.tensor(rng.standard_normal((4, 3, 5, 900)), dtype=torch.float32).cuda()
    w = buffer[1:, :, ::2, 50:850].transpose(0, 1)                   # [3 layers, 3 sequences, 3 heads, 800]
    check_select(w, [800, 1 << 30, -5], 100, 4, 30)
    check_select(w[0], [1, 0, 799], 100, 4, 30)
    index = torch.full((3, 3, 3, 7), 99, dtype=torch.int32, device="cuda")
    assert rq.kv4_select(w, ints([800, 400, 7]), 7, index=index) is index
    assert rq.kv4_select(w, ints([800, 400, 7]), 0).shape == (3, 3, 3, 0)
    assert (rq.kv4_select(w[..., :0], ints([0, 3, 7]), 2) == -1).all()


def test_select_refuses():
    w, lens = torch.zeros((2, 3, 50), device="cuda"), ints([50, 50])
    for bad in (dict(keep=-1), dict(keep=4, sinks=3, recent=2), dict(keep=4, sinks=-1), dict(keep=4, recent=-1), dict(keep=1 << 31)):
        with pytest.raises(rq.RotqError):
            rq.kv4_select(w, lens, **bad)
    for weights, n, index in ((w.double(), lens, None), (w.cpu(), lens, None), (w[0], lens, None), (w, lens[:1], None), (w, lens.long(), None),
                              (w.transpose(1, 2), lens, None), (w, lens, torch.zeros((2, 3, 5), dtype=torch.int32, device="cuda")),
                              (w, lens, torch.zeros((2, 3, 4), dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            rq.kv4_select(weights, n, 4, index=index)


# ---- evict

def filled(rng, pages, kv, d, page, layers):
    """A cache of random rows (every slot another) as values: [layers][slot][head]"""
    cache = rq.kv4_cache(pages, kv, d, page, layers)
    for i in range(layers):
        x = torch.tensor(rng.standard_normal((2, pages * page, kv, d)), dtype=torch.float32).cuda()
        rq.kv4_append(None, cache.layer(i), x[0], x[1], torch.arange(pages * page).cuda())
    return cache


def values(cache):
    """[layers, slots, 2, heads, d]"""
    slots = torch.arange(cache.pages * cache.page_size).cuda()
    return torch.stack([torch.stack(rq.kv4_read(None, cache.layer(i), slots, out_dtype=torch.float32), 1) for i in range(cache.layers)]).cpu()


def expected(before, index, table, to, page, pages):
    """What the slots hold afterwards; index [layers][batch][heads][keep]"""
    after = before.clone()
    for layer, b, y in itertools.product(*map(range, index.shape[:3])):
        for i, at in enumerate(index[layer, b, y].tolist()):
            if at < 0 or at // page >= table.shape[1] or i // page >= to.shape[1]:
                continue
            src, dst = int(table[b, at // page]), int(to[b, i // page])
            if 0 <= src < pages and 0 <= dst < pages:
                after[layer, dst * page + i % page, :, y] = before[layer, src * page + at % page, :, y]
    return after


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d,page,kv,layers", [(128, 64, 2, 1), (64, 16, 3, 2), (128, 16, 1, 3), (64, 256, 2, 1), (128, 32, 5, 1), (64, 16, 43, 2), (128, 64, 67, 2)])
@pytest.mark.parametrize("lens,keep", [([300, 17, 0, 120], 100), ([1, 500], 1), ([260, 260, 259], 16), ([400], 399), ([300, 300], 129)])
def test_evict(in_place, d, page, kv, layers, lens, keep):
    rng = np.random.default_rng(d + keep)
    need = [max(1, -(-n // page)) for n in lens]
    fresh = -(-keep // page)
    pages = sum(need) + len(lens) * fresh + 2
    order, at = rng.permutation(pages), 0
    table = np.full((len(lens), max(need + [fresh])), -1)
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    to = order[at:at + len(lens) * fresh].reshape(len(lens), fresh)
    index = np.full((layers, len(lens), kv, keep), -1)
    for layer, b, y in itertools.product(range(layers), range(len(lens)), range(kv)):
        kept = np.sort(rng.choice(lens[b], min(keep, lens[b]), replace=False))
        index[layer, b, y, :len(kept)] = kept
    cache = filled(rng, pages, kv, d, page, layers)
    before = values(cache)
    n = keep + 37
    w = torch.tensor(rng.uniform(0, 1, (layers, len(lens), kv, max(n, max(lens)))), dtype=torch.float32).cuda()
    moved = torch.zeros_like(w)
    for layer, b, y in itertools.product(range(layers), range(len(lens)), range(kv)):
        kept = index[layer, b, y]
        kept = torch.tensor(kept[kept >= 0]).cuda()
        moved[layer, b, y, :len(kept)] = w[layer, b, y, kept]
    new = None if in_place else ints(to.tolist())
    rq.kv4_evict(cache, ints((index if layers > 1 else index[0]).tolist()), ints(table.tolist()), new_table=new, weights=w if layers > 1 else w[0])
    assert torch.equal(values(cache), expected(before, index, table, table if in_place else to, page, pages))
    assert torch.equal(w, moved)


@pytest.mark.parametrize("in_place", [True, False])
def test_evict_leaves_rows_without_a_place(in_place):
    """negative and too large positions in the middle, page numbers that are none"""
    rng = np.random.default_rng(2)
    cache = filled(rng, 12, 2, 64, 16, 1)
    before, table, to = values(cache), np.array([[3, -1, 5, 99], [0, 1, 2, 4]]), np.array([[7, 8, -4], [9, 1 << 20, 10]])
    index = np.full((1, 2, 2, 40), -1)
    index[0, :, :, :] = np.arange(40) + np.array([[[5], [24]], [[0], [9]]])
    index[0, 0, 0, 7], index[0, 1, 1, 3], index[0, 1, 1, 39] = -1, -(1 << 31), (1 << 31) - 1
    rq.kv4_evict(cache, ints(index[0].tolist()), ints(table.tolist()), new_table=None if in_place else ints(to.tolist()))
    assert torch.equal(values(cache), expected(before, index, table, table if in_place else to, 16, 12))


def test_evict_into_other_pages_in_any_order():
    """positions in no order, and the same one again"""
    rng = np.random.default_rng(4)
    cache = filled(rng, 30, 2, 128, 32, 2)
    before, table, to = values(cache), np.arange(20).reshape(2, 10), np.arange(20, 30).reshape(2, 5)
    index = rng.integers(0, 320, (2, 2, 2, 150))
    rq.kv4_evict(cache, ints(index.tolist()), ints(table.tolist()), new_table=ints(to.tolist()))
    assert torch.equal(values(cache), expected(before, index, table, to, 32, 30))


def test_evict_of_what_stays_where_it_is():
    cache = filled(np.random.default_rng(3), 6, 2, 128, 16, 1)
    before, index = cache.data.clone(), torch.arange(50, dtype=torch.int32).expand(1, 2, 50).contiguous().cuda()
    w = torch.rand((1, 2, 96), device="cuda")
    old = w.clone()
    rq.kv4_evict(cache, index, ints([[5, 1, 3, 0, 2, 4]]), weights=w)
    assert torch.equal(cache.data, before) and torch.equal(w[..., :50], old[..., :50]) and (w[..., 50:] == 0).all()


def test_evict_of_nothing():
    cache = filled(np.random.default_rng(4), 2, 2, 64, 16, 1)
    before, w = cache.data.clone(), torch.rand((1, 2, 30), device="cuda")
    none = torch.zeros((1, 2, 0), dtype=torch.int32, device="cuda")
    rq.kv4_evict(cache, none, ints([[0, 1]]))
    rq.kv4_evict(cache, none, ints([[0, 1]]), weights=w)
    rq.kv4_evict(cache, none[:0], ints([[0, 1]])[:0])
    assert torch.equal(cache.data, before) and (w == 0).all()


def test_evict_in_a_graph_and_on_another_stream():
    rng = np.random.default_rng(5)
    cache = filled(rng, 8, 2, 128, 64, 2)
    start, table = cache.data.clone(), ints([[0, 3, 2, 1], [7, 5, 4, 6]])
    weights = torch.rand((2, 2, 2, 256), device="cuda")
    first, lens = weights.clone(), ints([256, 200])
    index = rq.kv4_select(weights, lens, 90, 4, 20)
    rq.kv4_evict(cache, index, table, weights=weights)
    want = cache.data.clone(), weights.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        i = rq.kv4_select(weights, lens, 90, 4, 20)
        rq.kv4_evict(cache, i, table, weights=weights)
    s = torch.cuda.Stream()
    for k in range(3):
        cache.data.copy_(start), weights.copy_(first)
        if k < 2:
            g.replay()
        else:
            s.wait_stream(torch.cuda.current_stream())
            j = rq.kv4_select(weights, lens, 90, 4, 20, stream=s)
            rq.kv4_evict(cache, j, table, weights=weights, stream=s)
            s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(cache.data, want[0]) and torch.equal(weights, want[1])


def test_evict_refuses():
    cache, index, table = rq.kv4_cache(6, 2, 64, 16), torch.zeros((1, 2, 20), dtype=torch.int32, device="cuda"), ints([[0, 1]])
    w = torch.zeros((1, 2, 20), device="cuda")
    for bad in (dict(index=index.long()), dict(index=index.cpu()), dict(index=index[:, :1]), dict(index=index[None].expand(2, 1, 2, 20).contiguous()),
                dict(index=index[..., ::2]), dict(table=table.long()), dict(table=table[:0]), dict(new_table=table.long()), dict(new_table=ints([[2, 3], [4, 5]])),
                dict(weights=w.double()), dict(weights=w[..., :19]), dict(weights=w[:, :1]), dict(weights=w[None].expand(2, 1, 2, 20)), dict(weights=w.cpu())):
        with pytest.raises(ValueError):
            rq.kv4_evict(**{**dict(cache=cache, index=index, table=table), **bad})
    for bad in (dict(table=ints([[0]])), dict(new_table=ints([[2]])), dict(weights=w[:, :1].expand(1, 2, 20))):
        with pytest.raises(rq.RotqError):
            rq.kv4_evict(**{**dict(cache=cache, index=index, table=table), **bad})

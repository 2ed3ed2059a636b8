"""GPU: eviction of more positions than a workgroup moves at once: stretches that follow one another, sources that are looked up for the next ones,
long rows of weights, against their definitions."""
import numpy as np
import pytest

from test_gpu_kv4_evict import filled, ints

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402

pytestmark = pytest.mark.gpu


def values(cache):
    """[layers, slots, 2, heads, d]"""
    slots = torch.arange(cache.pages * cache.page_size).cuda()
    return torch.stack([torch.stack(rq.kv4_read(None, cache.layer(i), slots, out_dtype=torch.bfloat16), 1) for i in range(cache.layers)])


def expected(before, w, index, table, to, page):
    """(what the slots hold afterwards, the weights); index [layers][batch][heads][keep]"""
    after, moved = before.clone(), torch.zeros_like(w)
    at = torch.tensor(index).cuda()
    layer, b, y, i = torch.nonzero(at >= 0, as_tuple=True)
    src = at[layer, b, y, i]
    table, to = torch.tensor(table).cuda(), torch.tensor(to).cuda()
    after[layer, to[b, i // page] * page + i % page, :, y] = before[layer, table[b, src // page] * page + src % page, :, y]
    moved[layer, b, y, i] = w[layer, b, y, src]
    return after, moved


# (64 rows, of heads, sequences and layers, and fewer are moved by four workgroups each, 512 positions at once; more rows by one, 128 at once, sources
# looked up for 512; weights 4096 at once in place, 2048 into other pages)
ROWS = [(128, 64, 2, 1), (64, 16, 1, 2), (128, 16, 3, 1), (64, 256, 2, 1), (64, 16, 35, 1), (128, 32, 33, 1), (128, 256, 2, 17), (64, 64, 67, 1)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("keep,drop", [(513, "few"), (513, "last"), (1025, "half"), (1700, "few"), (1700, "first"), (1700, "half"), (4099, "few")])
@pytest.mark.parametrize("d,page,kv,layers", ROWS)
def test_evict_stretch_after_stretch(in_place, keep, drop, d, page, kv, layers):
    rng = np.random.default_rng(keep + d + page)
    batch = 2
    lens = [keep + {"few": 5, "half": keep, "first": 130, "last": 40}[drop], max(1, keep - 70)]      # the second one keeps all
    need, fresh = [max(-(-n // page), -(-keep // page)) for n in lens], -(-keep // page)
    pages = sum(need) + batch * fresh + 1
    order = rng.permutation(pages)
    table = np.zeros((batch, max(need)), np.int64)
    table[0, :need[0]], table[1, :need[1]] = order[:need[0]], order[need[0]:sum(need)]
    to = order[sum(need):sum(need) + batch * fresh].reshape(batch, fresh)
    index = np.full((layers, batch, kv, keep), -1)
    for layer in range(layers):
        for y in range(kv):
            n = lens[0]
            if drop == "first":                   # all of a stretch's sources in later ones
                kept = np.arange(n - keep, n)
            elif drop == "last":
                kept = np.arange(keep)
            else:                                 # few: what a stretch writes touches what the next one reads
                kept = np.sort(rng.choice(n, keep, replace=False))
            index[layer, 0, y] = kept
            index[layer, 1, y, :lens[1]] = np.arange(lens[1])
    cache = filled(rng, pages, kv, d, page, layers)
    before = values(cache)
    w = torch.tensor(rng.uniform(0, 1, (layers, batch, kv, max(lens) + 37)), dtype=torch.float32).cuda()
    want, moved = expected(before, w, index, table, table if in_place else to, page)
    rq.kv4_evict(cache, torch.tensor(index if layers > 1 else index[0], dtype=torch.int32).cuda(), ints(table.tolist()), new_table=None if in_place else ints(to.tolist()),
                 weights=w if layers > 1 else w[0])
    assert torch.equal(w, moved)
    assert torch.equal(values(cache), want)


@pytest.mark.parametrize("in_place", [True, False])
def test_rows_of_weights_longer_than_are_moved_at_once(in_place):
    """twice round the loop and a remainder, alone of several heads; rows without a source among them"""
    rng = np.random.default_rng(1)
    keep, n, page = 8300, 13001, 256
    index = np.stack([np.sort(rng.choice(n, keep, replace=False)) for _ in range(3)])[None, None]
    index[0, 0, 1, rng.choice(keep, 50, replace=False)] = -1
    cache = filled(rng, 86, 3, 64, page, 1)
    table, to = rng.permutation(86)[None], None
    table, to = table[:, :51], table[:, 51:84]
    before = values(cache)
    w = torch.tensor(rng.uniform(0, 1, (1, 1, 3, n)), dtype=torch.float32).cuda()
    want, moved = expected(before, w, index, table, table if in_place else to, page)
    rq.kv4_evict(cache, ints(index[0].tolist()), ints(table.tolist()), new_table=None if in_place else ints(to.tolist()), weights=w[0])
    assert torch.equal(w, moved)
    assert torch.equal(values(cache), want)

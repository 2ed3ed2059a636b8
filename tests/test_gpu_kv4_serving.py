"""GPU: the 4-bit cache's operators for long contexts one after the other, as a server uses them: a prompt, branches off it, decode steps that read
what the branches share once, the attention that positions receive, the positions that are kept, and further steps on these."""
import math

import numpy as np
import pytest

import kv4_long_reference as long_ref
import kv4_reference as ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402

pytestmark = pytest.mark.gpu

LAYERS, DECAY = 2, 0.98
U_OUT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


class Server:
    def __init__(self, heads, kv, d, page, dtype):
        self.heads, self.kv, self.d, self.page, self.dtype = heads, kv, d, page, dtype
        self.pool, self.cache, self.h = rq.PagePool(160, page), rq.kv4_cache(160, kv, d, page, LAYERS), rq.hadamard_build(d)
        self.g = torch.Generator(device="cuda").manual_seed(d)
        self.turn = ref.sylvester(d)

    def random(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda").to(self.dtype)

    def tables(self, seqs, first=0):
        tables = [self.pool.table(s)[first:] for s in seqs]
        width = max(map(len, tables)) + 1
        return ints([t + [-1] * (width - len(t)) for t in tables])

    def lens(self, seqs, first=0):
        return ints([self.pool.length(s) - first * self.page for s in seqs])

    def append(self, seqs, n):
        """n random tokens each"""
        slots, copies = [], []
        for s in seqs:
            new, pairs = self.pool.extend(s, n)
            slots += new
            copies += pairs
        if copies:
            src, dst = torch.tensor(copies, dtype=torch.int32).t().contiguous().cuda()
            rq.kv4_copy_pages(self.cache, src, dst)
        for i in range(LAYERS):
            rq.kv4_append(self.h, self.cache.layer(i), self.random(len(slots), self.kv, self.d), self.random(len(slots), self.kv, self.d), torch.tensor(slots).cuda())

    def rows(self, layer, seq):
        """(keys, values, steps and centres of the keys) of a sequence, as they are stored"""
        c = ref.Pages(0, self.kv, self.d, self.page)
        c.data = self.cache.layer(layer).data.cpu().numpy()
        table = self.pool.table(seq)
        slots = [table[j // self.page] * self.page + j % self.page for j in range(self.pool.length(seq))]
        mids = np.zeros((len(slots), self.kv))
        for i, s in enumerate(slots):
            p, t = divmod(s, self.page)
            for y in range(self.kv):
                w = c.data[p, y * c.block + self.page * self.d + 4 * t + 2:][:2].view(np.uint16).astype(np.uint32) << 16
                mids[i, y] = w.view(np.float32)[0]
        return [*c.rows(slots), c.steps(slots), mids]

    def check(self, layer, seqs, q, start, o, lse, old, new):
        """attention, and what it adds to the weights"""
        x = q.double().cpu().numpy()
        y, got, z, u = x @ self.turn, o.double().cpu().numpy(), lse.double().cpu().numpy(), U_OUT[self.dtype]
        for b, s in enumerate(seqs):
            at = slice(start[b], start[b + 1])
            k, v, steps, mids = self.rows(layer, s)
            want, want_lse, bound = ref.attention(y[at], k, v, steps, self.d ** -0.5)
            assert (abs(got[at] - want) <= bound * (1 + u) + u * abs(want)).all(), s
            assert (abs(z[at] - want_lse) <= 0.05 + 1e-3 * abs(want_lse)).all(), s
            n = len(k)
            before, after = (w[b].double().cpu().numpy() for w in (old, new))
            want, bound = long_ref.weights(before[:, :n], y[at], x[at], k, steps, mids, z[at], self.d ** -0.5, DECAY)
            assert (abs(after[:, :n] - want) <= bound).all(), s
            assert np.array_equal(after[:, n:], before[:, n:]), s


@pytest.mark.parametrize("heads,kv,d,page,dtype", [(8, 2, 128, 16, torch.bfloat16), (6, 6, 64, 64, torch.float16)])
def test_prompt_branches_selection_eviction(heads, kv, d, page, dtype):
    t = Server(heads, kv, d, page, dtype)
    t.pool.add("prompt")
    t.append(["prompt"], 331)
    branches = [0, 1, 2, 3, 4]
    weights = torch.zeros((LAYERS, len(branches), kv, 600), device="cuda")

    # a prompt's last 20 queries count; its branches begin with these weights
    for i in range(LAYERS):
        q, lse, old = t.random(20, heads, d), torch.empty((20, heads), device="cuda"), weights[i].clone()
        start, table, lens = ints([0, 20]), t.tables(["prompt"]), t.lens(["prompt"])
        o = rq.kv4_attention(t.h, t.cache.layer(i), q, table, lens, start, lse=lse)
        rq.kv4_attention_weights(t.h, t.cache.layer(i), q, lse, table, lens, weights[i, :1], start, decay=DECAY)
        t.check(i, ["prompt"], q, [0, 20], o, lse, old, weights[i])
    weights[:, 1:] = weights[:, :1]
    for s in branches:
        t.pool.fork("prompt", s)
    t.pool.free("prompt")
    t.append(branches[1:3], 70)                   # two of them are longer

    def step(check):
        t.append(branches, 1)
        shared = t.pool.common_pages(branches)
        table, lens = t.tables(branches), t.lens(branches)
        for i in range(LAYERS):
            q, lse, old = t.random(len(branches), heads, d), torch.empty((len(branches), heads), device="cuda"), weights[i].clone()
            cache = t.cache.layer(i)
            if shared:
                prefix = ints([t.pool.table(0)[:shared]])
                o = rq.kv4_prefix_attention(t.h, cache, q, prefix, ints([shared * page]), ints([0, len(branches)]), t.tables(branches, shared), t.lens(branches, shared),
                                            lse=lse)
            else:
                o = rq.kv4_attention(t.h, cache, q, table, lens, lse=lse)
            rq.kv4_attention_weights(t.h, cache, q, lse, table, lens, weights[i, :len(branches)], decay=DECAY)
            if check:
                t.check(i, branches, q, list(range(len(branches) + 1)), o, lse, old, weights[i])
        return shared

    for n in range(6):
        assert step(n in (0, 5)) == 331 // page

    def evict(keep, fresh):
        nonlocal branches
        index = rq.kv4_select(weights, t.lens(branches), keep, 4, 16)
        before, old = [[t.rows(i, s) for s in branches] for i in range(LAYERS)], weights.cpu().numpy()
        for i in range(LAYERS):
            for b, s in enumerate(branches):
                for y in range(kv):
                    assert index[i, b, y].tolist() == long_ref.select(old[i, b, y], t.pool.length(s), keep, 4, 16)
        table, new = t.tables(branches), None
        after = branches
        if fresh:                                 # (pages that several hold stay as they are)
            after = ["%s, %d kept" % (s, keep) for s in branches]
            for s, name in zip(branches, after):
                t.pool.add(name)
                t.pool.extend(name, min(keep, t.pool.length(s)))
            new = t.tables(after)
        rq.kv4_evict(t.cache, index, table, new, weights)
        for s, name in zip(branches, after):
            if fresh:
                t.pool.free(s)
            else:
                t.pool.truncate(s, min(keep, t.pool.length(s)))
        branches = after
        moved = weights.cpu().numpy()
        for i in range(LAYERS):
            for b, s in enumerate(branches):
                kept = index[i, b].cpu().numpy()
                n = int((kept[0] >= 0).sum())
                assert t.pool.length(s) == n
                for x, was in zip(t.rows(i, s), before[i][b]):
                    for y in range(kv):
                        assert np.array_equal(x[:, y], was[kept[y, :n], y]), (i, s, y)
                for y in range(kv):
                    assert np.array_equal(moved[i, b, y, :n], old[i, b, y, kept[y, :n]]) and not moved[i, b, y, n:].any()

    evict(150, True)
    src_dst = t.pool.compact()
    if src_dst:
        src, dst = torch.tensor(src_dst, dtype=torch.int32).t().contiguous().cuda()
        rq.kv4_copy_pages(t.cache, src, dst)
    for n in range(6):
        assert step(n in (0, 5)) == 0
    evict(100, False)
    for n in range(3):
        step(n == 2)
    evict(100, False)
    step(True)
    assert [t.pool.length(s) for s in branches] == [101] * 5 and math.isfinite(float(weights.sum()))

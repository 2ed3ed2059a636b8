"""GPU: attention that cached positions receive, against its definition (tests/kv4_long_reference.py, NumPy, 64 bits)."""
import math

import numpy as np
import pytest

import kv4_long_reference as long_ref
import kv4_reference as ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


class Batch:
    """Sequences of `lens` cached positions in shuffled pages, and queries of the last `counts`."""

    def __init__(self, seed, lens, counts, heads, kv, d, page, dtype="bf16", rotate=True, spare=2, width=0):
        rng = np.random.default_rng(seed)
        self.lens, self.counts, self.heads, self.kv, self.d, self.page = lens, counts, heads, kv, d, page
        need = [-(-n // page) for n in lens]
        self.cache = rq.kv4_cache(sum(need) + spare, kv, d, page)
        order = rng.permutation(sum(need) + spare)
        self.h = rq.hadamard_build(d) if rotate else None
        width = max(width, max(need + [1]))
        table = np.full((len(lens), width), -1, np.int64)            # (what stands behind a sequence's pages is no page)
        self.slots, at = [], 0
        for i, (n, m) in enumerate(zip(lens, need)):
            table[i, :m] = order[at:at + m]
            at += m
            j = np.arange(n)
            self.slots.append(table[i, j // page] * page + j % page)
        slots = np.concatenate(self.slots).astype(np.int64)
        k = rng.standard_normal((len(slots), kv, d)) * rng.uniform(0.5, 2, (len(slots), kv, 1)) + 0.3
        k[:, :, 5] *= 6
        k = torch.tensor(k, dtype=torch.float32).cuda()
        rq.kv4_append(self.h, self.cache, k, k, torch.tensor(slots).cuda())
        self.table, self.kv_lens = ints(table.tolist()), ints(list(lens))
        start = [sum(counts[:i]) for i in range(len(counts) + 1)]
        self.start = None if all(c == 1 for c in counts) else ints(start)
        self.q = torch.tensor(rng.standard_normal((sum(counts), heads, d)) * 1.5, dtype=torch.float32).to(DT[dtype]).cuda()
        self.old = torch.tensor(rng.uniform(0, 0.1, (len(lens), kv, width * page)), dtype=torch.float32).cuda()
        self.pages = ref.Pages(0, kv, d, page)
        self.pages.data = self.cache.data.cpu().numpy()

    def lse(self, **kw):
        lse = torch.empty((len(self.q), self.heads), device="cuda")
        rq.kv4_attention(self.h, self.cache, self.q, self.table, self.kv_lens, self.start, lse=lse, **kw)
        return lse

    def weigh(self, lse, weights, **kw):
        rq.kv4_attention_weights(self.h, self.cache, self.q, lse, self.table, self.kv_lens, weights, self.start, **kw)

    def mids(self, slots):
        out = np.zeros((len(slots), self.kv))
        for i, s in enumerate(slots):
            page, t = divmod(int(s), self.page)
            for y in range(self.kv):
                w = self.pages.data[page, y * self.pages.block + self.page * self.d + 4 * t + 2:][:2].view(np.uint16).astype(np.uint32) << 16
                out[i, y] = w.view(np.float32)[0]
        return out

    def check(self, lse, got, old=None, decay=1.0, causal=True, window=0, scale=None):
        """Returns the relative error (2-norm) of what the call adds."""
        got, old, lse = got.double().cpu().numpy(), (self.old if old is None else old).double().cpu().numpy(), lse.double().cpu().numpy()
        x = self.q.double().cpu().numpy()
        q = x if self.h is None else x @ ref.sylvester(self.d)
        at, off, size = 0, 0.0, 0.0
        for b, (n, m) in enumerate(zip(self.lens, self.counts)):
            assert np.array_equal(got[b, :, n:], old[b, :, n:], equal_nan=True)          # behind the last position
            if n:
                k, _ = self.pages.rows(self.slots[b])
                want, bound = long_ref.weights(old[b, :, :n], q[at:at + m], x[at:at + m] if self.h else q[at:at + m], k, self.pages.steps(self.slots[b]),
                                               self.mids(self.slots[b]), lse[at:at + m], scale or self.d ** -0.5, decay, causal, window)
                assert (np.abs(got[b, :, :n] - want) <= bound).all()
                off += ((got[b, :, :n] - want) ** 2).sum()
                size += ((want - decay * np.nan_to_num(old[b, :, :n])) ** 2).sum()
            at += m
        return math.sqrt(off / size) if size else 0.0


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (6, 2), (8, 2), (5, 1), (16, 2), (12, 1), (17, 1), (40, 2)])
@pytest.mark.parametrize("d,page,dtype,rotate", [(128, 64, "bf16", True), (64, 16, "f16", True), (128, 32, "f16", False), (64, 128, "bf16", False)])
def test_one_query_a_sequence(heads, kv, d, page, dtype, rotate):
    t = Batch(heads + d, [1, 0, 63, 64, 65, 200, 331], [1] * 7, heads, kv, d, page, dtype, rotate)
    lse, w = t.lse(), t.old.clone()
    t.weigh(lse, w)
    # (2^-18: an exponent of size 8 is good to 2^-20, its roundings and those of a score's 128 products add up to a few of these)
    assert t.check(lse, w) <= 2.0 ** -18
    # each query's weights add up to 1, as far as its lse is that of the same scores, which attention has to 2^-11 of scale * sum |q| |k|: 50 here at
    # most
    sums = (w - t.old).sum(-1).cpu()
    for b, n in enumerate(t.lens):
        assert (sums[b] - (heads // kv if n else 0)).abs().max() <= 50 * 2.0 ** -11 * heads / kv


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 50), (False, 70), (True, 1000)])
@pytest.mark.parametrize("heads,kv,d,page,dtype,rotate", [(4, 2, 128, 16, "bf16", True), (7, 1, 64, 64, "f16", False), (3, 3, 128, 64, "f16", True)])
def test_many_queries(causal, window, heads, kv, d, page, dtype, rotate):
    # among them a sequence of no positions, one of no queries, one of more queries than positions
    t = Batch(window + d, [150, 0, 70, 9, 64, 257], [150, 3, 0, 20, 64, 5], heads, kv, d, page, dtype, rotate)
    lse, w = t.lse(causal=causal, window=window), t.old.clone()
    t.weigh(lse, w, causal=causal, window=window, decay=0.5)
    assert t.check(lse, w, decay=0.5, causal=causal, window=window) <= 2.0 ** -18


@pytest.mark.parametrize("window", [1, 64, 100])
def test_one_query_with_a_window(window):
    t = Batch(3, [1, 64, 300, 129], [1] * 4, 8, 2, 128, 32)
    lse, w = t.lse(window=window), t.old.clone()
    t.weigh(lse, w, window=window)
    t.check(lse, w, window=window)


def test_decay():
    t = Batch(4, [90, 20], [1, 1], 4, 2, 64, 16)
    lse = t.lse()
    for decay in (0.0, 0.25, 1.0):
        w = t.old.clone()
        t.weigh(lse, w, decay=decay)
        t.check(lse, w, decay=decay)
    old = torch.full_like(t.old, float("nan"))     # not looked at with decay 0
    w = old.clone()
    t.weigh(lse, w, decay=0.0)
    t.check(lse, w, old=old, decay=0.0)
    w = t.old.clone()                              # no queries: the weights decay
    rq.kv4_attention_weights(t.h, t.cache, t.q[:0], lse[:0], t.table, t.kv_lens, w, ints([0, 0, 0]), decay=0.5)
    for b, n in enumerate(t.lens):
        assert torch.equal(w[b, :, :n], t.old[b, :, :n] * 0.5) and torch.equal(w[b, :, n:], t.old[b, :, n:])


def test_steps_add_up():
    """three steps with decay are one sum in 64 bits"""
    t = Batch(5, [130, 77], [1, 1], 4, 1, 128, 64)
    w, want = t.old.clone(), t.old.double()
    for i in range(3):
        t.q = (t.q.float() * 0.9 + 0.1 * i).to(t.q.dtype)
        lse, one = t.lse(), torch.zeros_like(t.old)
        t.weigh(lse, one, decay=0.0)
        t.weigh(lse, w, decay=0.75)
        for b, n in enumerate(t.lens):
            want[b, :, :n] = want[b, :, :n] * 0.75 + one[b, :, :n].double()
    assert ((w.double() - want).abs() <= 3 * 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("counts", [[1, 1, 1], [40, 3, 1]])
def test_long_sequences(counts):
    """several workgroups a sequence, several tiles a wave"""
    t = Batch(6, [3000, 5, 1700], counts, 2, 1, 64, 16, "f16", False)
    lse, w = t.lse(), t.old.clone()
    t.weigh(lse, w)
    t.check(lse, w)


def test_strides_and_short_rows():
    """weights in a wider buffer, heads before sequences; queries as a slice of a fused projection; max_len below the table's pages"""
    t = Batch(7, [100, 64], [1, 1], 4, 2, 128, 16, width=40)
    lse, want = t.lse(), t.old.clone()
    t.weigh(lse, want)
    for pad in (8, 3):
        wide = torch.zeros((2, 8, 128 + pad), dtype=torch.bfloat16, device="cuda")
        wide[:, 2:6, :128] = t.q
        buffer = torch.full((2, 3, 700), -7.0, device="cuda")
        w = buffer[:, 1:, 9:109].transpose(0, 1)
        w[:] = t.old[..., :100]
        rq.kv4_attention_weights(t.h, t.cache, wide[:, 2:6, :128], lse, t.table, t.kv_lens, w, max_len=100)
        assert torch.equal(w, want[..., :100])
        buffer[:, 1:, 9:109] = -7.0
        assert (buffer == -7.0).all()


def test_scale():
    t = Batch(8, [90], [3], 4, 2, 64, 16)
    lse, w = t.lse(scale=0.5), t.old.clone()
    t.weigh(lse, w, scale=0.5)
    t.check(lse, w, scale=0.5)


def test_keys_and_queries_that_are_not_finite():
    t = Batch(9, [150, 80], [4, 4], 2, 1, 64, 16, rotate=False)
    lse = t.lse()
    want = t.old.clone()
    t.weigh(lse, want)
    bad = torch.zeros((1, 1, 64), device="cuda")
    bad[..., 3] = float("inf")
    rq.kv4_append(None, t.cache, bad, bad, torch.tensor([int(t.slots[0][140])]).cuda())
    w = t.old.clone()
    t.weigh(lse, w)                                # one key: its own weight
    nan = torch.isnan(w)
    assert nan[0, 0, 140] and nan.sum() == 1
    assert torch.equal(w[~nan], want[~nan])
    rq.kv4_append(None, t.cache, bad, bad, torch.tensor([int(t.slots[0][149])]).cuda())
    w = t.old.clone()
    t.weigh(lse, w)
    assert torch.isnan(w[0, 0, 149]) and torch.isnan(w).sum() == 2
    # a query: the positions that it sees
    t = Batch(9, [150, 80], [4, 4], 2, 1, 64, 16, rotate=False)
    t.q[1, 0, 7] = float("nan")
    w = t.old.clone()
    t.weigh(lse, w)
    nan = torch.isnan(w)
    assert nan[0, 0, :148].all() and nan.sum() == 148
    assert torch.equal(w[~nan], want[~nan])


def test_the_same_bits_again_and_in_a_graph():
    """two graphs and eager calls in turn; each replay adds the same"""
    a, b = Batch(10, [700, 90], [1, 1], 8, 2, 128, 64), Batch(11, [300, 90], [30, 60], 4, 2, 64, 16)
    graphs, lses, ws = [], [], []
    for t in (a, b):
        lse, w = t.lse(), t.old.clone()
        t.weigh(lse, w.clone())
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            t.weigh(lse, w)
        graphs.append(g), lses.append(lse), ws.append(w)
    for t, w in zip((a, b), ws):
        w.copy_(t.old)
    want = [t.old.clone() for t in (a, b)]
    for _ in range(3):
        for i, t in enumerate((a, b)):
            graphs[i].replay()
            t.weigh(lses[i], want[i])
            torch.cuda.synchronize()
            assert torch.equal(ws[i], want[i])


@pytest.mark.parametrize("shape", [([300, 90], [30, 60], 4, 2, 64, 16), ([900, 500], [300, 400], 8, 2, 128, 64, "f16")])
def test_queries_behind_the_last_sequence_do_not_count(shape):
    t = Batch(14, *shape)
    lse, n = t.lse(), len(t.q)
    t.q = torch.cat([t.q, torch.full((41, t.heads, t.d), float("nan"), dtype=t.q.dtype, device="cuda")])
    lse, w = torch.cat([lse, torch.full((41, t.heads), float("nan"), device="cuda")]), t.old.clone()
    t.weigh(lse, w)
    t.q = t.q[:n]
    assert t.check(lse[:n], w, decay=1.0) <= 2.0 ** -18


def test_two_calls_at_once_and_two_graphs_with_one_workspace():
    t = Batch(15, [900, 500], [300, 400], 8, 2, 128, 64)
    lse, want = t.lse(), t.old.clone()
    t.weigh(lse, want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [t.old.clone() for _ in streams]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for s, w in zip(streams, got):
        t.weigh(lse, w, stream=s)
    for s in streams:
        s.synchronize()
    assert all(torch.equal(w, want) for w in got)
    other = Batch(16, [300, 90], [70, 60], 4, 4, 64, 16, "f16")
    space, graphs, outs, wants = torch.empty(64 << 20, dtype=torch.uint8, device="cuda"), [], [], []
    for b in (t, other):
        lse, w, x = b.lse(), b.old.clone(), b.old.clone()
        b.weigh(lse, x, workspace=space)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.weigh(lse, w, workspace=space)
        graphs.append((g, lse)), outs.append(w), wants.append(x)
    for _ in range(3):
        for b, (g, _), w, x in zip((t, other), graphs, outs, wants):
            w.copy_(b.old)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(w, x)


def test_on_another_stream():
    t = Batch(12, [900, 90], [1, 1], 8, 2, 128, 64)
    lse, want = t.lse(), t.old.clone()
    t.weigh(lse, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    w = t.old.clone()
    s.wait_stream(torch.cuda.current_stream())
    t.weigh(lse, w, stream=s)
    s.synchronize()
    assert torch.equal(w, want)


def test_refusals():
    t = Batch(13, [40, 20], [1, 1], 4, 2, 64, 16)
    lse, w = t.lse(), t.old.clone()
    t.weigh(lse, w)
    for bad in (dict(decay=1.5), dict(decay=-0.1), dict(decay=float("nan")), dict(window=-1), dict(scale=0.0), dict(max_len=-1)):
        with pytest.raises(rq.RotqError):
            t.weigh(lse, w, **bad)
    for weights in (w[:1], w[:, :1], w.double(), w.cpu(), w[..., :20], w[None], w.transpose(1, 2)):
        with pytest.raises(ValueError):
            t.weigh(lse, weights)
    with pytest.raises(rq.RotqError):              # rows that share elements
        t.weigh(lse, w[:, :1].expand(2, 2, -1))
    for other in (lse[:1], lse.double(), lse.cpu(), lse.t()):
        with pytest.raises(ValueError):
            t.weigh(other, w)
    with pytest.raises(ValueError):
        rq.kv4_attention_weights(t.h, t.cache, t.q[:1], lse[:1], t.table, t.kv_lens, w)


#         lens, counts, heads, kv, d, page, window | positions of keys that are not finite and that no query sees, beside others in their block that some do
UNSEEN = [
    ([300], [20], 2, 1, 64, 16, 30, [10, 63, 64, 200, 250]),
    ([700, 513], [100, 3], 4, 2, 128, 64, 200, [300, 383, 400]),
    ([300], [1], 20, 1, 128, 32, 100, [3, 130, 199]),                # (one query, more heads than the kernel for single ones takes)
    ([300], [1], 4, 2, 64, 64, 30, [3, 200, 260, 269]),
    ([900], [1], 7, 1, 128, 16, 600, [70, 290, 299]),
]


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("decay", [0.0, 0.5])
@pytest.mark.parametrize("case", range(len(UNSEEN)))
def test_keys_that_are_not_finite_and_that_no_query_sees(case, decay, value):
    """their weights decay as any that are not seen"""
    *shape, window, at = UNSEEN[case]
    t = Batch(20 + case, *shape, rotate=False)
    lse, want = t.lse(window=window), t.old.clone()
    t.weigh(lse, want, window=window, decay=decay)
    assert t.check(lse, want, decay=decay, window=window) <= 2.0 ** -18
    bad = torch.zeros((len(at), t.kv, t.d), device="cuda")
    bad[..., 3] = value
    rq.kv4_append(None, t.cache, bad, bad, torch.tensor([int(t.slots[0][j]) for j in at]).cuda())
    assert torch.equal(t.lse(window=window), lse)
    w = t.old.clone()
    t.weigh(lse, w, window=window, decay=decay)
    assert torch.equal(w, want)

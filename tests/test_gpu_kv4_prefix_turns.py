"""GPU: attention over shared prefixes of more queries than its workspace holds partial results of: they are taken in turns."""
import ctypes as C

import numpy as np
import pytest

import kv4_reference as ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402
from paper_2504_13989_amd import binding  # noqa: E402

pytestmark = pytest.mark.gpu

MOST = 1 << 30


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def workspace(tokens, heads, kv, d, groups, batch, decode, prefix, own, window=0):
    c = binding.RqKv4(1 << 20, 1 << 20, kv, d, 64)
    return binding.lib().rq_kv4_prefix_attention_workspace(C.byref(c), tokens, heads, groups, batch, decode, window, prefix, own)


def test_workspace_is_bounded():
    """prompts of 64 x 2048 and 8 x 4096 queries behind one prefix, and as many single queries as a call may have"""
    for tokens, heads, kv, d, groups, batch, decode, prefix, own in ((64 * 2048, 64, 8, 128, 1, 64, 0, 8192, 2048), (8 * 4096, 64, 8, 128, 2, 8, 0, 8192, 4096),
                                                                     (1 << 20, 64, 8, 128, 9, 1 << 20, 1, 1000, 100), (1 << 20, 8, 8, 64, 1, 1 << 20, 1, 65536, 4000),
                                                                     (1 << 24, 32, 2, 64, 1, 3, 0, 4096, 1 << 23)):
        need = workspace(tokens, heads, kv, d, groups, batch, decode, prefix, own)
        assert MOST // 4 < need <= MOST, (tokens, need)
    # (what fits is not cut: two chunks of 64 queries each at least)
    assert workspace(64, 32, 8, 128, 1, 64, 1, 8192, 300) % (64 * 32 * 129 * 4) == 0


class Batch:
    """Groups of sequences behind prefixes of whole pages, so that they have whole tables too."""

    def __init__(self, seed, prefix, sizes, lens, counts, heads, kv, d, page, dtype):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.prefix, self.lens, self.counts, self.heads, self.kv, self.d, self.page = prefix, lens, counts, heads, kv, d, page
        self.group = np.repeat(np.arange(len(sizes)), sizes)
        assert all(n % page == 0 for n in prefix) and len(self.group) == len(lens) == len(counts)
        first = np.cumsum([0] + [n // page for n in prefix])
        own = first[-1] + np.cumsum([0] + [-(-n // page) for n in lens])
        order = np.random.default_rng(seed).permutation(own[-1])
        self.h, self.cache = rq.hadamard_build(d), rq.kv4_cache(int(own[-1]), kv, d, page)
        n = int(own[-1]) * page
        for at in range(0, n, 1 << 16):
            slots = torch.arange(at, min(n, at + (1 << 16))).cuda()
            k, v = (torch.randn((len(slots), kv, d), generator=g, device="cuda") + 0.2 for _ in "kv")
            rq.kv4_append(self.h, self.cache, k, v, slots)
        cut = lambda a, width: np.stack([np.r_[order[i:j], np.full(width - (j - i), -1, np.int64)] for i, j in zip(a[:-1], a[1:])])  # noqa: E731
        self.prefix_pages, self.own_pages = cut(first, max(1, int(np.diff(first).max()))), cut(own, max(1, int(np.diff(own).max())))
        self.start = np.cumsum([0] + list(counts))
        self.q = (torch.randn((int(self.start[-1]), heads, d), generator=g, device="cuda") * 1.5).to(dtype)
        self.group_start = np.searchsorted(self.group, np.arange(len(sizes) + 1))

    def ragged(self):
        return None if set(self.counts) == {1} else ints(self.start)

    def attend(self, **kw):
        return rq.kv4_prefix_attention(self.h, self.cache, self.q, ints(self.prefix_pages), ints(self.prefix), ints(self.group_start), ints(self.own_pages), ints(self.lens),
                                       self.ragged(), **kw)

    def plan(self):
        c, p = binding.RqKv4(1 << 20, self.cache.pages, self.kv, self.d, self.page), binding.RqKv4PrefixPlan()
        assert binding.lib().rq_kv4_prefix_attention_plan(C.byref(c), 0 if self.q.dtype == torch.bfloat16 else 2, len(self.q), self.heads, len(self.prefix),
                                                          len(self.lens), int(self.ragged() is None), 0, self.prefix_pages.shape[1] * self.page,
                                                          self.own_pages.shape[1] * self.page, 0, C.byref(p)) == 0
        return p

    def whole_table(self, b):
        g = self.group[b]
        return np.r_[self.prefix_pages[g, :self.prefix[g] // self.page], self.own_pages[b]]

    def whole(self, **kw):
        tables = [self.whole_table(b) for b in range(len(self.lens))]
        width = max(map(len, tables))
        return rq.kv4_attention(self.h, self.cache, self.q, ints([np.r_[t, np.full(width - len(t), -1)] for t in tables]),
                                ints([self.prefix[g] + n for g, n in zip(self.group, self.lens)]), self.ragged(), **kw)

    def steps(self, c, slots, kv):
        """of the keys [slots, kv heads]: the low half of a token's parameters"""
        at = np.array([[y * c.block + self.page * self.d + 4 * (s % self.page) + i for i in (0, 1)] for s in slots for y in kv]).reshape(len(slots), len(kv), 2)
        raw = c.data[(slots // self.page)[:, None, None], at].astype(np.uint32)
        return ((raw[..., 0] | raw[..., 1] << 8) << 16).astype(np.uint32).view(np.float32).astype(np.float64)

    def check(self, o, tokens):
        """some tokens, the first and the last kv head's first queries, against 64 bits"""
        c = ref.Pages(0, self.kv, self.d, self.page)
        c.data = self.cache.data.cpu().numpy()
        u = 2.0 ** -8 if o.dtype == torch.bfloat16 else 2.0 ** -11
        for t in tokens:
            b = int(np.searchsorted(self.start, t, side="right")) - 1
            n = self.prefix[self.group[b]] + self.lens[b] - (self.counts[b] - 1 - (t - self.start[b]))       # positions up to its own
            j = np.arange(n)
            slots = self.whole_table(b)[j // self.page] * self.page + j % self.page
            kv, heads = [0, self.kv - 1], [0, self.heads - self.heads // self.kv]
            k, v = np.array([[c.get(s, y) for y in kv] for s in slots]).transpose(2, 0, 1, 3)
            q = self.q[t:t + 1, heads].double().cpu().numpy() @ ref.sylvester(self.d)
            want, _, bound = ref.attention(q, k, v, self.steps(c, slots, kv), self.d ** -0.5)
            y = o[t:t + 1, heads].double().cpu().numpy()
            assert (abs(y - want) <= bound * (1 + u) + u * abs(want)).all(), t


#         prefix, sizes, lens, counts, heads, kv, d, page, dtype
TURNS = [
    ([192, 64, 128], [9000, 1, 10999], [i % 4 + 1 for i in range(20000)], [1] * 20000, 64, 8, 128, 16, torch.bfloat16),
    ([64], [30011], [i % 3 + 1 for i in range(30011)], [1] * 30011, 72, 72, 64, 16, torch.float16),
    ([128, 64], [3, 2], [5003, 0, 7000, 4001, 2999], [5003, 0, 7000, 4001, 2997], 64, 8, 128, 64, torch.bfloat16),
    ([128], [4001], [i % 9 + 1 for i in range(4001)], [i % 9 + 1 for i in range(4001)], 64, 8, 128, 16, torch.float16),
]


@pytest.mark.parametrize("case", range(len(TURNS)))
def test_in_turns(case):
    b = Batch(case, *TURNS[case])
    tokens, chunk_bytes = len(b.q), len(b.q) * b.heads * (b.d + 1) * 4
    need = workspace(tokens, b.heads, b.kv, b.d, len(b.prefix), len(b.lens), int(b.ragged() is None), b.prefix_pages.shape[1] * b.page, b.own_pages.shape[1] * b.page)
    assert MOST // 4 < need <= MOST < 2 * chunk_bytes
    o, lse = torch.full_like(b.q, 1e4), torch.full(b.q.shape[:2], 1e4, device="cuda")
    b.attend(out=o, lse=lse)
    assert torch.equal(o, b.attend())
    want_lse = torch.empty_like(lse)
    want = b.whole(lse=want_lse)
    # (each is within the bound of kv4_reference of the true result, which is about this; and a rounding each)
    rows, size = (o.float() - want.float()).norm(dim=-1), want.float().norm(dim=-1)
    assert rows.norm() <= 2.0 ** -7 * size.norm()
    # a row of another token would be off by its own size; one row's part of the bound above is far from half of it
    assert (rows <= 0.5 * size).all()
    assert (lse - want_lse).abs().max() <= 0.1 + 2e-3 * want_lse.abs().max()
    # around every token with which a turn begins
    p = b.plan()
    turn = need // ((p.shared_chunks + p.own_chunks) * b.heads * (b.d + 1) * 4)
    assert not p.separate and tokens // 4 < turn < tokens
    b.check(o, sorted({0, tokens - 1, *(t + i for t in range(turn, tokens, turn) for i in (-1, 0))}))

"""GPU: attention over the 4-bit cache in each form that a call can take (rq_kv4_attention_plan says which), in ways that show a tile of
64 keys left out or taken twice."""
import ctypes as C
import math

import numpy as np
import pytest

import kv4_reference as ref

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402
from paper_2504_13989_amd import binding  # noqa: E402

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
CODE = {"bf16": binding.RQ_BF16, "f16": binding.RQ_F16}
U_OUT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


class Filled:
    """Sequences in a cache of their own, shuffled pages; keys and values f(sequence's positions) [n, kv heads, d]."""

    def __init__(self, lens, kv, d, page, rotate, keys, values):
        rng = np.random.default_rng(1)
        need = [-(-n // page) for n in lens]
        self.lens, self.kv, self.d, self.page = lens, kv, d, page
        self.h = rq.hadamard_build(d) if rotate else None
        self.cache = rq.kv4_cache(sum(need) + 1, kv, d, page)
        self.cache.data.fill_(0xFF)                      # slots that nothing is appended to: NaN parameters
        order, at = rng.permutation(sum(need) + 1), 0
        table, self.slots = np.full((len(lens), max(need)), -1, np.int32), []
        for i, (n, m) in enumerate(zip(lens, need)):
            table[i, :m] = order[at:at + m]
            at += m
            pos = np.arange(n)
            self.slots.append(torch.tensor(table[i, pos // page].astype(np.int64) * page + pos % page).cuda())
            t = torch.arange(n, device="cuda")
            rq.kv4_append(self.h, self.cache, keys(t), values(t), self.slots[-1])
        self.table, self.kv_lens = torch.tensor(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()

    def stored(self, i):
        """(keys, values) of sequence i as they are stored, float64 [n, kv heads, d]"""
        return [x.double() for x in rq.kv4_read(None, self.cache, self.slots[i], out_dtype=torch.float32)]

    def steps(self, i):
        """steps of its keys, float64 [n, kv heads]"""
        p, block = self.page, self.page * (self.d + 8)
        data = self.cache.data.view(-1, self.kv, block)[..., p * self.d:p * (self.d + 4)].unflatten(-1, (p, 4))
        s = self.slots[i]
        return data[s // p, :, s % p, :2].contiguous().view(torch.bfloat16)[..., 0].double()

    def run(self, q, counts, causal, window, form=None):
        """(o, lse), after a look at the form that the call takes"""
        start = torch.tensor(np.concatenate(([0], np.cumsum(counts))), dtype=torch.int32).cuda()
        decode = set(counts) == {1}
        if form is not None:
            p = plan(self, q, counts, causal, window)
            got = dict(many=p.many, waves=p.waves, groups=p.groups, shared=p.workers > 0, chunked=p.chunks > 1)
            assert got == {**got, **form}, got
        lse = torch.full(q.shape[:2], float("nan"), device="cuda")
        o = rq.kv4_attention(self.h, self.cache, q, self.table, self.kv_lens, None if decode else start, causal=causal, window=window,
                             max_len=max(self.lens), lse=lse)
        return o, lse


def plan(f, q, counts, causal, window):
    c, p = f.cache, binding.RqKv4Plan()
    cache = binding.RqKv4(c.data.data_ptr(), c.pages, c.kv_heads, c.head_dim, c.page_size)
    code = {v: CODE[k] for k, v in DT.items()}[q.dtype]
    assert binding.lib().rq_kv4_attention_plan(C.byref(cache), code, q.shape[0], q.shape[1], len(counts), int(set(counts) == {1}), int(causal),
                                               window, max(f.lens), 0, C.byref(p)) == binding.RQ_OK
    return p


def ranges(n, m, causal, window):
    """[lo, hi) of the positions that each of m queries at the end of n positions sees"""
    pos = torch.arange(m, device="cuda") + (n - m)
    hi = (pos + 1).clamp(min=0) if causal else torch.full_like(pos, n)
    lo = (pos - window + 1).clamp(min=0) if window else torch.zeros_like(pos)
    return lo, torch.maximum(hi, lo)


def check_coverage(lens, counts, kv, group, d, page, causal, window, dtype, form):
    """Queries of 2^-20: all keys weigh the same, to expm1(2 e), e the largest score that |q| |k| allows.  Tile t's values are 1 in one element and 0
    in the others, so each row's result is the number of its tiles' keys, and the log-sum the number of all.  Values and weights are
    rounded to fp16 (2^-11 each), sums are fp32: a lane adds a 32nd of the keys, to sums below their number."""
    gen = torch.Generator(device="cuda").manual_seed(3)

    def values(t):
        at = (t // 64)[:, None] + 5 * torch.arange(kv, device="cuda")
        return torch.nn.functional.one_hot(at % d, d).float()

    f = Filled(lens, kv, d, page, True, lambda t: torch.randn(len(t), kv, d, generator=gen, device="cuda"), values)
    q = (torch.randn(sum(counts), kv * group, d, generator=gen, device="cuda") * 2.0 ** -20).to(DT[dtype])
    o, lse = f.run(q, counts, causal, window, form)
    at = 0
    for i, (n, m) in enumerate(zip(lens, counts)):
        k, v = f.stored(i)
        lo, hi = ranges(n, m, causal, window)
        count = (hi - lo).double()[:, None, None]
        sums = [torch.cat((torch.zeros_like(x[:1]), x.cumsum(0))) for x in (v, v.abs())]
        want, size = [((s[hi] - s[lo]) / count.clamp(min=1)).repeat_interleave(group, 1) for s in sums]
        e = float(q.double().norm(dim=-1).max() * k.norm(dim=-1).max()) / math.sqrt(d)
        tol = (math.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT[dtype] * want.abs() + n / 32 * 2.0 ** -24
        assert (tol < 16 / count.clamp(min=1)).all()      # a quarter of what one tile of one row adds
        off = (o[at:at + m].double() - want).abs()
        assert (off <= tol).all(), (i, float((off / tol).max()))
        none = (hi == lo)
        assert torch.equal(torch.isinf(lse[at:at + m]), none[:, None].expand(-1, kv * group)) and (o[at:at + m][none] == 0).all()
        off = (lse[at:at + m].double() - count[..., 0].clamp(min=1).log())[~none].abs()
        assert (off <= 2 * e + 1e-5).all(), (i, float(off.max()))
        at += m


def check_values(lens, counts, kv, group, d, page, causal, window, dtype, form):
    """Some rows against 64 bits.  A score is off by the rounding of q and of k to fp16 (2^-11 each) and by sums of codes that carry 1024 in
    fp32 (16 roundings, see kv4_reference.attention): e at most; p and v are rounded to fp16 once each, sums are fp32."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows = lambda t: torch.randn(len(t), kv, d, generator=gen, device="cuda")  # noqa: E731
    f = Filled(lens, kv, d, page, True, rows, rows)
    q = torch.randn(sum(counts), kv * group, d, generator=gen, device="cuda").to(DT[dtype])
    o, lse = f.run(q, counts, causal, window, form)
    hd, at, rng = torch.tensor(ref.sylvester(d)).cuda(), 0, np.random.default_rng(5)
    for i, (n, m) in enumerate(zip(lens, counts)):
        k, v = f.stored(i)
        step, (lo, hi) = f.steps(i), ranges(n, m, causal, window)
        for t in sorted({0, m - 1, *rng.integers(0, m, 12).tolist()}):
            a, b = int(lo[t]), int(hi[t])
            for j in range(kv):
                heads = slice(j * group, (j + 1) * group)
                x = q[at + t, heads].double() @ hd
                s = x @ k[a:b, j].t() / math.sqrt(d)
                e = ((2.0 ** -10 * (x.abs() @ k[a:b, j].abs().t()) + 2.0 ** -10 * step[a:b, j] * x.abs().sum(-1, keepdim=True)) / math.sqrt(d)).amax(-1)
                p, total = torch.softmax(s, -1), torch.logsumexp(s, -1)
                want, size = p @ v[a:b, j], p @ v[a:b, j].abs()
                tol = (torch.expm1(2 * e)[:, None] + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT[dtype] * want.abs()
                off = (o[at + t, heads].double() - want).abs()
                assert (off <= tol).all(), (i, t, j, float((off / tol).max()))
                assert ((lse[at + t, heads].double() - total).abs() <= e + 2.0 ** -11 + 2.0 ** -16 + 2.0 ** -20 * total.abs()).all(), (i, t, j)
        at += m


def form(many, waves, groups=1, shared=False, chunked=False):
    return dict(many=many, waves=waves, groups=groups, shared=shared, chunked=chunked)


# lens, counts, kv heads, group, head_dim, page, causal, window, form
CHUNKS = form(1, 4, chunked=True)
BEHIND = [
    ([8192], [1024], 4, 4, 128, 64, False, 4096, CHUNKS),
    ([8000, 3230], [1500, 900], 2, 4, 128, 16, False, 4096, CHUNKS),
    ([8100], [4814], 2, 2, 64, 128, False, 2000, CHUNKS),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(BEHIND)))
def test_windows_of_queries_that_are_not_causal(case, dtype):
    """With many queries and keys in chunks: all positions from the window's first to the end of the sequence count."""
    check_coverage(*BEHIND[case][:-1], dtype, BEHIND[case][-1])
    check_values(*BEHIND[case][:-1], dtype, BEHIND[case][-1])


@pytest.mark.parametrize("kv,many", [(1, 0), (32, 1)])
def test_windows_of_any_size(kv, many):
    """A window over all positions is none, however large, also where there are more queries than positions."""
    lens, counts = [700, 40], [1400, 900]
    gen = torch.Generator(device="cuda").manual_seed(6)
    rows = lambda t: torch.randn(len(t), kv, 64, generator=gen, device="cuda")  # noqa: E731
    f = Filled(lens, kv, 64, 16, True, rows, rows)
    q = torch.randn(sum(counts), kv * 2, 64, generator=gen, device="cuda").bfloat16()
    for causal in (True, False):
        want, sums = f.run(q, counts, causal, 0, dict(many=many))
        assert torch.isfinite(want).all() and (want != 0).any()
        for window in (700, 1 << 30, (1 << 31) - 1500, (1 << 31) - 1):
            o, lse = f.run(q, counts, causal, window)
            assert torch.equal(o, want) and torch.equal(lse, sums), window


def test_results_that_overlap_are_refused():
    rows = lambda t: torch.randn(len(t), 2, 64, device="cuda")  # noqa: E731
    f = Filled([40, 30], 2, 64, 16, True, rows, rows)
    q = torch.randn(2, 4, 64, device="cuda").half()
    call = lambda q, out: rq.kv4_attention(f.h, f.cache, q, f.table[:len(q)], f.kv_lens[:len(q)], out=out)  # noqa: E731
    want = call(q, None)
    for out in (torch.empty_like(q[:1]).expand(2, 4, 64), torch.empty_like(q[:, :1]).expand(2, 4, 64), torch.empty_like(q).view(-1).as_strided((2, 4, 64), (256, 32, 1))):
        with pytest.raises(rq.RotqError):
            call(q, out)
    turned = torch.empty(4, 2, 64, dtype=torch.float16, device="cuda").transpose(0, 1)           # heads further apart than tokens
    assert torch.equal(call(q, turned), want)
    one = torch.empty(256, dtype=torch.float16, device="cuda").as_strided((1, 4, 64), (0, 64, 1))  # (one token: its stride is never used)
    assert torch.equal(call(q[:1], one), want[:1])


def column(n, at, row, rest):
    """[n, d] rows `rest`, row `at` of them `row`"""
    x = rest.clone()
    x[at] = row
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("at", [0, 8191])
def test_many_small_weights_add_up(at, dtype):
    """One key 17.6 above 8191 others, whose weights of 2^-25.4 make 2^-12 together, all of them a workgroup's.  All numbers but q * scale * log2(e), rounded to fp16, are
    powers of two or exact in fp16; a weight of 2^-18.4 (the largest is 2^7) is rounded to 2^-24."""
    n, d, kv = 8192, 64, 32
    rest = torch.zeros(n, d, device="cuda")
    keys, values = column(n, at, 2.0, rest), column(n, at, 0.0, rest + 1)
    f = Filled([n], kv, d, 64, False, *(lambda t, x=x: x[t][:, None].repeat(1, kv, 1) for x in (keys, values)))
    q = torch.full((1200, 2 * kv, d), 1.1015625, device="cuda").to(DT[dtype])
    o, lse = f.run(q, [1200], False, 0, form(1, 8))
    score = 64 * 2 * 1.1015625 / 8
    want = (n - 1) / (n - 1 + math.exp(score))
    off = math.expm1(score * 2.0 ** -11) + 2.0 ** -25 / 2.0 ** (7 - score / math.log(2)) + U_OUT[dtype]
    assert ((o.double() - want).abs() <= off * want).all(), float(o.double().mean() / want)
    assert ((lse.double() - math.log(n - 1 + math.exp(score))).abs() <= score * 2.0 ** -11 + 1e-4).all()


def reference(f, q, causal, scale=None):
    """(o, log of the sums, sum of p |v|, largest |score|) of a batch of one sequence whose queries are all its last positions, float64"""
    k, v = f.stored(0)
    n, m, group = k.shape[0], q.shape[0], q.shape[1] // f.kv
    seen = ranges(n, m, causal, 0)[1]
    hidden = torch.arange(n, device="cuda")[None] >= seen[:, None]
    x = q.double() @ torch.tensor(ref.sylvester(f.d)).cuda() if f.h else q.double()
    out = []
    for h in range(q.shape[1]):
        s = (x[:, h] @ k[:, h // group].t() / math.sqrt(f.d)).masked_fill(hidden, -math.inf)
        p = torch.softmax(s, -1)
        out.append((p @ v[:, h // group], torch.logsumexp(s, -1), p @ v[:, h // group].abs(), s.masked_fill(hidden, 0).abs().amax(-1)))
    return [torch.stack(y, 1) for y in zip(*out)]


LARGE = {"step": (-1e38, 1e38), "centre": (1.6e38, 1.6e38)}       # (rows whose least + largest element overflows are stored as not finite)


@pytest.mark.parametrize("what", LARGE)
def test_values_up_to_the_end_of_the_range(what):
    """A value row that is finite, however large, makes no result NaN.  What is 2^-40 of it and less is lost beside it (fp16's least number is 2^-24, its largest
    2^16), also for rows that do not see it where it is in a tile that their workgroup comes to."""
    n, kv, d, at = 1300, 32, 64, 700
    gen = torch.Generator(device="cuda").manual_seed(8)
    rows = lambda t: torch.randn(len(t), kv, d, generator=gen, device="cuda")  # noqa: E731
    values = rows(torch.arange(n))
    values[at] = torch.linspace(*LARGE[what], d, device="cuda")
    f = Filled([n], kv, d, 64, False, rows, lambda t: values[t])
    q = torch.randn(n, 2 * kv, d, generator=gen, device="cuda").bfloat16()
    o, lse = f.run(q, [n], True, 0, form(1, 8))
    want, sums, size, most = reference(f, q, True)
    assert torch.isfinite(o).all()
    k, step = f.stored(0)[0].abs().amax(0).repeat_interleave(2, 0), f.steps(0).max()
    e = float(((2.0 ** -10 * (q.double().abs() * k).sum(-1) + 2.0 ** -10 * step * q.double().abs().sum(-1)) / math.sqrt(d)).max())
    tol = (math.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT["bf16"] * want.abs()
    near = torch.arange(n, device="cuda") >= at // 64 * 64            # (rows whose tiles of keys end with the large one's or go on)
    tol = tol + 2.0 ** (128 - 40) * near[:, None, None]
    assert ((o.double() - want).abs() <= tol).all()
    assert ((lse.double() - sums).abs() <= e + 2.0 ** -11 + 2.0 ** -16 + 2.0 ** -20 * sums.abs()).all()


def test_keys_up_to_the_end_of_the_range():
    """A key of 1e38 takes all weight of rows that see it or none (queries of 2^-12: its scores are beyond 1e30, the others' below 0.01); the other
    keys' scores, lost beside it or not, weigh them alike to expm1(2 s), s the largest of them."""
    n, kv, d, at = 1300, 32, 64, 700
    gen = torch.Generator(device="cuda").manual_seed(9)
    rows = lambda t: torch.randn(len(t), kv, d, generator=gen, device="cuda")  # noqa: E731
    keys = rows(torch.arange(n))
    keys[at] = torch.linspace(-1e38, 1e38, d, device="cuda")
    f = Filled([n], kv, d, 64, False, lambda t: keys[t], rows)
    sign = 2.0 * (torch.rand(n, 2 * kv, 1, generator=gen, device="cuda") < 0.5) - 1
    q = sign * torch.linspace(-1, 1, d, device="cuda") + 0.25 * torch.randn(n, 2 * kv, d, generator=gen, device="cuda")
    q = (q * 2.0 ** -12).bfloat16()
    o, lse = f.run(q, [n], True, 0, form(1, 8))
    want, sums, size, _ = reference(f, q, True)
    k = f.stored(0)[0].repeat_interleave(2, 1)
    assert ((q.double() * k[at]).sum(-1).abs() / math.sqrt(d) > 1e30).all()
    k[at] = 0
    s = float(q.double().norm(dim=-1).max() * k.norm(dim=-1).max()) / math.sqrt(d)
    assert s < 0.01
    assert ((o.double() - want).abs() <= (math.expm1(2 * s) + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT["bf16"] * want.abs()).all()
    assert ((lse.double() - sums).abs()[:at] <= s + 2.0 ** -11 + 2.0 ** -16 + 1e-5).all()


SHARED, EIGHT = form(0, 4, shared=True), form(0, 8)


@pytest.mark.parametrize("dtype,n,counts,kv,want_form", [
    ("bf16", 20000, [1], 1, SHARED), ("f16", 20000, [1], 1, SHARED), ("bf16", 1500, [1], 1, EIGHT), ("f16", 1500, [1], 1, EIGHT),
    ("bf16", 900, [300], 32, form(0, 1)), ("f16", 3000, [1300], 32, form(1, 8)), ("bf16", 3000, [1300], 32, form(1, 8))])
def test_sums_do_not_go_by_the_size_of_values(dtype, n, counts, kv, want_form):
    """One key whose score is 10 among others of 0, values of 1e37: a weight of e^-10 is not lost.  (The score is off by the rounding of q * scale *
    log2(e) to fp16; results are compared where their type holds them: p and v are rounded to fp16 besides, or p * step.)"""
    d = 64
    line = torch.linspace(-1e37, 1e37, d, device="cuda")
    keys = lambda t: ((t == 7) * 2.0)[:, None, None].repeat(1, kv, d)  # noqa: E731
    f = Filled([n], kv, d, 64, False, keys, lambda t: torch.where((t == 7)[:, None, None], -line, line).expand(-1, kv, d))
    q = torch.full((sum(counts), 2 * kv, d), 0.625, device="cuda").to(DT[dtype])
    o, lse = f.run(q, counts, False, 0, want_form)
    one, rest = math.exp(10), n - 1
    assert ((lse.double() - math.log(one + rest)).abs() <= 10 * 2.0 ** -11 + 1e-4).all()
    if dtype == "bf16":
        v = f.stored(0)[1]
        want = (v[7, 0] * one + v[8, 0] * rest) / (one + rest)
        tol = (math.expm1(2 * 10 * 2.0 ** -11) + 2.0 ** -10 + 2.0 ** -16) * v[8, 0].abs() + U_OUT[dtype] * want.abs()
        assert ((o.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,n,kv,many", [("bf16", 400, 1, 0), ("f16", 400, 1, 0), ("f16", 1300, 32, 1), ("bf16", 1300, 32, 1)])
def test_log_sums_beside_a_large_value(dtype, n, kv, many):
    """Values of 2^-57 and one of 1e37 behind them: the sums are those of the scores, for rows that see it and for rows that do not."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    d, at = 64, n // 2 + 5
    keys, values = [torch.randn(n, kv, d, generator=gen, device="cuda") for _ in range(2)]
    values *= 2.0 ** -57
    values[at] = torch.linspace(-1e37, 1e37, d, device="cuda")
    f = Filled([n], kv, d, 64, True, lambda t: keys[t], lambda t: values[t])
    q = torch.randn(n, 2 * kv, d, generator=gen, device="cuda").to(DT[dtype])
    o, lse = f.run(q, [n], True, 0, dict(many=many))
    _, sums, _, _ = reference(f, q, True)
    k, step = f.stored(0)[0].abs().amax(0).repeat_interleave(2, 0), f.steps(0).max()
    x = (q.double() @ torch.tensor(ref.sylvester(d)).cuda()).abs()
    e = float(((2.0 ** -10 * (x * k).sum(-1) + 2.0 ** -10 * step * x.sum(-1)) / math.sqrt(d)).max())
    assert ((lse.double() - sums).abs() <= e + 2.0 ** -11 + 2.0 ** -16 + 2.0 ** -20 * sums.abs()).all()
    assert not torch.isnan(o).any()


def test_a_large_centre_beside_small_steps():
    """A flat row of 1e25 among values of 2^-48, which set the factor of sums: nothing overflows."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    n, d, at = 300, 64, 9
    keys, values = [torch.randn(n, 1, d, generator=gen, device="cuda") for _ in range(2)]
    values *= 2.0 ** -48
    values[at] = 1e25
    f = Filled([n], 1, d, 64, False, lambda t: keys[t], lambda t: values[t])
    q = torch.randn(1, 4, d, generator=gen, device="cuda").bfloat16()
    o, lse = f.run(q, [1], True, 0, dict(many=0))
    want, sums, size, _ = reference(f, q, True)
    k, step = f.stored(0)[0].abs().amax(0), f.steps(0).max()
    e = float(((2.0 ** -10 * (q.double().abs() * k).sum(-1) + 2.0 ** -10 * step * q.double().abs().sum(-1)) / math.sqrt(d)).max())
    assert ((o.double() - want).abs() <= (math.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT["bf16"] * want.abs()).all()
    assert ((lse.double() - sums).abs() <= e + 2.0 ** -16 + 2.0 ** -20 * sums.abs()).all()


FORMS = [
    # few rows: keys shared out, 4, 8 and 16 rows a tile; a row tile a workgroup of eight, four waves and of one
    ([8192], [1], 2, 4, 128, 64, True, 0, SHARED),
    ([8000, 100, 3000], [1] * 3, 1, 1, 64, 16, True, 0, SHARED),
    ([4000, 900], [1] * 2, 2, 8, 64, 32, True, 0, SHARED),
    ([8000], [1], 2, 16, 128, 256, True, 0, SHARED),
    ([20000], [8], 1, 2, 64, 64, True, 0, SHARED),
    ([8192] * 4, [1] * 4, 2, 4, 128, 64, True, 4096, SHARED),
    ([30000, 700], [1] * 2, 1, 40, 64, 16, False, 5000, SHARED),
    ([2000] * 3, [1] * 3, 4, 16, 128, 128, True, 0, EIGHT),
    ([1000, 300, 64], [1] * 3, 4, 4, 64, 16, True, 0, EIGHT),
    ([3000, 50, 2000], [1, 40, 1], 8, 4, 64, 64, True, 0, EIGHT),
    ([3000] * 20, [1] * 20, 32, 2, 64, 64, True, 0, form(0, 4)),
    ([2000, 700], [300, 500], 4, 2, 128, 16, False, 1000, form(0, 4)),
    ([300, 129, 64, 1, 200] * 8, [1] * 40, 32, 1, 64, 64, True, 0, form(0, 1)),
    ([300, 129, 64, 1, 200] * 8, [1] * 40, 32, 1, 128, 16, True, 100, form(0, 1)),
    # many rows: four waves, keys in chunks, two groups of four, eight waves; with windows, causal and not
    ([4000], [4000], 8, 2, 64, 16, True, 1000, form(1, 4)),
    ([4000], [3999], 8, 2, 128, 64, False, 1000, form(1, 4)),
    ([8192], [1024], 4, 4, 128, 64, True, 4096, CHUNKS),
    ([8192], [700], 4, 4, 128, 32, True, 0, CHUNKS),
    ([8192], [700], 4, 4, 64, 64, False, 0, CHUNKS),
    ([3900], [3900], 8, 1, 64, 16, True, 3000, form(1, 4, 2)),
    ([4096, 3000], [4096, 2000], 1, 4, 64, 64, False, 1000, form(1, 4, 2)),
    ([4096], [4096], 8, 1, 64, 64, True, 0, form(1, 4, 2)),
    ([4096], [2048], 8, 4, 128, 64, True, 0, {"bf16": form(1, 4, 2), "f16": form(1, 4)}),
    ([4096], [4096], 8, 2, 128, 64, True, 1500, {"bf16": form(1, 4), "f16": form(1, 4)}),
    ([2500], [2500], 32, 2, 128, 64, True, 1000, form(1, 8)),
    ([2500], [2500], 32, 2, 64, 16, False, 1000, form(1, 8)),
    ([1300, 900], [1300, 700], 32, 2, 128, 16, True, 0, form(1, 8)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(FORMS)))
def test_every_form_takes_every_key_once(case, dtype):
    *shape, want_form = FORMS[case]
    want_form = want_form.get(dtype, want_form)
    check_coverage(*shape, dtype, want_form)
    check_values(*shape, dtype, want_form)


@pytest.mark.parametrize("dtype,n,kv,many,big", [("bf16", 400, 1, 0, 14), ("f16", 400, 1, 0, 14), ("f16", 1300, 32, 1, 14), ("bf16", 1300, 32, 1, 24)])
def test_rows_beside_a_large_one_that_they_do_not_see(dtype, n, kv, many, big):
    """A key and value row 2^big times the others.  It sets the range of the row tiles that come to it, and rows of these that do not see it keep
    their results, but for what the header says is lost: of p * step what is below 2^-25 / 2^6 of the largest step, with elements up to 8 steps;
    bf16 results of many rows: of elements 2^-40 of twice the largest (8 steps and the centre)."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    d, at = 64, n // 2 + 5
    keys, values = [torch.randn(n, kv, d, generator=gen, device="cuda") for _ in range(2)]
    for x in (keys, values):
        x[at] *= 2.0 ** big
    f = Filled([n], kv, d, 64, True, lambda t: keys[t], lambda t: values[t])
    q = torch.randn(n, 2 * kv, d, generator=gen, device="cuda").to(DT[dtype])
    o, lse = f.run(q, [n], True, 0, dict(many=many))
    o, lse, q = o[:at], lse[:at], q[:at]
    k, v = f.stored(0)
    step, largest = f.steps(0)[:at].max(), max(float(k.abs().max()), float(v.abs().max()))
    hd = torch.tensor(ref.sylvester(d)).cuda()
    for h in range(2 * kv):
        x = q[:, h].double() @ hd
        s = (x @ k[:at, h // 2].t() / math.sqrt(d)).masked_fill(torch.ones(at, at, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        p, total = torch.softmax(s, -1), torch.logsumexp(s, -1)
        lost_k = 2.0 ** -40 * 2 * 2 * largest if many and dtype == "bf16" else 0.0
        e = ((2.0 ** -10 * (x.abs() @ k[:at, h // 2].abs().amax(0)) + 2.0 ** -10 * step * x.abs().sum(-1) + lost_k * x.abs().sum(-1)) / math.sqrt(d))[:, None]
        ones = torch.exp(total - s.amax(-1))[:, None]                     # the sum of weights, the largest 1
        seen = torch.arange(1, at + 1, device="cuda")[:, None]
        lost_v = lost_k if many and dtype == "bf16" else seen / ones * 8 * 2.0 ** -31 * (2 * largest / 15)
        want, size = p @ v[:at, h // 2], p @ v[:at, h // 2].abs()
        tol = (torch.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -16) * size + U_OUT[dtype] * want.abs() + lost_v
        assert ((o[:, h].double() - want).abs() <= tol).all(), h
        assert ((lse[:, h].double() - total).abs() <= e[:, 0] + 2.0 ** -11 + 2.0 ** -16 + 2.0 ** -20 * total.abs()).all(), h


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,kv,many", [(400, 1, 0), (1300, 32, 1)])
def test_tiny_queries_and_keys(n, kv, many, dtype):
    """Queries of 2^-105 against keys of 2^-60 (fp16: of 2^-24 against the same): all scores are 0 next to 1, and hidden keys stay hidden."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    d = 64
    keys, values = [torch.randn(n, kv, d, generator=gen, device="cuda") for _ in range(2)]
    f = Filled([n], kv, d, 64, False, lambda t: keys[t] * 2.0 ** -60, lambda t: values[t])
    q = (torch.randn(n, 2 * kv, d, generator=gen, device="cuda") * 2.0 ** (-105 if dtype == "bf16" else -24)).to(DT[dtype])
    o, lse = f.run(q, [n], True, 0, dict(many=many))
    v = f.stored(0)[1]
    count = torch.arange(1, n + 1, device="cuda", dtype=torch.float64)[:, None, None]
    want, size = (x.cumsum(0).div(count).repeat_interleave(2, 1) for x in (v, v.abs()))
    assert ((o.double() - want).abs() <= (2.0 ** -10 + 2.0 ** -16) * size + U_OUT[dtype] * want.abs()).all()
    assert ((lse.double() - count[..., 0].log()).abs() <= 1e-5).all()

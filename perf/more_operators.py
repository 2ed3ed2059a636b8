"""What a server does with a 4-bit paged key/value cache when contexts are long, as cases that can be timed and compared.

  * prefix_attention: a batch whose sequences begin with the same tokens (branches of one prompt, requests behind one system
    prompt or one document) attends over the shared pages once for all of them, and over each sequence's own pages;
  * attention_weights: how much attention every cached position has received, summed over queries and over the heads that share
    a key head, kept up from step to step;
  * select: the positions of each key head that are worth keeping, by these sums, beside the first and the most recent ones;
  * evict: the kept rows move together, in place or into other pages, in one layer or in all, and their sums with them.

The layout of the cache (see KV4Cache) is restated by `_fields` and `_values`.  The plain forms work on the same bytes.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
GOLDEN = 0.6180339887498949
CHUNK = 1 << 27                      # codes generated at a time


def listed():
    return [
        # a decode step of four branches of one short conversation: latency
        {"name": "prefix_branches", "op": "prefix_attention", "groups": 1, "batch": 4, "q_len": 1, "prefix": 1000, "kv_len": 25, "heads": 32,
         "kv_heads": 8, "head_dim": 128, "page": 16, "dtype": "bf16", "rotate": True, "causal": True, "window": 0},
        # a decode step of 64 answers sampled from one long prompt, grouped heads
        {"name": "prefix_sampling", "op": "prefix_attention", "groups": 1, "batch": 64, "q_len": 1, "prefix": 8192, "kv_len": 300, "heads": 32,
         "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0},
        # requests behind three system prompts of different length, every head with keys of its own, short heads
        {"name": "prefix_requests", "op": "prefix_attention", "groups": 3, "batch": 45, "q_len": 1, "prefix": 4001, "kv_len": 701, "heads": 16,
         "kv_heads": 16, "head_dim": 64, "page": 32, "dtype": "f16", "rotate": True, "causal": True, "window": 0},
        # candidate answers of up to 40 tokens scored against one long document
        {"name": "prefix_scoring", "op": "prefix_attention", "groups": 1, "batch": 12, "q_len": 40, "prefix": 65411, "kv_len": 40, "heads": 64,
         "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "f16", "rotate": True, "causal": True, "window": 0},
        # one token of a single short conversation: latency
        {"name": "weights_one", "op": "attention_weights", "batch": 1, "q_len": 1, "kv_len": 1025, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0, "decay": 1.0},
        # a decode step on the benchmark's full KV configuration: 16 sequences x 32 heads x 8192 positions
        {"name": "weights_step", "op": "attention_weights", "batch": 16, "q_len": 1, "kv_len": 8192, "even": True, "heads": 32,
         "kv_heads": 32, "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0, "decay": 0.99},
        # the last 64 queries of a prompt say which of its positions matter
        {"name": "weights_last_queries", "op": "attention_weights", "batch": 1, "q_len": 64, "kv_len": 16384, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0, "decay": 0.0},
        # all queries of two prompts, seven a key head, short heads, a sliding window
        {"name": "weights_prompts", "op": "attention_weights", "batch": 2, "q_len": 4000, "kv_len": 5003, "heads": 14, "kv_heads": 2,
         "head_dim": 64, "page": 16, "dtype": "f16", "rotate": False, "causal": True, "window": 1024, "decay": 0.0},
        # one layer of a small batch
        {"name": "select_layer", "op": "select", "layers": 1, "batch": 4, "kv_heads": 8, "kv_len": 4099, "keep": 1024, "sinks": 4, "recent": 64},
        # all layers of the benchmark's KV configuration
        {"name": "select_model", "op": "select", "layers": 32, "batch": 16, "kv_heads": 8, "kv_len": 8192, "keep": 2048, "sinks": 4,
         "recent": 256},
        # one layer of four sequences into pages of their own (the old ones are shared with other branches)
        {"name": "evict_layer", "op": "evict", "layers": 1, "batch": 4, "kv_heads": 8, "head_dim": 128, "page": 64, "kv_len": 8192,
         "keep": 1000, "in_place": False},
        # all layers of four sequences where they are
        {"name": "evict_model", "op": "evict", "layers": 32, "batch": 4, "kv_heads": 8, "head_dim": 128, "page": 64, "kv_len": 4096,
         "keep": 1024, "in_place": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("prefix_attention", "prefix_attention", "attention_weights", "attention_weights", "select", "evict"))
    d = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 128))
    kv, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 5, 7, 8))
    if kv == 32:
        group = 1
    heads = {"heads": kv * group, "kv_heads": kv, "head_dim": d, "page": page, "dtype": rng.choice(("bf16", "f16")),
             "rotate": rng.random() < 0.6, "causal": True, "window": 0}
    if op == "prefix_attention":
        batch = _log(rng, 2, 96)
        q_len = 1 if rng.random() < 0.6 else _log(rng, 2, 64)
        prefix = _log(rng, 64, max(64, min(65536, int(1.2e11 / (kv * group * batch * q_len * d)))))
        kv_len = max(q_len, _log(rng, 1, 1500))
        if rng.random() < 0.2:
            heads["causal"] = False
        if rng.random() < 0.2:
            heads["window"] = _log(rng, 16, 2 * (prefix + kv_len))
        return {"op": op, "groups": min(batch, rng.choice((1, 1, 2, 5))), "batch": batch, "q_len": q_len, "prefix": prefix, "kv_len": kv_len, **heads}
    if op == "attention_weights":
        heads["window"] = rng.choice((0, 0, 0, 128, 1000, 4096))
        decay = rng.choice((0.0, 0.5, 0.99, 1.0))
        if rng.random() < 0.5:                                        # a decode step
            batch = _log(rng, 1, 64)
            most = min(131072, 16 * 32 * 8192 // (kv * batch))
            return {"op": op, "batch": batch, "q_len": 1, "kv_len": _log(rng, 1, most), **heads, "decay": decay}
        batch = _log(rng, 1, 6)
        kv_len = _log(rng, 2, 16384)
        most = int(8000 * 5003 * 14 // (batch * kv * group * kv_len))
        return {"op": op, "batch": batch, "q_len": _log(rng, 2, max(2, min(kv_len, most))), "kv_len": kv_len, **heads, "decay": decay}
    layers = rng.choice((1, 1, 2, 16, 32))
    batch = _log(rng, 1, 16)
    if op == "select":
        most = min(131072, 32 * 16 * 8 * 8192 // (layers * batch * kv))
        n = _log(rng, 16, most)
        keep = _log(rng, 1, n)
        return {"op": op, "layers": layers, "batch": batch, "kv_heads": kv, "kv_len": n, "keep": keep, "sinks": min(keep // 4, rng.choice((0, 1, 4))),
                "recent": min(keep // 2, rng.choice((0, 16, 64, 250)))}
    most = min(65536, 32 * 4 * 8 * 4096 // (layers * batch * kv))
    n = _log(rng, 16, most)
    return {"op": op, "layers": layers, "batch": batch, "kv_heads": kv, "head_dim": d, "page": page, "kv_len": n, "keep": _log(rng, 1, max(1, n // 2)),
            "in_place": rng.random() < 0.5}


def _lens(case):
    """(query lengths, key lengths) of the sequences of a batch: the longest first, the others spread over the range."""
    q, kv, b = case.get("q_len", 1), case["kv_len"], case["batch"]
    if case.get("even"):
        return [q] * b, [kv] * b
    ql = [q if i == 0 else max(1, int(q * (i * GOLDEN * 3) % q) if q > 1 else 1) for i in range(b)]
    return ql, [kv if i == 0 else max(ql[i], int(kv * ((i * GOLDEN) % 1.0)), 1) for i in range(b)]


def _shared(case):
    """(first sequence of each group and behind the last, prefix lengths)"""
    g, b = case["groups"], case["batch"]
    return [i * b // g for i in range(g + 1)], [case["prefix"] if i == 0 else int(case["prefix"] * ((i * GOLDEN) % 1.0)) for i in range(g)]


def _pages(tokens, page):
    return -(-tokens // page)


def _seen(case, at, total):
    """The first position that the query at position `at` of a sequence of `total` sees, and the one behind the last."""
    hi = min(total, at + 1) if case["causal"] else total
    return max(0, at - case["window"] + 1) if case["window"] else 0, max(0, hi)


def work(case):
    kv = case["kv_heads"]
    if case["op"] == "select":
        _, kl = _lens(case)
        rows = case["layers"] * kv
        return {"bytes": rows * (4 * sum(kl) + 4 * case["keep"] * case["batch"]), "flops": 0}
    d = case["head_dim"]
    row = d + 8                                                       # bytes of a token's key and value of one head
    if case["op"] == "evict":
        _, kl = _lens(case)
        n = case["layers"] * kv * sum(min(case["keep"], x) for x in kl)
        return {"bytes": n * (2 * row + 8 + 4), "flops": 0}
    ql, kl = _lens(case)
    group = case["heads"] // kv
    if case["op"] == "attention_weights":
        keys = pairs = 0
        for q, k in zip(ql, kl):
            first = k
            for i in range(q):
                lo, hi = _seen(case, k - q + i, k)
                first, pairs = min(first, lo), pairs + hi - lo
            keys += k - first
        old = 8 if case["decay"] else 4
        return {"bytes": kv * (keys * (d // 2 + 4) + old * sum(kl)) + sum(ql) * case["heads"] * (2 * d + 4), "flops": 2 * d * kv * group * pairs}
    start, prefix = _shared(case)
    pairs = keys = 0
    for g, p in enumerate(prefix):
        least = p
        for b in range(start[g], start[g + 1]):
            total, first = p + kl[b], p + kl[b]
            for i in range(ql[b]):
                lo, hi = _seen(case, total - ql[b] + i, total)
                first, pairs = min(first, lo), pairs + hi - lo
            least = min(least, first)
            keys += total - max(p, first)
        keys += p - least
    n = sum(ql) * case["heads"] * d
    return {"bytes": keys * kv * row + 4 * n, "flops": 4 * d * kv * group * pairs}


# ---- inputs

def _filled(gen, layers, pages, case):
    """A pool of pages as appended tokens leave them: bell-shaped codes, steps and centres of unit-scale rows."""
    kv, d, p = case["kv_heads"], case["head_dim"], case["page"]
    data = torch.empty((layers * pages, kv, p * (d + 8)), dtype=torch.uint8, device="cuda")
    step = max(1, CHUNK // (kv * p * d * 2))
    for at in range(0, layers * pages, step):
        part = data[at:at + step]
        c = torch.randn((len(part), kv, p * d, 2), generator=gen, device="cuda", dtype=torch.float16)
        c = c.mul_(2.7).add_(7.5).round_().clamp_(0, 15).to(torch.uint8)
        part[..., :p * d] = c[..., 0] | (c[..., 1] << 4)
        s = 0.37 * (0.5 + torch.rand((len(part), kv, 2 * p), generator=gen, device="cuda"))
        m = 0.5 * s * torch.randn((len(part), kv, 2 * p), generator=gen, device="cuda")
        part[..., p * d:] = torch.stack((s, m), -1).to(torch.bfloat16).view(torch.uint8).flatten(-2)
    return data.view(layers, pages, -1)


def _tables(gen, lists, extra=3):
    """Tables of page numbers for lists of page counts, all from one pool whose order is shuffled, and the pool's size."""
    pages = sum(map(sum, lists)) + extra
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    out, at = [], 0
    for need in lists:
        table = torch.zeros((len(need), max(need)), dtype=torch.int32, device="cuda")
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        out.append(table)
    return out, pages


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _sums(gen, shape):
    """Attention as it adds up: a few positions have most of it, many have none that 32 bits hold."""
    x = torch.randn(shape, generator=gen, device="cuda").mul_(2.5)
    return x.exp().mul_(0.01).masked_fill_(x < -2.5, 0.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kv = case["kv_heads"]
    s = dict(case)
    ql, kl = _lens(case)
    s["kv_lens"] = _ints(kl)
    if case["op"] in ("prefix_attention", "attention_weights"):
        d, p = case["head_dim"], case["page"]
        need = [_pages(n, p) for n in kl]
        if case["op"] == "prefix_attention":
            start, prefix = _shared(case)
            (s["prefix_table"], s["table"]), pages = _tables(gen, ([max(1, _pages(n, p)) for n in prefix], need))
            s["group_start"], s["prefix_lens"] = _ints(start), _ints(prefix)
            at = [sum(ql[:i]) for i in range(len(ql) + 1)]
            s["group_most"] = max(at[b] - at[a] for a, b in zip(start, start[1:]))
        else:
            (s["table"],), pages = _tables(gen, (need,))
        s["data"] = _filled(gen, 1, pages, case)
        s["q_start"] = _ints([sum(ql[:i]) for i in range(len(ql) + 1)])
        s["q_most"] = max(ql)
        s["q"] = torch.randn((sum(ql), case["heads"], d), generator=gen, device="cuda").mul_(1.5).to(DTYPES[case["dtype"]])
        if case["op"] == "attention_weights":                         # what the attention before it has returned
            t, live = _scores(s)
            s["lse"] = t.logsumexp(-1).permute(0, 3, 1, 2).flatten(2)[live].contiguous()
            # a step or two of attention is in the sums already
            s["weights"] = _sums(gen, (case["batch"], kv, s["table"].shape[1] * p)) * (case["heads"] // kv * case["q_len"] / case["kv_len"])
    else:
        lead = (case["layers"], case["batch"], kv)
        most = max(kl)
        if case["op"] == "select":
            s["weights"] = _sums(gen, lead + (most,))
        else:
            p, keep = case["page"], case["keep"]
            need = [_pages(n, p) for n in kl]
            rows = [need] if case["in_place"] else [need, [_pages(keep, p)] * len(kl)]
            tables, pages = _tables(gen, rows)
            s["table"], s["new_table"] = tables[0], None if case["in_place"] else tables[1]
            s["data"] = _filled(gen, case["layers"], pages, case)
            s["weights"] = _sums(gen, lead + (s["table"].shape[1] * p,))
            score = torch.rand(lead + (most,), generator=gen, device="cuda")
            score.masked_fill_(torch.arange(most, device="cuda") >= s["kv_lens"][:, None, None], -1.0)
            top = score.topk(keep, -1)
            index = torch.where(top.values < 0, most, top.indices).sort(-1).values.to(torch.int32)
            s["index"] = torch.where(index == most, -1, index)
    if own:                                                           # what a server keeps: the cache and the rotation
        import paper_2504_13989_amd as rq
        s["rq"] = rq
        if "data" in s:
            s["h"] = rq.hadamard_build(case["head_dim"]) if case.get("rotate") else None
            s["cache"] = rq.KV4Cache(s["data"], kv, case["head_dim"], case["page"])
            s["layer"] = s["cache"].layer(0)
    return s


# ---- the passes

def run(s):
    if own:
        return _own(s)
    return {"prefix_attention": _prefix_attention, "attention_weights": _attention_weights, "select": _select, "evict": _evict}[s["op"]](s)


def _own(s):
    rq = s["rq"]
    if s["op"] == "select":
        return rq.kv4_select(s["weights"], s["kv_lens"], s["keep"], sinks=s["sinks"], recent=s["recent"])
    if s["op"] == "evict":
        rq.kv4_evict(s["cache"], s["index"], s["table"], new_table=s["new_table"], weights=s["weights"])
        return s["data"], s["weights"]
    start = None if s["q_most"] == 1 else s["q_start"]
    if s["op"] == "attention_weights":
        rq.kv4_attention_weights(s["h"], s["layer"], s["q"], s["lse"], s["table"], s["kv_lens"], s["weights"], start, causal=s["causal"],
                                 window=s["window"], decay=s["decay"])
        return s["weights"]
    return rq.kv4_prefix_attention(s["h"], s["layer"], s["q"], s["prefix_table"], s["prefix_lens"], s["group_start"], s["table"], s["kv_lens"],
                                   start, causal=s["causal"], window=s["window"])


def _signs(d):
    """The Sylvester matrix of order d, in 32 bits: (-1) to the number of bits that i and j share."""
    i = torch.arange(d, device="cuda")
    x = i[:, None] & i
    x = x ^ (x >> 4)
    x = x ^ (x >> 2)
    x = x ^ (x >> 1)
    return 1.0 - 2.0 * (x & 1)


def _queries(s):
    """The queries in 32 bits, rotated as the keys were."""
    q, d = s["q"].float(), s["head_dim"]
    return torch.matmul(q, _signs(d)) * torch.tensor(d ** -0.5, device=q.device) if s["rotate"] else q


def _fields(data, s):
    """(key codes, value codes, key parameters, value parameters) of pages [..., page bytes], as views."""
    kv, d, p = s["kv_heads"], s["head_dim"], s["page"]
    x = data.unflatten(-1, (kv, p * (d + 8)))
    half = p * d // 2
    k = x[..., :half].unflatten(-1, (p, d // 2))                                 # [token][two values a byte]
    v = x[..., half:2 * half].unflatten(-1, (p // 4, 16, d // 64, 4, 2))         # [token / 4][16 runs][fours][token % 4][two]
    return k, v, x[..., 2 * half:2 * half + 4 * p].unflatten(-1, (p, 4)), x[..., 2 * half + 4 * p:].unflatten(-1, (p, 4))


def _values(codes, params):
    """(code - 7.5) * step + centre, in 32 bits: codes [..., bytes], params [..., 4 bytes]"""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 7.5
    sm = params.contiguous().view(torch.bfloat16).float()
    return c * sm[..., :1] + sm[..., 1:]


def _keys(s, table):
    """Keys of the sequences of a table: [sequences, kv heads, positions, d]"""
    fk, _, fpk, _ = _fields(s["data"][0][table.long()], s)
    return _values(fk, fpk).transpose(1, 2).reshape(len(table), s["kv_heads"], -1, s["head_dim"])


def _vals(s, table):
    _, fv, _, fpv = _fields(s["data"][0][table.long()], s)
    return _values(fv.movedim(-2, -4).flatten(-3).flatten(-3, -2), fpv).transpose(1, 2).reshape(len(table), s["kv_heads"], -1, s["head_dim"])


def _padded(q, start, most, s):
    """(queries of stretches of tokens [stretches, kv heads, group * most, d], which rows are there [stretches, most], the tokens they are)"""
    n = len(start) - 1
    i = torch.arange(most, device=q.device)
    live = i < (start[1:] - start[:-1])[:, None]
    row = (start[:-1, None].long() + i).clamp(max=len(q) - 1)
    kv, d = s["kv_heads"], s["head_dim"]
    return q[row].view(n, most, kv, -1, d).permute(0, 2, 3, 1, 4).reshape(n, kv, -1, d), live, row


def _mask(s, j, pos, total):
    """Which positions j a query at `pos` of a sequence of `total` sees: [..., positions]"""
    seen = (j < total[..., None]).expand(pos.shape + j.shape)
    if s["causal"]:
        seen = seen & (j <= pos[..., None])
    if s["window"]:
        seen = seen & (j > pos[..., None] - s["window"])
    return seen


def _part(t, seen, v, n, most, s):
    """(maximum, sum, sum of values) of the rows of scores t [n, kv, group * most, keys], token by token: [n, most, heads, ...]"""
    t = t.view(n, s["kv_heads"], -1, most, t.shape[-1])
    t.masked_fill_(~seen[:, None, None], -math.inf)
    m = t.amax(-1, keepdim=True).clamp(min=-1e30)
    t.sub_(m).exp_()
    total = t.sum(-1, keepdim=True)
    o = torch.matmul(t.flatten(2, 3), v).view(n, s["kv_heads"], -1, most, s["head_dim"])
    return [x.permute(0, 3, 1, 2, 4).flatten(2, 3) for x in (m, total, o)]


def _prefix_attention(s):
    q, scale = _queries(s), s["head_dim"] ** -0.5
    qs, gs, prefix, lens = s["q_start"].long(), s["group_start"].long(), s["prefix_lens"].long(), s["kv_lens"].long()
    token = torch.arange(len(q), device=q.device)
    seq = torch.searchsorted(qs, token, right=True) - 1               # of a token
    of = torch.searchsorted(gs, seq, right=True) - 1                  # group of a token
    total = prefix[of] + lens[seq]
    pos = total - qs[seq + 1] + token
    # the shared positions: all queries of a group at once
    start = qs[gs]
    x, live, row = _padded(q, start, s["group_most"], s)
    k = _keys(s, s["prefix_table"])
    j = torch.arange(k.shape[2], device=q.device)
    seen = _mask(s, j, pos[row], torch.minimum(prefix[:, None], total[row]))
    shared = [y[live] for y in _part(torch.matmul(x, k.transpose(-1, -2)) * scale, seen, _vals(s, s["prefix_table"]), len(start) - 1, s["group_most"], s)]
    # each sequence's own
    x, live, row = _padded(q, qs, s["q_most"], s)
    k = _keys(s, s["table"])
    j = torch.arange(k.shape[2], device=q.device)
    before = prefix[of[row]]
    seen = _mask(s, j, pos[row] - before, total[row] - before)
    alone = [y[live] for y in _part(torch.matmul(x, k.transpose(-1, -2)) * scale, seen, _vals(s, s["table"]), len(qs) - 1, s["q_most"], s)]
    m = torch.maximum(shared[0], alone[0])
    a, b = (shared[0] - m).exp(), (alone[0] - m).exp()
    return ((a * shared[2] + b * alone[2]) / (a * shared[1] + b * alone[1]).clamp(min=1e-30)).to(s["q"].dtype)


def _scores(s):
    """Scores [batch, kv heads, group, queries, positions] with -infinity where a query does not see, and which queries are there."""
    q = _queries(s)
    x, live, _ = _padded(q, s["q_start"].long(), s["q_most"], s)
    k = _keys(s, s["table"])
    b, n, most = len(live), k.shape[2], s["q_most"]
    t = torch.matmul(x, k.transpose(-1, -2)).mul_(s["head_dim"] ** -0.5).view(b, s["kv_heads"], -1, most, n)
    qs, lens = s["q_start"].long(), s["kv_lens"].long()
    pos = (lens - qs[1:] + qs[:-1])[:, None] + torch.arange(most, device=q.device)
    seen = _mask(s, torch.arange(n, device=q.device), pos, lens[:, None].expand(pos.shape)) & live[..., None]
    t.masked_fill_(~seen[:, None, None], -math.inf)
    return t, live


def _attention_weights(s):
    t, live = _scores(s)
    b, kv, group, most, n = t.shape
    lse = torch.zeros((b, most, kv * group), device=t.device)
    lse[live] = s["lse"]
    w = t.sub_(lse.view(b, most, kv, group, 1).permute(0, 2, 3, 1, 4)).exp_().sum((2, 3))
    there = (torch.arange(n, device=w.device) < s["kv_lens"][:, None, None]).expand(b, kv, n)
    old = s["weights"][..., :n]
    s["weights"][..., :n] = torch.where(there, old * s["decay"] + w if s["decay"] else w, old)
    return s["weights"]


def _select(s):
    w, keep, sinks, recent = s["weights"], s["keep"], s["sinks"], s["recent"]
    n = w.shape[-1]
    j = torch.arange(n, device=w.device)
    lens = s["kv_lens"].long()[:, None, None]
    always = (j < sinks) | (j >= lens - recent)
    x = torch.where(always, math.inf, w).masked_fill(j >= lens, -math.inf)
    order = x.sort(dim=-1, descending=True, stable=True).indices[..., :keep]         # ties: the lowest first
    order = torch.where(order < lens, order, n).sort(-1).values
    out = torch.full(w.shape[:-1] + (keep,), -1, dtype=torch.int32, device=w.device)
    out[..., :order.shape[-1]] = torch.where(order < n, order, -1).to(torch.int32)
    return out


def _evict(s):
    d, p = s["head_dim"], s["page"]
    index = s["index"].long()                                                    # [layers, batch, kv heads, keep]
    to = s["table"] if s["new_table"] is None else s["new_table"]
    layers, batch, kv, keep = index.shape
    i = torch.arange(keep, device=index.device).expand(index.shape)
    kept = index >= 0
    layer, b, h, i = (x.expand(index.shape)[kept] for x in (
        torch.arange(layers, device=index.device).view(-1, 1, 1, 1), torch.arange(batch, device=index.device).view(-1, 1, 1),
        torch.arange(kv, device=index.device).view(-1, 1), i))
    at = index[kept]
    fk, fv, fpk, fpv = _fields(s["data"], s)                                     # [layers, pages, kv heads, ...]
    page, off = s["table"][b, at // p].long(), at % p
    rows = fk[layer, page, h, off], fv[layer, page, h, off // 4, :, :, off % 4], fpk[layer, page, h, off], fpv[layer, page, h, off]
    page, off = to[b, i // p].long(), i % p
    fk[layer, page, h, off], fpk[layer, page, h, off], fpv[layer, page, h, off] = rows[0], rows[2], rows[3]
    fv[layer, page, h, off // 4, :, :, off % 4] = rows[1]
    w = torch.zeros_like(s["weights"])
    w[..., :keep] = torch.where(kept, s["weights"].gather(-1, index.clamp(min=0)), 0.0)
    s["weights"].copy_(w)
    return s["data"], s["weights"]


# ---- the same from the definitions in 64 bits

def _sylvester(d):
    h = torch.ones((1, 1), dtype=torch.float64, device="cuda")
    while len(h) < d:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h / math.sqrt(d)


def _decoded(s, page):
    """Keys and values [tokens, kv heads, d] of the pages, in 64 bits."""
    kv, d, p = s["kv_heads"], s["head_dim"], s["page"]
    keys, values = [], []
    for part in page.long().split(max(1, 8192 // p)):
        n = len(part)
        rec = s["data"][0][part].view(n, kv, p * (d + 8)).to(torch.int32)
        at = torch.arange(p * d, device="cuda")
        nib = (rec[..., at // 2] >> (4 * (at % 2))) & 15                         # key codes
        tok, e = at // d, at % d
        per = d // 16
        run_, part_, f = e // per, e % per // 4, e % 4
        byte = p * d // 2 + ((((tok // 4) * 16 + run_) * (d // 64) + part_) * 4 + tok % 4) * 2 + f // 2
        vib = (rec[..., byte] >> (4 * (f % 2))) & 15
        word = rec[..., p * d:].view(n, kv, 2, p, 2, 2)
        bits = ((word[..., 0] | (word[..., 1] << 8)) << 16).view(torch.float32).double()
        for i, (c, out) in enumerate(((nib, keys), (vib, values))):
            x = (c.view(n, kv, p, d) - 7.5) * bits[:, :, i, :, :1] + bits[:, :, i, :, 1:]
            out.append(x.transpose(1, 2).reshape(n * p, kv, d))
    return torch.cat(keys), torch.cat(values)


def _hidden(case, j, pos):
    bad = torch.zeros((len(pos), len(j)), dtype=torch.bool, device="cuda")
    if case["causal"]:
        bad |= j > pos[:, None]
    if case["window"]:
        bad |= j <= pos[:, None] - case["window"]
    return bad


def exact(case, seed):
    global own
    if case["op"] == "select":
        return None
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    if case["op"] == "evict":                                         # (the rows are bytes)
        out = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda").flatten(0, -2)
        for row, old, index in zip(out, s["weights"].flatten(0, -2), s["index"].flatten(0, -2)):
            index = index[index >= 0].long()
            row[:len(index)] = old[index].double()
        return None, out.view(s["weights"].shape)
    d, group = case["head_dim"], case["heads"] // case["kv_heads"]
    turn = _sylvester(d) if case["rotate"] else torch.eye(d, dtype=torch.float64, device="cuda")
    ql, kl = _lens(case)
    at = [sum(ql[:i]) for i in range(len(ql) + 1)]
    if case["op"] == "attention_weights":
        if sum(a * b for a, b in zip(ql, kl)) * case["heads"] * d > 4e11:
            return None
        out = s["weights"].double()
        for b, (nq, n) in enumerate(zip(ql, kl)):
            k = _decoded(s, s["table"][b, :_pages(n, case["page"])])[0][:n]
            j = torch.arange(n, device="cuda")
            out[b, :, :n] *= case["decay"]
            for head in range(case["heads"]):
                for part in torch.arange(nq, device="cuda").split(max(1, (1 << 26) // n)):
                    t = (s["q"][at[b] + part, head].double() @ turn) @ k[:, head // group].t() / math.sqrt(d)
                    p = (t - s["lse"][at[b] + part, head].double()[:, None]).exp()
                    out[b, head // group, :n] += p.masked_fill(_hidden(case, j, n - nq + part), 0.0).sum(0)
        return out
    start, prefix = _shared(case)
    if sum(ql[b] * (p + kl[b]) for g, p in enumerate(prefix) for b in range(start[g], start[g + 1])) * case["heads"] * d > 4e11:
        return None
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for g, p in enumerate(prefix):
        first = _decoded(s, s["prefix_table"][g, :max(1, _pages(p, case["page"]))])
        for b in range(start[g], start[g + 1]):
            nq, n = ql[b], p + kl[b]
            k, v = (torch.cat((x[:p], y[:kl[b]])) for x, y in zip(first, _decoded(s, s["table"][b, :_pages(kl[b], case["page"])])))
            j = torch.arange(n, device="cuda")
            bad = _hidden(case, j, n - nq + torch.arange(nq, device="cuda"))
            for head in range(case["heads"]):
                t = (s["q"][at[b]:at[b + 1], head].double() @ turn) @ k[:, head // group].t() / math.sqrt(d)
                w = torch.softmax(t.masked_fill(bad, -math.inf), -1).nan_to_num(0.0)
                out[at[b]:at[b + 1], head] = w @ v[:, head // group]
    return out

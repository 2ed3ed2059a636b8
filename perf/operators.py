"""The 4-bit paged key/value cache as a server uses it, as cases that can be timed and compared.

A model served with rotated, quantized keys and values does four things with its cache:

  * append: the keys and values of new tokens are rotated (keys), quantized to 4 bits a value and written to
    the tokens' slots; one decode step of a batch, a prompt, a ragged mix of both;
  * attention: queries of one decode step, of whole prompts or of chunks of prompts against the cache;
  * read: rows of the cache back as numbers, in the original basis, for scoring or for moving them elsewhere;
  * copy_pages: pages of a forked sequence or of a compaction, in all layers at once.

The layout of the cache (see KV4Cache) is restated by `_fields` and `_values`.  The plain forms work on the same bytes.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
GOLDEN = 0.6180339887498949
CHUNK = 1 << 27                      # codes generated at a time


def listed():
    return [
        # one decode step of the benchmark's KV configuration (16 sequences, 32 heads of 128): launches and the host decide
        {"name": "append_step", "op": "append", "tokens": 16, "batch": 16, "kv_heads": 32, "head_dim": 128, "page": 64,
         "dtype": "bf16", "rotate": True, "fused": True, "clip": 1.0, "skip": 0},
        # a whole prompt of that configuration, one layer
        {"name": "append_prompt", "op": "append", "tokens": 8192, "batch": 1, "kv_heads": 32, "head_dim": 128, "page": 64,
         "dtype": "bf16", "rotate": True, "fused": True, "clip": 1.0, "skip": 0},
        # a ragged mix of fp32 tokens in a padded batch (every 7th one is padding), short heads, short pages
        {"name": "append_ragged_f32", "op": "append", "tokens": 1037, "batch": 5, "kv_heads": 8, "head_dim": 64, "page": 16,
         "dtype": "f32", "rotate": True, "fused": False, "clip": 0.9, "skip": 7},
        # rows picked out of the cache back to the original basis
        {"name": "read_rows", "op": "read", "rows": 999, "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "bf16",
         "rotate": True, "order": "picked"},
        # a long sequence read back whole, to be moved or re-quantized
        {"name": "read_sequence", "op": "read", "rows": 65536, "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "f16",
         "rotate": False, "order": "whole"},
        # one token of a single short conversation: latency
        {"name": "decode_one", "op": "attention", "batch": 1, "q_len": 1, "kv_len": 1025, "heads": 32, "kv_heads": 8,
         "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0},
        # a decode step on the benchmark's full KV configuration: 16 sequences x 32 heads x 8192 positions
        {"name": "decode_full", "op": "attention", "batch": 16, "q_len": 1, "kv_len": 8192, "even": True, "heads": 32,
         "kv_heads": 32, "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0},
        # a decode step of few sequences of very different length, grouped heads: work has to be split over the long ones
        {"name": "decode_ragged_long", "op": "attention", "batch": 6, "q_len": 1, "kv_len": 65411, "heads": 64, "kv_heads": 8,
         "head_dim": 128, "page": 32, "dtype": "f16", "rotate": True, "causal": True, "window": 0},
        # a prompt of 8192 tokens against its own cache
        {"name": "prompt", "op": "attention", "batch": 1, "q_len": 8192, "kv_len": 8192, "even": True, "heads": 32,
         "kv_heads": 8, "head_dim": 128, "page": 64, "dtype": "bf16", "rotate": True, "causal": True, "window": 0},
        # chunks of several prompts and single tokens in one batch, sliding window, seven queries a key head, short heads
        {"name": "chunks_windowed", "op": "attention", "batch": 5, "q_len": 701, "kv_len": 5003, "heads": 14, "kv_heads": 2,
         "head_dim": 64, "page": 16, "dtype": "f16", "rotate": False, "causal": True, "window": 1024},
        # a sequence forked four ways: the last, partly filled page of each branch becomes its own in all layers
        {"name": "fork", "op": "copy_pages", "pairs": 4, "layers": 32, "kv_heads": 8, "head_dim": 128, "page": 64},
        # compaction: the live pages at the end of the pool move into the holes of freed ones
        {"name": "compact", "op": "copy_pages", "pairs": 257, "layers": 8, "kv_heads": 8, "head_dim": 128, "page": 64},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("append", "attention", "attention", "attention", "read", "copy_pages"))
    d = rng.choice((64, 128, 128))
    page = rng.choice((16, 32, 64, 128))
    if op == "append":
        kv = rng.choice((1, 2, 4, 8, 32))
        tokens = _log(rng, 1, min(131072, 8192 * 32 // kv))
        return {"op": op, "tokens": tokens, "batch": min(tokens, _log(rng, 1, 64)), "kv_heads": kv, "head_dim": d, "page": page,
                "dtype": rng.choice(("bf16", "f16", "f32")), "rotate": rng.random() < 0.7, "fused": rng.random() < 0.5,
                "clip": rng.choice((1.0, 0.95, 0.9)), "skip": rng.choice((0, 0, 5, 11))}
    if op == "read":
        kv = rng.choice((1, 2, 4, 8, 32))
        return {"op": op, "rows": _log(rng, 1, 65536 * 8 // kv), "kv_heads": kv, "head_dim": d, "page": page,
                "dtype": rng.choice(("bf16", "f16", "f32")), "rotate": rng.random() < 0.5, "order": rng.choice(("picked", "whole"))}
    if op == "copy_pages":
        kv = rng.choice((1, 2, 4, 8, 32))
        layers = rng.choice((1, 2, 8, 16, 32))
        most = max(1, 257 * 8 * 8 * 64 * 136 // (layers * kv * page * (d + 8)))
        return {"op": op, "pairs": _log(rng, 1, min(4096, most)), "layers": layers, "kv_heads": kv, "head_dim": d, "page": page}
    kv, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 5, 7, 8))
    if kv == 32:
        group = 1
    dtype = rng.choice(("bf16", "f16"))
    window = rng.choice((0, 0, 0, 128, 1000, 4096))
    if rng.random() < 0.5:                                            # a decode step
        batch = _log(rng, 1, 64)
        most = min(131072, 16 * 32 * 8192 // (kv * batch))
        case = {"batch": batch, "q_len": 1, "kv_len": _log(rng, 1, most), "causal": True}
    else:                                                             # prompts or chunks of them
        batch = _log(rng, 1, 6)
        kv_len = _log(rng, 2, 16384)
        most = int(8192 * 8192 * 16 // (batch * kv * group * kv_len))
        q_len = _log(rng, 2, max(2, min(kv_len, most, 8192)))
        case = {"batch": batch, "q_len": q_len, "kv_len": kv_len, "causal": rng.random() < 0.8}
    return {"op": op, **case, "heads": kv * group, "kv_heads": kv, "head_dim": d, "page": page, "dtype": dtype,
            "rotate": rng.random() < 0.6, "window": window}


def _lens(case):
    """(query lengths, key lengths) of the sequences of a batch: the longest first, the others spread over the range."""
    q, kv, b = case["q_len"], case["kv_len"], case["batch"]
    if case.get("even"):
        return [q] * b, [kv] * b
    share = [1.0 if i == 0 else (i * GOLDEN) % 1.0 for i in range(b)]
    ql = [q if i == 0 else max(1, int(q * (i * GOLDEN * 3) % q) if q > 1 else 1) for i in range(b)]
    return ql, [max(ql[i], int(kv * share[i]), 1) for i in range(b)]


def _pages(tokens, page):
    return -(-tokens // page)


def _page_bytes(case):
    return case["kv_heads"] * case["page"] * (case["head_dim"] + 8)


def work(case):
    d, kv = case["head_dim"], case["kv_heads"]
    row = d + 8                                                       # bytes of a token's key and value of one head
    if case["op"] == "append":
        n = case["tokens"] * kv
        rotation = d * int(math.log2(d)) if case["rotate"] else 0
        return {"bytes": 2 * n * d * SIZE[case["dtype"]] + n * row + 2 * n * d * 2, "flops": n * (rotation + 12 * d)}
    if case["op"] == "read":
        n = case["rows"] * kv
        rotation = d * int(math.log2(d)) if case["rotate"] else 0
        return {"bytes": n * row + 2 * n * d * SIZE[case["dtype"]] + 8 * case["rows"], "flops": n * (rotation + 4 * d)}
    if case["op"] == "copy_pages":
        return {"bytes": 2 * case["pairs"] * case["layers"] * _page_bytes(case), "flops": 0}
    ql, kl = _lens(case)
    pairs = keys = 0
    for q, k in zip(ql, kl):
        last = [k - q + i if case["causal"] else k - 1 for i in (0, q - 1)]
        first = [max(0, k - q + i - case["window"] + 1) if case["window"] else 0 for i in (0, q - 1)]
        keys += last[1] - first[0] + 1
        if not case["window"]:
            pairs += (last[0] + last[1] + 2) * q // 2
        else:
            pairs += sum((k - q + i if case["causal"] else k - 1) - max(0, k - q + i - case["window"] + 1) + 1 for i in range(q))
    n = sum(ql) * case["heads"] * d
    return {"bytes": keys * kv * row + 2 * n * SIZE[case["dtype"]], "flops": 4 * d * case["heads"] * pairs}


# ---- inputs

def _rows(gen, shape, scale_rows):
    """Token rows as heads see them: normal, two strong channels a head, some rows larger than others."""
    x = torch.randn(shape, generator=gen, device="cuda")
    strong = torch.randint(0, shape[-1], (shape[1], 2), generator=gen, device="cuda")
    gain = torch.ones(shape[1:], device="cuda").scatter_(1, strong, 8.0) if scale_rows else 1.0
    return x * gain * (0.5 + torch.rand(shape[:2] + (1,), generator=gen, device="cuda"))


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


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    d, kv, p = case["head_dim"], case["kv_heads"], case["page"]
    s = dict(case)
    if case["op"] == "append":
        t, b = case["tokens"], case["batch"]
        dt = DTYPES[case["dtype"]]
        if case["fused"]:                                             # slices of a fused projection's output
            qkv = torch.empty((t, 3 * kv, d), dtype=dt, device="cuda")
            qkv[:, kv:2 * kv] = _rows(gen, (t, kv, d), True)
            qkv[:, 2 * kv:] = _rows(gen, (t, kv, d), False)
            s["k"], s["v"] = qkv[:, kv:2 * kv], qkv[:, 2 * kv:]
        else:
            s["k"], s["v"] = _rows(gen, (t, kv, d), True).to(dt), _rows(gen, (t, kv, d), False).to(dt)
        # each sequence goes on from a length of its own
        per = [t // b + (i < t % b) for i in range(b)]
        begun = [int(97 * ((i * GOLDEN) % 1.0)) if b > 1 else 0 for i in range(b)]
        need = [_pages(n + o, p) for n, o in zip(per, begun)]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=gen, device="cuda")
        first = [sum(need[:i]) for i in range(b)]
        pos = torch.cat([torch.arange(n, device="cuda") + o + f * p for n, o, f in zip(per, begun, first)])
        slots = order[pos // p] * p + pos % p
        if case["skip"]:
            slots[::case["skip"]] = -1
        s["slots"] = slots
        s["data"] = torch.zeros((1, pages, _page_bytes(case)), dtype=torch.uint8, device="cuda")
    elif case["op"] == "read":
        n = case["rows"]
        pages = _pages(n, p) + 2
        s["data"] = _filled(gen, 1, pages, case)
        order = torch.randperm(pages, generator=gen, device="cuda")
        pos = torch.randperm(pages * p, generator=gen, device="cuda")[:n] if case["order"] == "picked" else torch.arange(n, device="cuda")
        s["slots"] = order[pos // p] * p + pos % p
    elif case["op"] == "copy_pages":
        n = case["pairs"]
        pages = 2 * n + 5
        size = (case["layers"], pages, _page_bytes(case))
        s["data"] = torch.randint(0, 256, size, generator=gen, device="cuda", dtype=torch.uint8)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        s["src"], s["dst"] = order[:n].contiguous(), order[n:2 * n].contiguous()
    else:
        ql, kl = _lens(case)
        need = [_pages(n, p) for n in kl]
        pages, width = sum(need) + 3, max(need)
        s["data"] = _filled(gen, 1, pages, case)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.zeros((len(kl), width), dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        s["table"] = table
        s["kv_lens"] = torch.tensor(kl, dtype=torch.int32, device="cuda")
        s["q_start"] = torch.tensor([sum(ql[:i]) for i in range(len(ql) + 1)], dtype=torch.int32, device="cuda")
        s["q_most"] = max(ql)
        s["q"] = torch.randn((sum(ql), case["heads"], d), generator=gen, device="cuda").mul_(1.5).to(DTYPES[case["dtype"]])
    if own:                                                           # what a server keeps: the cache and the rotation
        import paper_2504_13989_amd as rq
        s["rq"] = rq
        s["h"] = rq.hadamard_build(d) if case.get("rotate") else None
        s["cache"] = rq.KV4Cache(s["data"], kv, d, p)
        s["layer"] = s["cache"].layer(0)
    return s


# ---- the passes

def run(s):
    if own:
        return _own(s)
    return {"append": _append, "read": _read, "copy_pages": _copy_pages, "attention": _attention}[s["op"]](s)


def _own(s):
    rq = s["rq"]
    if s["op"] == "append":
        rq.kv4_append(s["h"], s["layer"], s["k"], s["v"], s["slots"], clip=s["clip"])
        return rq.kv4_read(None, s["layer"], s["slots"], out_dtype=torch.bfloat16)  # the rows as they are stored
    if s["op"] == "read":
        return rq.kv4_read(s["h"], s["layer"], s["slots"], out_dtype=DTYPES[s["dtype"]])
    if s["op"] == "copy_pages":
        rq.kv4_copy_pages(s["cache"], s["src"], s["dst"])
        return s["data"]
    return rq.kv4_attention(s["h"], s["layer"], s["q"], s["table"], s["kv_lens"], None if s["q_most"] == 1 else s["q_start"],
                            causal=s["causal"], window=s["window"])


def _rotated(x):
    """x H / sqrt(d) over the last axis, H the Sylvester matrix: butterflies over strides 1, 2, 4 ..."""
    d, w = x.shape[-1], 1
    while w < d:
        y = x.unflatten(-1, (d // (2 * w), 2, w))
        x = torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).flatten(-3)
        w *= 2
    return x * torch.tensor(d ** -0.5, dtype=torch.float32, device=x.device)


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


def _quantized(y, clip):
    """(codes [T, H, d] u8, parameters [T, H, 4] u8) of rows in 32 bits"""
    lo, hi = clip * y.amin(-1, keepdim=True), clip * y.amax(-1, keepdim=True)
    step = ((hi - lo) / torch.tensor(15.0, device=y.device)).to(torch.bfloat16)
    mid = (0.5 * (hi + lo)).to(torch.bfloat16)
    flat = step.float() < 2.0 ** -100
    step = torch.where(flat, torch.zeros_like(step), step)
    inv = torch.where(flat, torch.zeros_like(lo), 1.0 / step.float())
    c = (((y - mid.float()) * inv) + 7.5).round().clamp(0, 15).to(torch.uint8)
    return c, torch.cat((step, mid), -1).view(torch.uint8)


def _append(s):
    d, p = s["head_dim"], s["page"]
    k, v = s["k"].float(), s["v"].float()
    clip = torch.tensor(s["clip"], dtype=torch.float32, device=k.device)
    ck, pk = _quantized(_rotated(k) if s["rotate"] else k, clip)
    cv, pv = _quantized(v, clip)
    kept = s["slots"] >= 0
    slot = s["slots"][kept]
    page, off = slot // p, slot % p
    fk, fv, fpk, fpv = _fields(s["data"][0], s)
    bk, bv = ck[..., 0::2] | (ck[..., 1::2] << 4), cv[..., 0::2] | (cv[..., 1::2] << 4)
    fk[page, :, off] = bk[kept]
    fv[page, :, off // 4, :, :, off % 4] = bv[kept].unflatten(-1, (16, d // 64, 2))
    fpk[page, :, off], fpv[page, :, off] = pk[kept], pv[kept]
    return _stored(s, False, torch.bfloat16)


def _stored(s, back, dtype):
    p = s["page"]
    page, off = s["slots"].clamp(min=0) // p, s["slots"].clamp(min=0) % p
    fk, fv, fpk, fpv = _fields(s["data"][0], s)
    k = _values(fk[page, :, off], fpk[page, :, off])
    v = _values(fv[page, :, off // 4, :, :, off % 4].flatten(-3), fpv[page, :, off])
    k = _rotated(k) if back else k
    none = (s["slots"] < 0)[:, None, None]
    return k.masked_fill(none, 0.0).to(dtype), v.masked_fill(none, 0.0).to(dtype)


def _read(s):
    return _stored(s, s["rotate"], DTYPES[s["dtype"]])


def _copy_pages(s):
    s["data"][:, s["dst"].long()] = s["data"][:, s["src"].long()]
    return s["data"]


def _attention(s):
    b, d, kv, heads = s["batch"], s["head_dim"], s["kv_heads"], s["heads"]
    fk, fv, fpk, fpv = _fields(s["data"][0][s["table"].long()], s)               # [b, width, kv, page, ...]
    k = _values(fk, fpk).transpose(1, 2).reshape(b, kv, -1, d)
    v = _values(fv.movedim(-2, -4).flatten(-3).flatten(-3, -2), fpv).transpose(1, 2).reshape(b, kv, -1, d)
    n, most = k.shape[2], s["q_most"]
    q = s["q"].float()
    q = _rotated(q) if s["rotate"] else q
    q_len = (s["q_start"][1:] - s["q_start"][:-1]).long()
    i = torch.arange(most, device=q.device)
    live = i < q_len[:, None]                                                    # [b, most]
    row = (s["q_start"][:-1, None].long() + i).clamp(max=q.shape[0] - 1)
    qp = q[row].view(b, most, kv, heads // kv, d).permute(0, 2, 3, 1, 4).reshape(b, kv, -1, d)
    t = torch.matmul(qp, k.transpose(-1, -2)).view(b, kv, heads // kv, most, n) * d ** -0.5
    j = torch.arange(n, device=q.device)
    pos = (s["kv_lens"].long() - q_len)[:, None] + i
    seen = (j < s["kv_lens"][:, None, None]).expand(b, most, n)
    if s["causal"]:
        seen = seen & (j <= pos[..., None])
    if s["window"]:
        seen = seen & (j > pos[..., None] - s["window"])
    t.masked_fill_(~seen[:, None, None], -math.inf)
    t.sub_(t.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = t.sum(-1, keepdim=True)
    o = torch.matmul(t.view(b, kv, -1, n), v).view(b, kv, heads // kv, most, d) / total.clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(b, most, heads, d)[live].to(s["q"].dtype)


# ---- the same from the definitions in 64 bits

def _sylvester(d):
    h = torch.ones((1, 1), dtype=torch.float64, device="cuda")
    while len(h) < d:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h / math.sqrt(d)


def _decoded(data, s, page):
    """Keys and values [tokens, kv heads, d] of the pages, in 64 bits."""
    kv, d, p = s["kv_heads"], s["head_dim"], s["page"]
    n = len(page)
    rec = data[page].view(n, kv, p * (d + 8)).to(torch.int32)
    at = torch.arange(p * d, device="cuda")
    nib = (rec[..., at // 2] >> (4 * (at % 2))) & 15                             # key codes
    tok, e = at // d, at % d
    per = d // 16
    run_, part, f = e // per, e % per // 4, e % 4
    byte = p * d // 2 + ((((tok // 4) * 16 + run_) * (d // 64) + part) * 4 + tok % 4) * 2 + f // 2
    vib = (rec[..., byte] >> (4 * (f % 2))) & 15
    word = rec[..., p * d:].view(n, kv, 2, p, 2, 2)
    bits = ((word[..., 0] | (word[..., 1] << 8)) << 16).view(torch.float32).double()
    out = [(c.view(n, kv, p, d) - 7.5) * bits[:, :, i, :, :1] + bits[:, :, i, :, 1:] for i, c in enumerate((nib, vib))]
    return [x.transpose(1, 2).reshape(n * p, kv, d) for x in out]


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    d, p = s["head_dim"], s["page"]
    h = _sylvester(d)
    if s["op"] == "copy_pages":
        return None
    if s["op"] in ("append", "read"):
        out = []
        if s["op"] == "read":
            pages = s["slots"] // p
            for part in torch.arange(len(pages), device="cuda").split(max(1, 16384 // p)):
                k, v = _decoded(s["data"][0], s, pages[part])
                row = torch.arange(len(part), device="cuda") * p + s["slots"][part] % p
                out.append((k[row] @ h if s["rotate"] else k[row], v[row]))
            return torch.cat([x[0] for x in out]), torch.cat([x[1] for x in out])
        clip = float(torch.tensor(s["clip"], dtype=torch.float32))
        for x, turn in ((s["k"].double(), s["rotate"]), (s["v"].double(), False)):
            y = x @ h if turn else x
            lo, hi = clip * y.amin(-1, keepdim=True), clip * y.amax(-1, keepdim=True)
            step, mid = ((hi - lo) / 15).to(torch.bfloat16).double(), ((hi + lo) / 2).to(torch.bfloat16).double()
            c = ((y - mid) / step.clamp(min=1e-30) + 7.5).round().clamp(0, 15)
            out.append(((c - 7.5) * step + mid) * (s["slots"] >= 0)[:, None, None])
        return tuple(out)
    group = s["heads"] // s["kv_heads"]
    ql, kl = _lens(case)
    if sum(a * b for a, b in zip(ql, kl)) * s["heads"] * d > 4e11:
        return None
    outs, at = [], 0
    for b, (nq, n) in enumerate(zip(ql, kl)):
        k, v = [], []
        for part in s["table"][b, :_pages(n, p)].long().split(max(1, 8192 // p)):
            x, y = _decoded(s["data"][0], s, part)
            k.append(x)
            v.append(y)
        k, v = torch.cat(k)[:n], torch.cat(v)[:n]
        o = torch.empty((nq, s["heads"], d), dtype=torch.float64, device="cuda")
        j = torch.arange(n, device="cuda")
        for head in range(s["heads"]):
            for part in torch.arange(nq, device="cuda").split(max(1, (1 << 26) // n)):
                q = s["q"][at + part, head].double()
                t = (q @ h if s["rotate"] else q) @ k[:, head // group].t() / math.sqrt(d)
                pos = (n - nq + part)[:, None]
                bad = torch.zeros_like(t, dtype=torch.bool)
                if s["causal"]:
                    bad |= j > pos
                if s["window"]:
                    bad |= j <= pos - s["window"]
                w = torch.softmax(t.masked_fill(bad, -math.inf), -1)
                o[part, head] = w @ v[:, head // group]
        outs.append(o)
        at += nq
    return torch.cat(outs)

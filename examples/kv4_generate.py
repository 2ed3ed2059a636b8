"""Serving with the 4-bit paged cache: a prompt in two chunks, two branches forked off it, decode steps, a branch that ends, compaction.

A toy transformer (attention only, random weights) whose cache is what rq_kv4_* keep: keys and values of every layer go through
kv4_append, queries through kv4_attention, branches and compaction through PagePool and kv4_copy_pages.  At the end the cached
rows come back with kv4_read, and the result is set against the same model without a cache.

    python examples/kv4_generate.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2504_13989_amd as rq  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM, LAYERS, VOCAB, PAGE = 8, 2, 128, 2, 256, 16
HIDDEN = HEADS * HEAD_DIM


class Model:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)

        self.embed = weight(VOCAB, HIDDEN) * HIDDEN ** 0.5
        self.qkv = [weight((HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN) for _ in range(LAYERS)]
        self.out = [weight(HIDDEN, HIDDEN) for _ in range(LAYERS)]

    def run(self, ids, attend):
        """Logits of the tokens; attend(layer, q, k, v) -> o, all [tokens, heads, head_dim] (q, k, v: slices of one product)."""
        x = self.embed[ids]
        for i in range(LAYERS):
            y = torch.nn.functional.rms_norm(x, (HIDDEN,))
            qkv = (y @ self.qkv[i].T).view(len(ids), HEADS + 2 * KV_HEADS, HEAD_DIM)
            o = attend(i, qkv[:, :HEADS], qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:])
            x = x + o.reshape(len(ids), HIDDEN) @ self.out[i].T
        return torch.nn.functional.rms_norm(x, (HIDDEN,)) @ self.embed.T


class Server:
    def __init__(self, model, pages=64):
        self.model, self.h = model, rq.hadamard_build(HEAD_DIM)
        self.cache = rq.kv4_cache(pages, KV_HEADS, HEAD_DIM, PAGE, layers=LAYERS)
        self.pool = rq.PagePool(pages, PAGE)

    def copy(self, pairs):
        if pairs:
            src, dst = torch.tensor(pairs, dtype=torch.int32).t().contiguous().cuda()
            rq.kv4_copy_pages(self.cache, src, dst)

    def feed(self, batch):
        """Appends tokens to sequences ({name: token ids}) and returns the logits behind each one's last token."""
        slots, copies, start = [], [], [0]
        for seq, ids in batch.items():
            new, pairs = self.pool.extend(seq, len(ids))
            slots += new
            copies += pairs
            start.append(start[-1] + len(ids))
        self.copy(copies)
        tables = [self.pool.table(seq) for seq in batch]
        width = max(map(len, tables))
        table = torch.tensor([t + [-1] * (width - len(t)) for t in tables], dtype=torch.int32).cuda()
        lens = torch.tensor([self.pool.length(seq) for seq in batch], dtype=torch.int32).cuda()
        slots = torch.tensor(slots).cuda()
        single = start[-1] == len(batch)          # a decode step: one token a sequence
        q_start = None if single else torch.tensor(start, dtype=torch.int32).cuda()

        def attend(layer, q, k, v):
            cache = self.cache.layer(layer)
            rq.kv4_append(self.h, cache, k, v, slots)
            return rq.kv4_attention(self.h, cache, q, table, lens, q_start)

        logits = self.model.run(torch.cat([torch.as_tensor(ids) for ids in batch.values()]).cuda(), attend)
        return dict(zip(batch, logits[torch.tensor(start[1:]).cuda() - 1]))


def plain_attention(layer, q, k, v):
    """Causal attention of one sequence without a cache."""
    k, v = (x.float().repeat_interleave(HEADS // KV_HEADS, 1).transpose(0, 1) for x in (k, v))
    s = q.float().transpose(0, 1) @ k.transpose(1, 2).contiguous() * HEAD_DIM ** -0.5
    n = s.shape[-1]
    s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
    return (s.softmax(-1) @ v).transpose(0, 1).to(q.dtype)


def main(steps=20, seed=0):
    """Returns how far the branches' last logits are from the model's without a cache (relative 2-norm), and the bytes of a cached token."""
    model = Model(seed)
    server = Server(model)
    prompt = torch.randint(0, VOCAB, (75,), generator=torch.Generator().manual_seed(seed)).tolist()
    server.pool.add("a")
    server.feed({"a": prompt[:50]})
    logits = server.feed({"a": prompt[50:]})["a"]                   # a chunk behind what is cached
    server.pool.fork("a", "b")                                      # both share the prompt's pages
    tokens = {"a": list(prompt), "b": list(prompt)}
    first = logits.topk(2).indices.tolist()
    step = {"a": [first[0]], "b": [first[1]]}                       # the two likeliest tokens
    for _ in range(steps):
        for seq, ids in step.items():
            tokens[seq] += ids
        last = server.feed(step)                                    # the first step copies the page that both would write to
        step = {seq: [int(x.argmax())] for seq, x in last.items()}
    server.pool.free("a")
    server.copy(server.pool.compact())                              # b's pages move to the front
    tokens["b"] += step["b"]
    last["b"] = server.feed({"b": step["b"]})["b"]

    far = {}
    for seq, x in last.items():
        want = model.run(torch.tensor(tokens[seq]).cuda(), plain_attention)[-1].float()
        far[seq] = float((x.float() - want).norm() / want.norm())
    table = server.pool.table("b")
    slots = torch.tensor([table[i // PAGE] * PAGE + i % PAGE for i in range(server.pool.length("b"))]).cuda()
    k, _ = rq.kv4_read(server.h, server.cache.layer(0), slots)      # keys in the model's own basis
    ids = torch.tensor(tokens["b"]).cuda()
    y = torch.nn.functional.rms_norm(model.embed[ids], (HIDDEN,)) @ model.qkv[0].T
    want = y.view(len(ids), -1, HEAD_DIM)[:, HEADS:HEADS + KV_HEADS].float()
    far["keys"] = float((k.float() - want).norm() / want.norm())
    return far, rq.kv4_page_bytes(KV_HEADS, HEAD_DIM, PAGE) // PAGE


if __name__ == "__main__":
    far, size = main()
    print("a cached token of a layer: %d bytes (%d in bfloat16)" % (size, 4 * KV_HEADS * HEAD_DIM))
    for name, x in far.items():
        print("%-5s off by %.3f" % (name, x))

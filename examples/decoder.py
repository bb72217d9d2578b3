"""A small decoder, trained on packed documents and then served.

    python examples/decoder.py [--steps 60] [--requests 12] [--new 24]

Training packs documents of all lengths into one row of tokens:
``softmax_packed_attention`` keeps each document's tokens to themselves and
gives the gradients.  Serving keeps the keys and values of all requests in one
paged cache: a step takes prompt chunks and single tokens of any requests
together, ``softmax_cache_slots`` hands out blocks and slots for the new tokens
on the device, ``softmax_cache_append`` writes their keys and values, and
``softmax_paged_attention_fwd`` reads them.  Positions come from a bias that
falls with distance, scores are capped, both in training and in serving.

The data are synthetic: in a document the next token follows from the last
one by a fixed random table, with a part of the tokens drawn anew.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1904_12380_amd as sm  # noqa: E402

VOCAB, WIDTH, LAYERS, HEADS, KV_HEADS, HEAD = 256, 256, 2, 8, 2, 64
CAP = 30.0


class Decoder(torch.nn.Module):
    """Attention and a two-layer block per layer; float32 parameters, bfloat16
    queries, keys and values."""

    def __init__(self, device="cuda"):
        super().__init__()
        linear = lambda i, o: torch.nn.Linear(i, o, bias=False, device=device)  # noqa: E731
        self.embed = torch.nn.Embedding(VOCAB, WIDTH, device=device)
        self.qkv = torch.nn.ModuleList(linear(WIDTH, (HEADS + 2 * KV_HEADS) * HEAD)
                                       for _ in range(LAYERS))
        self.out = torch.nn.ModuleList(linear(HEADS * HEAD, WIDTH) for _ in range(LAYERS))
        self.up = torch.nn.ModuleList(linear(WIDTH, 4 * WIDTH) for _ in range(LAYERS))
        self.down = torch.nn.ModuleList(linear(4 * WIDTH, WIDTH) for _ in range(LAYERS))
        self.head = linear(WIDTH, VOCAB)
        self.register_buffer("slopes", torch.tensor(
            [2.0 ** (-8.0 * (i + 1) / HEADS) for i in range(HEADS)], device=device))

    def forward(self, tokens, attend):
        """Logits of ``tokens``; ``attend(layer, q, k, v)`` is the attention of
        [tokens, heads, d] slices of one projection."""
        x = self.embed(tokens)
        for i in range(LAYERS):
            rows = self.qkv[i](_norm(x)).bfloat16().unflatten(1, (-1, HEAD))
            q, k, v = rows.split([HEADS, KV_HEADS, KV_HEADS], 1)
            x = x + self.out[i](attend(i, q, k, v).float().flatten(1))
            x = x + self.down[i](torch.relu(self.up[i](_norm(x))))
        return self.head(_norm(x))

    def packed(self, tokens, cu):
        """Logits of packed documents, differentiable."""
        return self(tokens, lambda _, q, k, v: sm.softmax_packed_attention(
            q, k, v, cu, cap=CAP, slopes=self.slopes))


def _norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


class Server:
    """A paged cache for each layer, and the requests' block tables over it.
    Lengths, tables and the free list stay on the device."""

    def __init__(self, model, requests, blocks=256, size=16, width=64):
        device = model.slopes.device
        self.model, self.size = model, size
        self.caches = torch.zeros(LAYERS, 2, blocks, size, KV_HEADS, HEAD, dtype=torch.bfloat16,
                                  device=device)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device=device)
        self.held = torch.zeros(requests, dtype=torch.int32, device=device)
        self.free = torch.arange(blocks, dtype=torch.int32, device=device)
        self.left = torch.tensor([blocks], dtype=torch.int32, device=device)

    @torch.no_grad()
    def step(self, tokens, lens):
        """Logits of new tokens, ``lens[b]`` (int32, on the device) of request
        b; any of them may be a single token, a chunk or nothing."""
        s = sm.softmax_cache_slots(self.held, lens, self.table, self.free, self.left,
                                   len(tokens), self.size)
        self.held, self.left, self.missing = s["key_lens"], s["free_count"], s["missing"]

        def attend(layer, q, k, v):
            k_cache, v_cache = self.caches[layer]
            sm.softmax_cache_append(k, v, k_cache, v_cache, s["slots"])
            return sm.softmax_paged_attention_fwd(q, k_cache, v_cache, self.table, s["cu_q"],
                                                  s["key_lens"], cap=CAP,
                                                  slopes=self.model.slopes)
        return self.model(tokens, attend)


def documents(g, table, count, longest):
    """(tokens, sums of the lengths) of documents of 2 .. longest tokens."""
    lens = torch.randint(2, longest + 1, (count,), generator=g)
    rows = []
    for n in lens.tolist():
        doc = [int(torch.randint(VOCAB, (1,), generator=g))]
        fresh = torch.rand(n, generator=g) < 0.1
        drawn = torch.randint(VOCAB, (n,), generator=g)
        for i in range(1, n):
            doc.append(int(drawn[i]) if fresh[i] else int(table[doc[-1]]))
        rows += doc
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    return torch.tensor(rows).cuda(), cu.to(torch.int32).cuda(), lens.tolist()


def train(model, g, table, steps):
    """The loss of each step."""
    opt = torch.optim.AdamW(model.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        tokens, cu, lens = documents(g, table, 24, 120)
        last = cu[1:].long() - 1  # a document's last token has no successor in it
        keep = torch.ones(len(tokens), dtype=torch.bool, device=tokens.device)
        keep[last] = False
        logp = torch.log_softmax(model.packed(tokens, cu), 1)
        loss = -logp[keep].gather(1, tokens.roll(-1)[keep][:, None]).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


def serve(model, prompts, new):
    """The prompts' logits and ``new`` greedy tokens of each, its prompt taken
    in two chunks while requests with short prompts already decode."""
    n = len(prompts)
    device = prompts[0].device
    server = Server(model, n)
    first = [len(p) if len(p) < 20 else len(p) // 2 for p in prompts]
    lens = torch.tensor(first, dtype=torch.int32, device=device)
    parts = server.step(torch.cat([p[:k] for p, k in zip(prompts, first)]), lens).split(first)
    logits = [[x] for x in parts]
    out = [[] for _ in prompts]
    rest = [p[k:] for p, k in zip(prompts, first)]
    for i in range(new):
        tokens = []
        for b in range(n):
            if len(rest[b]):
                tokens.append(rest[b])
                rest[b] = rest[b][:0]
            else:
                out[b].append(logits[b][-1][-1:].argmax(1))
                tokens.append(out[b][-1])
        count = [len(t) for t in tokens]
        got = server.step(torch.cat(tokens), torch.tensor(count, dtype=torch.int32, device=device))
        for x, y in zip(logits, got.split(count)):
            x.append(y)
    assert int(server.missing) == 0, "the cache ran out of blocks"
    return [torch.cat(x) for x in logits], [torch.cat(o) for o in out]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--requests", type=int, default=12)
    p.add_argument("--new", type=int, default=24)
    a = p.parse_args(argv)
    torch.manual_seed(1)
    g = torch.Generator().manual_seed(2)
    table = torch.randperm(VOCAB, generator=g)
    model = Decoder()
    losses = train(model, g, table, a.steps)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} in {a.steps} steps", flush=True)

    tokens, _, lens = documents(g, table, a.requests, 200)
    prompts = list(tokens.split(lens))
    logits, out = serve(model, prompts, a.new)
    # The same tokens as packed documents.
    whole = [torch.cat([p, o]) for p, o in zip(prompts, out)]
    cu = torch.tensor([0] + [len(w) for w in whole], device=tokens.device).cumsum(0).int()
    with torch.no_grad():
        want = model.packed(torch.cat(whole), cu)
    have = torch.cat(logits)
    worst = float((have - want).abs().max())
    right = sum(int((table.cuda()[w[len(p) - 1:-1]] == w[len(p):]).sum())
                for w, p in zip(whole, prompts))
    made = sum(len(o) for o in out)
    print(f"served {made} tokens of {a.requests} requests: logits within {worst:.2e} of the packed "
          f"documents', {right} follow the table", flush=True)
    return losses, worst, right / made


if __name__ == "__main__":
    main()

"""Speculative decoding on an attention worker in front of an expert worker.

A small mixture-of-experts decoder with random weights: every layer normalises
and rotates queries and keys into the paged cache (``QkNormRope``), attends
over the cache and the drafted tree (``TreeAttention``) and sends the rows
through the expert forward (``EwForward``); a step ends with the verification
of the drafted tokens (``VerifyTree``), the compaction of the kept rows and the
checkpoint of their KV segments. Greedy decoding of drafted trees must give the
tokens of greedy decoding one by one, in fewer forwards (where two tokens' logits
are as good as equal, rounding decides).

    python examples/spec_decode.py [tokens]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_01310_amd import spec, synth, tg  # noqa: E402

D_MODEL, LAYERS, HQ, HKV, D, VOCAB, PAGE = 256, 2, 4, 2, 64, 512, 16
# Logits that lie no further apart are a tie: activations of 16 bits, added in
# other orders, move them by up to half of this.
TIE = 2.0 ** -5
# The drafted tree: node 0 is the last sampled token; (parent, which of the
# parent's candidates) of the others.
TREE = [(None, 0), (0, 0), (0, 1), (1, 0), (1, 1), (3, 0), (3, 1), (5, 0)]


def weights(device):
    g = torch.Generator(device=device)
    g.manual_seed(7)

    def w(*shape, std):
        return (torch.randn(shape, generator=g, device=device) * std).to(torch.bfloat16)

    angle = torch.arange(2048, device=device)[:, None] * 10000.0 ** (
        -torch.arange(0, D, 2, device=device) / D)[None, :]
    return dict(
        embed=w(VOCAB, D_MODEL, std=1.0), unembed=w(D_MODEL, VOCAB, std=0.1),
        qkv=[w(D_MODEL, (HQ + 2 * HKV) * D, std=0.06) for _ in range(LAYERS)],
        out=[w(HQ * D, D_MODEL, std=0.02) for _ in range(LAYERS)],
        norm=[(1 + w(D, std=0.1)).to(torch.bfloat16) for _ in range(2 * LAYERS)],
        cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float().contiguous())


def rms(x):
    return (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Worker:
    """A batch of B requests, up to T rows per forward and ``max_tokens`` in the
    cache per request, those of the rows in flight included."""

    def __init__(self, w, B, T, max_tokens=256, device="cuda"):
        if max_tokens > w["cos_sin"].shape[0]:
            raise ValueError(f"{max_tokens} tokens: angles for {w['cos_sin'].shape[0]} only")
        ints = dict(dtype=torch.int32, device=device)
        self.w, self.B, self.T = w, B, T
        width = -(-max_tokens // PAGE) + 1
        self.cache = spec.KvCache.empty(LAYERS, B * width, PAGE, HKV, D, B, width, device=device)
        self.lengths, self.new_lengths = torch.zeros(B, **ints), torch.zeros(B, **ints)
        self.offsets = torch.zeros(B + 1, **ints)
        self.tokens, self.slots = torch.zeros(T, **ints), torch.zeros(T, **ints)
        self.positions, self.status = torch.zeros(T, **ints), torch.zeros(B, **ints)
        self.mask = torch.zeros((T, 1), dtype=torch.int64, device=device)
        qkv = torch.zeros((T, HQ + 2 * HKV, D), dtype=torch.bfloat16, device=device)
        self.qkv = qkv
        self.rope = [spec.QkNormRope(self.cache, qkv, HQ, self.positions, self.slots, w["cos_sin"],
                                     w["norm"][2 * i], w["norm"][2 * i + 1]) for i in range(LAYERS)]
        self.attend = [spec.TreeAttention(self.cache, r.q_out, self.offsets, self.lengths,
                                          self.mask) for r in self.rope]
        for a in self.attend:
            a.out.zero_()  # rows that no request has are not written
        self.experts = [tg.EwForward(synth.make_custom(
            T=T, d=D_MODEL, E=8, k=2, I=512, n_local=8, shadow_experts=[0], gate="weights",
            seed=50 + i, device=device)) for i in range(LAYERS)]

    def forward(self):
        """Logits [T, VOCAB] of the rows that tokens, offsets, mask and
        positions describe; their K and V are in the cache afterwards."""
        w = self.w
        self.cache.reserve(self.lengths, self.offsets, self.slots, self.status)
        if not self.status.all():
            raise RuntimeError("the cache has no pages for these rows")
        x = w["embed"][self.tokens.long()].float()
        for i in range(LAYERS):
            torch.mm(rms(x), w["qkv"][i], out=self.qkv.view(self.T, -1))
            self.rope[i](layer=i)
            x = x + torch.mm(self.attend[i](layer=i).view(self.T, -1), w["out"][i]).float()
            self.experts[i].wl.x.copy_(rms(x))
            x = x + 0.3 * self.experts[i]().float()
        return torch.mm(rms(x).float(), w["unembed"].float())

    def rows(self, tokens, masks, depths):
        """Lays out the rows of all requests: lists per request."""
        flat = [t for r in tokens for t in r]
        off = [0]
        for r in tokens:
            off.append(off[-1] + len(r))
        pad = self.T - len(flat)
        base = self.lengths.tolist()
        place = [base[b] + d for b, r in enumerate(depths) for d in r]
        self.tokens.copy_(torch.tensor(flat + [0] * pad))
        self.offsets.copy_(torch.tensor(off))
        self.positions.copy_(torch.tensor(place + [0] * pad))
        self.mask.copy_(torch.tensor([m for r in masks for m in r] + [0] * pad)[:, None])
        return off

    def prefill(self, prompts):
        """All but the last token of each prompt into the cache, in chains."""
        todo = [list(p[:-1]) for p in prompts]
        most = min(self.T // self.B, 63)  # a row's mask is one signed word here
        while any(todo):
            part = [t[:most] for t in todo]
            todo = [t[most:] for t in todo]
            self.rows(part, [[(2 << i) - 1 for i in range(len(r))] for r in part],
                      [list(range(len(r))) for r in part])
            self.forward()
            self.lengths += torch.diff(self.offsets)


def room(prompts, n, nodes):
    """Cached tokens that a request of the batch may need: a request ends with
    its n-th token, which a step may pass by the nodes of a tree."""
    return max(256, max(map(len, prompts)) + n + nodes)


def greedy(w, prompts, n):
    """n tokens of each request, one forward per token."""
    B = len(prompts)
    worker = Worker(w, B, B, room(prompts, n, 1))
    worker.prefill(prompts)
    last, out = [p[-1] for p in prompts], [[] for _ in prompts]
    for _ in range(n):
        worker.rows([[t] for t in last], [[1]] * B, [[0]] * B)
        last = worker.forward().argmax(1).tolist()
        worker.lengths += 1
        for b in range(B):
            out[b].append(last[b])
    return out


def speculative(w, prompts, n, store=None):
    """The same tokens from drafted trees; returns them and the forwards
    needed. ``store``: a pinned host copy of the K pages to checkpoint into."""
    B, N = len(prompts), len(TREE)
    worker = Worker(w, B, B * N, room(prompts, n, N))
    worker.prefill(prompts)
    masks, depths = [1], [0]
    for j, (up, _) in enumerate(TREE[1:], 1):
        masks.append(masks[up] | 1 << j)
        depths.append(depths[up] + 1)
    # A draft model without layers: the likeliest tokens after each token.
    draft = torch.topk(torch.mm(rms(w["embed"].float()), w["unembed"]).float(), 2, 1).indices.cpu()
    probs = torch.zeros((B * N, VOCAB), device="cuda")
    zeros = torch.zeros(B * N, device="cuda")
    check = spec.VerifyTree(probs, worker.tokens, zeros, zeros[:B], worker.offsets, worker.mask,
                            max_path=N, status=worker.status)
    last, out, steps, seq = [p[-1] for p in prompts], [[] for _ in prompts], 0, 1
    while min(len(o) for o in out) < n:
        tokens = []
        for b in range(B):
            t = [last[b]]
            for up, which in TREE[1:]:
                t.append(int(draft[t[up], which]))
            tokens.append(t)
        going = [len(o) < n for o in out]  # a request ends with its n-th token
        worker.rows(*([x if on else [] for x, on in zip(rows, going)]
                      for rows in (tokens, [masks] * B, [depths] * B)))
        logits = worker.forward()
        probs.zero_().scatter_(1, logits.argmax(1, keepdim=True), 1.0)  # greedy: all mass on one
        new, path, kept = check()
        worker.cache.compact(path, kept, worker.lengths, worker.new_lengths)
        if store is not None:
            seq = checkpoint(worker, kept, store, seq)
        worker.lengths.copy_(worker.new_lengths)
        worker.cache.trim(worker.lengths)  # pages of refused rows
        steps += 1
        for b, (row, k) in enumerate(zip(new.tolist(), kept.tolist())):
            if k:
                out[b] += row[:k]
                last[b] = row[k - 1]
    return [o[:n] for o in out], steps, worker


def checkpoint(worker, kept, store, seq):
    """The kept rows' K segments of every layer, to host memory (V goes the
    same way): one segment per token and layer."""
    c, size = worker.cache, HKV * D * 2
    table, base, n = c.page_table.tolist(), worker.lengths.tolist(), kept.tolist()
    offsets = []
    for layer in range(LAYERS):
        for b in range(worker.B):
            for p in range(base[b], base[b] + n[b]):
                row = table[b][p // PAGE] * PAGE + p % PAGE
                offsets.append((layer * c.args.n_pages * PAGE + row) * size)
    off = torch.tensor(offsets, dtype=torch.int64, device="cuda")
    nbytes = torch.full((len(offsets),), size, dtype=torch.int32, device="cuda")
    tg.tg_kv_checkpoint(c.k, c.k.numel() * 2, off, nbytes, len(offsets), seq, store["k"],
                        store["log"], store["log"].shape[0], store["commit"])
    return seq + len(offsets)


def host_store(worker_cache_bytes):
    return dict(k=torch.zeros(worker_cache_bytes, dtype=torch.uint8, pin_memory=True),
                log=torch.zeros((4096, 3), dtype=torch.int64, pin_memory=True),
                commit=torch.zeros(1, dtype=torch.int64, pin_memory=True))


def apart(w, prompt, tokens, other):
    """How far apart the logits of the last token and of ``other`` lie after the
    prompt and the tokens before."""
    seq = prompt + tokens[:-1]
    worker = Worker(w, 1, 32, room([seq], 1, 32))
    worker.prefill([seq])
    worker.rows([seq[-1:]], [[1]], [[0]])
    logits = worker.forward()[0]
    return float((logits[tokens[-1]] - logits[other]).abs())


def main(n=40):
    w = weights("cuda")
    g = torch.Generator()
    g.manual_seed(3)
    prompts = [torch.randint(0, VOCAB, (k,), generator=g).tolist() for k in (5, 1, 23, 40)]
    one_by_one = greedy(w, prompts, n)
    tokens, steps, _ = speculative(w, prompts, n)
    gaps = []  # where a request's tokens part
    for p, a, b in zip(prompts, one_by_one, tokens):
        if a != b:
            i = next(i for i in range(n) if a[i] != b[i])
            gaps.append(apart(w, p, a[:i + 1], b[i]))
    if max(gaps, default=0.0) > TIE:
        raise RuntimeError(f"different tokens, whose logits lie {max(gaps)} apart")
    print(f"{n} tokens of {len(prompts)} requests: {steps} forwards of drafted trees instead of {n}; "
          f"the same tokens{f' up to ties, {max(gaps):.4f} apart' if gaps else ''}")
    return tokens, one_by_one, steps


if __name__ == "__main__":
    main(*[int(x) for x in sys.argv[1:2]])

"""Several samples of one prompt: a decode step whose requests share a prefix.

The model of ``spec_decode.py``. The prompt goes into the cache once; its request
is forked (``KvCache.fork``), and every sample goes on by itself: each step attends
over the shared pages once for all samples (``PrefixAttention``), sends the few rows
through the experts (``EwFew``) and draws the next tokens with temperature, top-k,
top-p and min-p (``SampleTokens``).

    python examples/parallel_sampling.py [samples] [tokens]
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import spec_decode as base  # noqa: E402
from paper_2601_01310_amd import spec, tg  # noqa: E402


class Sampler:
    """``n`` samples of ``prompt``, up to ``most`` tokens each."""

    def __init__(self, w, prompt, n, most, temperature=0.8, top_k=50, top_p=0.95, min_p=0.01):
        if not 2 <= n <= tg.MAX_FEW:
            raise ValueError(f"{n} samples: 2 to {tg.MAX_FEW}")
        self.w, self.n = w, n
        worker = self.worker = base.Worker(w, n, 8 * n, base.room([prompt], most, 1))
        worker.prefill([prompt] + [[0]] * (n - 1))
        ints = dict(dtype=torch.int32, device="cuda")
        self.cache, self.lengths = worker.cache, worker.lengths
        status = torch.zeros(n - 1, **ints)
        self.cache.fork(self.lengths, torch.zeros(n - 1, **ints), torch.arange(1, n, **ints), status)
        if not status.all():
            raise RuntimeError("the cache has no pages for the samples")
        # A fork shares whole pages and copies a last one that is in part used.
        whole = (len(prompt) - 1) // base.PAGE * base.PAGE
        groups = torch.tensor([0, n], **ints), torch.tensor([whole], **ints)
        self.offsets = torch.arange(n + 1, **ints)
        self.slots, self.status = torch.zeros(n, **ints), torch.zeros(n, **ints)
        self.tokens = torch.full((n,), prompt[-1], **ints)
        self.qkv = torch.zeros((n, base.HQ + 2 * base.HKV, base.D), dtype=torch.bfloat16, device="cuda")
        self.positions = torch.zeros(n, **ints)
        self.rope = [spec.QkNormRope(self.cache, self.qkv, base.HQ, self.positions, self.slots,
                                     w["cos_sin"], w["norm"][2 * i], w["norm"][2 * i + 1])
                     for i in range(base.LAYERS)]
        self.attend = [spec.PrefixAttention(self.cache, r.q_out, self.offsets, self.lengths, *groups,
                                            max_nodes=1) for r in self.rope]
        self.x = torch.zeros((n, base.D_MODEL), dtype=torch.bfloat16, device="cuda")
        wls = [e.wl for e in worker.experts]
        self.experts = [tg.EwFew(self.x, wl.wg, None, wl.ert, wl.alive, wl.w13, wl.w2, wl.k)
                        for wl in wls]
        self.logits = torch.zeros((n, base.VOCAB), device="cuda")
        self.u = torch.zeros(n, device="cuda")
        every = lambda v, dtype: torch.full((n,), v, dtype=dtype, device="cuda")  # noqa: E731
        self.draw = spec.SampleTokens(self.logits, self.u, every(temperature, torch.float32),
                                      every(top_k, torch.int32), every(top_p, torch.float32),
                                      every(min_p, torch.float32))

    def step(self, u):
        """The next token of every sample by the random numbers ``u`` [n]."""
        w = self.w
        self.cache.reserve(self.lengths, self.offsets, self.slots, self.status)
        self.positions.copy_(self.lengths)
        x = w["embed"][self.tokens.long()].float()
        for i in range(base.LAYERS):
            torch.mm(base.rms(x), w["qkv"][i], out=self.qkv.view(self.n, -1))
            self.rope[i](layer=i)
            x = x + torch.mm(self.attend[i](layer=i).view(self.n, -1), w["out"][i]).float()
            self.x.copy_(base.rms(x))
            x = x + 0.3 * self.experts[i]().float()
        torch.mm(base.rms(x).float(), w["unembed"].float(), out=self.logits)
        self.u.copy_(u)
        self.tokens.copy_(self.draw())
        self.lengths += 1
        return self.tokens


def main(samples=8, most=24):
    w = base.weights("cuda")
    g = torch.Generator()
    g.manual_seed(5)
    prompt = torch.randint(0, base.VOCAB, (150,), generator=g).tolist()
    s = Sampler(w, prompt, samples, most)
    out = torch.stack([s.step(torch.rand(samples, generator=g).cuda()).clone() for _ in range(most)], 1)
    if not s.status.all():
        raise RuntimeError("the cache had no pages for these rows")
    rows = out.tolist()
    print(f"{samples} samples of {most} tokens behind one prompt of {len(prompt)}: "
          f"{len(set(map(tuple, rows)))} different ones")
    return rows, prompt, s


if __name__ == "__main__":
    main(*[int(x) for x in sys.argv[1:3]])

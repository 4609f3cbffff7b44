"""What is measured of the operators around the paged KV cache of an attention
worker: one speculative decode step, part by part.

A case is a dict of plain values; ``op`` names the operator:

* ``qk``      per-head norms of queries and keys and their rotation by the
              row's position, K and V rows written into their cache pages;
* ``attn``    attention of each request's rows (one token, or a tree of
              drafted tokens) over its cached tokens;
* ``verify``  which drafted tokens stay, and the next token, from the
              target's probabilities and given random numbers;
* ``compact`` the accepted rows of every layer moved together in the cache;
* ``pages``   requests forked, rows reserved and pages given back.

``own`` selects the framework's kernels; the plain form computes the same in
elementary torch operations. Sizes: the attention heads of the Mixtral-8x7B
layer that ``synth.CONFIGS`` names (32 query and 8 KV heads of 128, 4096-byte
KV segments, 32 layers as in ``perf/cases.py``), and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
MIXTRAL = dict(Hq=32, Hkv=8, D=128)
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    return [
        # One new token of one request: latency.
        dict(name="qk_one", op="qk", T=1, **MIXTRAL, rot=128, pairs="half", dtype="bf16", page=16),
        # 64 requests with 16 drafted tokens each, small heads of which only
        # half is rotated, in neighbouring pairs.
        dict(name="qk_tree", op="qk", T=1024, Hq=24, Hkv=4, D=64, rot=32, pairs="next", dtype="f16",
             page=32),
        # A prefill chunk.
        dict(name="qk_prefill", op="qk", T=16383, **MIXTRAL, rot=128, pairs="half", dtype="bf16",
             page=16),
        # One token of one request over a short context: latency.
        dict(name="attn_one", op="attn", B=1, N=1, L=1023, **MIXTRAL, dtype="bf16", page=16),
        # An ordinary decode batch, ragged contexts: the cache's bytes.
        dict(name="attn_decode", op="attn", B=128, N=1, L=8192, **MIXTRAL, dtype="bf16", page=16),
        # Trees of up to 33 rows over ragged contexts.
        dict(name="attn_tree", op="attn", B=16, N=33, L=4096, **MIXTRAL, dtype="bf16", page=32),
        # One request with a very long context and a few drafted tokens.
        dict(name="attn_long", op="attn", B=1, N=7, L=131071, **MIXTRAL, dtype="bf16", page=64),
        # Wide trees and eight query heads to a KV head: matrix products.
        dict(name="attn_wide", op="attn", B=8, N=64, L=16384, Hq=64, Hkv=8, D=128, dtype="f16",
             page=64),
        # A small tree of one request over a 32000-token vocabulary: latency.
        dict(name="verify_one", op="verify", B=1, N=8, V=32000, sampled=False),
        # A batch of sampled chains over a large vocabulary.
        dict(name="verify_chain", op="verify", B=128, N=6, V=128000, sampled=True),
        # Accepted rows of 64 requests moved together in 32 layers.
        dict(name="compact", op="compact", B=64, N=16, layers=32, Hkv=8, D=128, dtype="bf16",
             page=16),
        # Eight of 64 requests are forked twice, all reserve rows for their
        # drafts, everything is given back.
        dict(name="pages", op="pages", B=64, N=16, L=2000, forks=16, layers=32, Hkv=8, D=128,
             dtype="bf16", page=16),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    D = rng.choice((64, 128, 128, 256))
    Hkv = rng.choice((1, 2, 4, 8))
    return dict(Hq=Hkv * rng.choice((1, 2, 3, 4, 6, 8)), Hkv=Hkv, D=D)


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(("qk", "qk", "attn", "attn", "attn", "attn", "verify", "verify", "compact",
                     "pages"))
    dtype, page = rng.choice(("bf16", "bf16", "f16")), rng.choice((8, 16, 32, 64, 128))
    if op == "qk":
        h = _heads(rng)
        T = _log(rng, 1, min(16384, 80_000_000 // ((h["Hq"] + 2 * h["Hkv"]) * h["D"])))
        return dict(op=op, T=T, **h, rot=h["D"] // rng.choice((1, 1, 2)),
                    pairs=rng.choice(("half", "half", "next")), dtype=dtype, page=page)
    if op == "attn":
        h, B = _heads(rng), _log(rng, 1, 128)
        N = rng.choice((1, 1, _log(rng, 2, 64)))
        row = h["Hkv"] * h["D"] * B
        L = _log(rng, 16, max(32, min(131072, 500_000_000 // row,
                                      2_000_000_000 // (N * h["Hq"] * h["D"] * B // 4))))
        return dict(op=op, B=B, N=N, L=L, **h, dtype=dtype, page=page)
    if op == "verify":
        V, sampled = _log(rng, 1000, 160000), rng.random() < 0.5
        N = _log(rng, 2, 64)
        B = _log(rng, 1, max(1, min(128, 98_000_000 // (V * N))))
        return dict(op=op, B=B, N=N, V=V, sampled=sampled)
    layers, N = rng.choice((1, 8, 32)), _log(rng, 6, 32)
    Hkv, D = rng.choice((2, 4, 8)), rng.choice((64, 128))
    case = dict(op=op, B=_log(rng, 1, 64), N=N, layers=layers, Hkv=Hkv, D=D, dtype=dtype, page=page)
    if op == "pages":
        case.update(B=max(4, case["B"]), L=_log(rng, 16, 2000))
        case["page"] = min(page, 32)
        case["forks"] = rng.randint(1, case["B"] // 4)
    return case


# --------------------------------------------------------------------------
# What a program has in hand before the call.
# --------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 71)
    return g


def _normal(shape, dtype, g, std=1.0):
    """Normal values of a 16-bit type, drawn in pieces."""
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device=DEV).mul_(std))
    return t


def _shape_rng(case):
    """Ragged lengths go by the case, not by the seed: its work is known."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """(committed tokens, rows) of each request: a long one, the others ragged."""
    r = _shape_rng(case)
    L = [case["L"]] + [max(1, int(case["L"] * r.uniform(0.1, 1.0))) for _ in range(case["B"] - 1)]
    N = [case["N"]] + [max(1, int(case["N"] * r.uniform(0.3, 1.0))) for _ in range(case["B"] - 1)]
    return L, N


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _offsets(N):
    off = [0]
    for n in N:
        off.append(off[-1] + n)
    return off


def _trees(N, rng, chain=False):
    """Ancestor bits of each node (its own among them) and its depth, parents
    before children."""
    masks, depths = [], []
    for n in N:
        m, d = [1], [0]
        for j in range(1, n):
            p = j - 1 if chain else rng.randrange(max(0, j - 6), j)
            m.append(m[p] | 1 << j)
            d.append(d[p] + 1)
        masks += m
        depths += d
    return torch.tensor([x - (1 << 64) if x >> 63 else x for x in masks], dtype=torch.int64,
                        device=DEV)[:, None].contiguous(), depths


def _pool(case, tokens, g, spare=0):
    """K and V pages in no order, [layers, pages, page, Hkv, D], and the page
    table of requests that hold ``tokens`` each."""
    page, layers = case["page"], case.get("layers", 1)
    held = [-(-t // page) for t in tokens]
    n = sum(held) + spare
    order = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    width = max(held) + 4
    table = torch.full((len(tokens), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    refs = torch.zeros(n, dtype=torch.int32, device=DEV)
    refs[order[:at].long()] = 1
    dims, dtype = (layers, n, page, case["Hkv"], case["D"]), DTYPES[case["dtype"]]
    return dict(k=_normal(dims, dtype, g), v=_normal(dims, dtype, g), table=table,
                held=_ints(held), refs=refs)


def _cache(case, s):
    from paper_2601_01310_amd import spec
    return spec.KvCache(s["k"], s["v"], s["table"], s["held"], s["refs"])


def prepare(case, seed):
    s = globals()["_prepare_" + case["op"]](case, int(seed))
    s["case"] = case
    return s


def _prepare_qk(case, seed):
    g, T, D, dtype = _gen(seed), case["T"], case["D"], DTYPES[case["dtype"]]
    heads = case["Hq"] + 2 * case["Hkv"]
    s = _pool(case, [T], g, spare=3)
    s["qkv"] = _normal((T, heads, D), dtype, g)
    s["qw"], s["kw"] = (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(dtype), \
        (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    places = 32768
    angle = torch.arange(places, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])[None, :]
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
    s["positions"] = (torch.arange(T, device=DEV) + int(torch.randint(0, places - T, (1,), generator=g, device=DEV))).int()
    at = torch.arange(T, device=DEV)
    s["slots"] = (s["table"][0, at // case["page"]] * case["page"] + at % case["page"]).int()
    if own:
        from paper_2601_01310_amd import spec
        s["call"] = spec.QkNormRope(_cache(case, s), s["qkv"], case["Hq"], s["positions"], s["slots"],
                                    s["cos_sin"], s["qw"], s["kw"], eps=EPS,
                                    interleaved=case["pairs"] == "next")
    return s


def _prepare_attn(case, seed):
    g, (L, N) = _gen(seed), _lengths(case)
    s = _pool(case, [a + b for a, b in zip(L, N)], g)
    off = _offsets(N)
    s["q"] = _normal((off[-1], case["Hq"], case["D"]), DTYPES[case["dtype"]], g)
    s["lengths"], s["offsets"] = _ints(L), _ints(off)
    s["mask"], _ = _trees(N, random.Random(seed))
    if own:
        from paper_2601_01310_amd import spec
        s["call"] = spec.TreeAttention(_cache(case, s), s["q"], s["offsets"], s["lengths"],
                                       s["mask"], max_nodes=max(N))
    return s


def _prepare_verify(case, seed):
    g, V = _gen(seed), case["V"]
    N = _lengths(dict(case, L=1))[1] if not case["sampled"] else [case["N"]] * case["B"]
    off = _offsets(N)
    T = off[-1]
    s = dict(offsets=_ints(off))
    s["mask"], _ = _trees(N, random.Random(seed), chain=case["sampled"])

    def draws(probs):  # one token of each row
        return torch.multinomial(probs, 1, generator=g)[:, 0]

    logits = torch.randn((T, V), generator=g, device=DEV).mul_(3.0)
    s["p"] = torch.softmax(logits, 1)
    s["q"] = None
    if case["sampled"]:  # a draft that is near the target: most tokens stay
        logits.add_(torch.randn((T, V), generator=g, device=DEV), alpha=0.5)
        s["q"] = torch.softmax(logits, 1)
        tokens = torch.roll(draws(s["q"]), 1)
    else:  # the likeliest tokens after each node, dealt to its children
        top = torch.topk(s["p"], min(16, V), dim=1).indices.cpu()
        masks, picks, seen = s["mask"][:, 0].tolist(), [0] * T, {}
        for b in range(case["B"]):
            for j in range(1, N[b]):
                up = masks[off[b] + j] & ((1 << j) - 1)
                at = off[b] + up.bit_length() - 1
                seen[at] = seen.get(at, -1) + 1
                picks[off[b] + j] = int(top[at, seen[at]])
        tokens = torch.tensor(picks, device=DEV)
    s["tokens"] = tokens.int()
    s["u"] = torch.rand(T, generator=g, device=DEV)
    s["u_next"] = torch.rand(case["B"], generator=g, device=DEV)
    if own:
        from paper_2601_01310_amd import spec
        s["call"] = spec.VerifyTree(s["p"], s["tokens"], s["u"], s["u_next"], s["offsets"],
                                    s["mask"], max_path=max(N), max_nodes=max(N),
                                    draft_probs=s["q"])
    return s


def _paths(case):
    """Accepted nodes of each request, the root first; every other one moves."""
    r, paths = _shape_rng(case), []
    for _ in range(case["B"]):
        paths.append([0] + sorted(r.sample(range(2, case["N"]), r.randint(1, case["N"] // 2 - 1))))
    return paths


def _prepare_compact(case, seed):
    g, B, N, r = _gen(seed), case["B"], case["N"], _shape_rng(case)
    L = [r.randint(1, 3 * case["page"]) for _ in range(B)]
    s = _pool(case, [x + N for x in L], g)
    paths = _paths(case)
    s["lengths"], s["keep"] = _ints(L), _ints([len(p) for p in paths])
    s["path"] = _ints([p + [-1] * (N - len(p)) for p in paths])
    s["new_lengths"] = torch.zeros_like(s["lengths"])
    if own:
        s["cache"] = _cache(case, s)
    return s


def _forks(case):
    """(parents, children): two children each, the last requests of the batch."""
    B, f = case["B"], case["forks"]
    return [i // 2 for i in range(f)], [B - f + i for i in range(f)]


def _prepare_pages(case, seed):
    g, (L, _) = _gen(seed), _lengths(case)
    src, dst = _forks(case)
    for b in dst:
        L[b] = 0
    need = case["B"] * (2 + case["N"] // case["page"])
    s = _pool(case, L, g, spare=need + case["forks"])
    width = -(-(case["L"] + case["N"]) // case["page"]) + 4
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device=DEV)
    table[:, :s["table"].shape[1]] = s["table"][:, :width]
    s["table"] = table
    s["lengths"], s["keep"] = _ints(L), _ints(L)
    s["src"], s["dst"] = _ints(src), _ints(dst)
    s["offsets"] = _ints([case["N"] * b for b in range(case["B"] + 1)])
    s["slots"] = torch.zeros(case["B"] * case["N"], dtype=torch.int32, device=DEV)
    s["fork_status"], s["status"] = torch.zeros_like(s["src"]), torch.zeros_like(s["lengths"])
    if own:
        s["cache"] = _cache(case, s)
    return s


# --------------------------------------------------------------------------
# One pass.
# --------------------------------------------------------------------------


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


def _own_qk(s):
    return {"q": s["call"](), "k": s["k"], "v": s["v"]}


def _own_attn(s):
    return s["call"]()


def _own_verify(s):
    tokens, path, n = s["call"]()
    return {"tokens": tokens, "path": path, "n": n}


def _own_compact(s):
    s["cache"].compact(s["path"], s["keep"], s["lengths"], s["new_lengths"])
    return {"k": s["k"], "v": s["v"], "lengths": s["new_lengths"]}


def _own_pages(s):
    c = s["cache"]
    c.fork(s["lengths"], s["src"], s["dst"], s["fork_status"])
    c.reserve(s["lengths"], s["offsets"], s["slots"], s["status"])
    c.trim(s["keep"])
    return _page_outputs(s)


def _page_outputs(s):
    return {n: s[n] for n in ("k", "v", "table", "held", "refs", "lengths", "slots", "fork_status",
                              "status")}


def _plain_qk(s):
    c = s["case"]
    Hq, Hkv, rot = c["Hq"], c["Hkv"], c["rot"]
    x = s["qkv"].float()
    cs = s["cos_sin"][s["positions"].long()][:, None, :]
    cos, sin = cs[..., :rot // 2], cs[..., rot // 2:]

    def head(v, w):
        v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * w.float()
        if c["pairs"] == "half":
            a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        else:
            a, b = v[..., 0:rot:2], v[..., 1:rot:2]
        y, z = a * cos - b * sin, b * cos + a * sin
        turned = torch.cat([y, z], -1) if c["pairs"] == "half" else torch.stack([y, z], -1).flatten(-2)
        return torch.cat([turned, v[..., rot:]], -1).to(s["qkv"].dtype)

    at = s["slots"].long()
    s["k"].view(-1, Hkv, c["D"])[at] = head(x[:, Hq:Hq + Hkv], s["kw"])
    s["v"].view(-1, Hkv, c["D"])[at] = s["qkv"][:, Hq + Hkv:]
    return {"q": head(x[:, :Hq], s["qw"]), "k": s["k"], "v": s["v"]}


def _rows_of(s, page, most):
    """Cache rows of the first ``most`` positions of every request."""
    at = torch.arange(most, device=DEV)
    of = s["table"].long()[:, (at // page).clamp(max=s["table"].shape[1] - 1)]
    return of.clamp(min=0) * page + at % page


def _plain_attn(s):
    c, off, L = s["case"], s["offsets"].long(), s["lengths"].long()
    B, N, Hq, Hkv, D = c["B"], c["N"], c["Hq"], c["Hkv"], c["D"]
    most = c["L"] + N
    rows = _rows_of(s, c["page"], most)
    K = s["k"].view(-1, Hkv, D)[rows].permute(0, 2, 3, 1).float().contiguous()  # [B, Hkv, D, most]
    V = s["v"].view(-1, Hkv, D)[rows].permute(0, 2, 1, 3).float().contiguous()
    node = torch.arange(N, device=DEV)
    row = (off[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)  # [B, N]
    q = s["q"][row].float().view(B, N, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    S = torch.matmul(q.reshape(B, Hkv, -1, D), K) / math.sqrt(D)
    at = torch.arange(most, device=DEV) - L[:, None]  # node that lies at a position
    bits = (s["mask"][:, 0][row][:, :, None] >> at.clamp(0, 63)[:, None, :]) & 1
    there = at < (off[1:] - off[:-1])[:, None]
    sees = (at < 0)[:, None, :] | ((bits == 1) & (at < 64)[:, None, :] & there[:, None, :])
    sees = sees[:, None, None].expand(B, 1, Hq // Hkv, N, most).reshape(B, 1, -1, most)
    S = S.masked_fill_(~sees, -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    O = torch.matmul(P, V) / P.sum(-1, keepdim=True)
    O = O.view(B, Hkv, Hq // Hkv, N, D).permute(0, 3, 1, 2, 4).reshape(B * N, Hq, D)
    T = s["q"].shape[0]
    b = torch.searchsorted(off, torch.arange(T, device=DEV), right=True) - 1
    return O[b * N + torch.arange(T, device=DEV) - off[b]].to(s["q"].dtype)


def _units(p):
    """Probabilities in units of 2**-36."""
    return (p.clamp(0, 1) * float(1 << 36)).long()


def _plain_verify(s):
    off, mask = s["offsets"].long(), s["mask"][:, 0]
    B, N, T, V = off.numel() - 1, s["case"]["N"], mask.numel(), s["p"].shape[1]
    node = torch.arange(N, device=DEV)
    there = node < (off[1:] - off[:-1])[:, None]  # [B, N]
    row = (off[:-1, None] + node).clamp(max=T - 1)
    up = torch.where(there, mask[row], 0)[:, :, None] >> node & 1  # up[b, j, i]: i is j or above it
    above = up.bool() & (node[None, :] < node[:, None])
    parent = torch.where(above, node, -1).amax(-1)  # [B, N]
    drafted = there & (parent >= 0)
    of = torch.gather(row, 1, parent.clamp(min=0))
    tok = s["tokens"][row].long()
    w = torch.where(drafted, _units(s["p"][of, tok]), 0)
    u = (s["u"][row] * (1 << 24)).long()
    older = (parent[:, :, None] == parent[:, None, :]) & (node[None, :] < node[:, None]) \
        & drafted[:, :, None] & drafted[:, None, :]  # older[b, j, i]: i comes before its sibling j
    if s["q"] is None:
        w = torch.where((older & (tok[:, :, None] == tok[:, None, :])).any(-1), 0, w)
        left = ((1 << 36) - (older * w[:, None, :]).sum(-1)).clamp(min=0)
        fits = drafted & (u * left < w << 24)
    else:
        fits = drafted & ~older.any(-1) & (u * _units(s["q"][of, tok]) < w << 24)
    good = fits & ~(older & fits[:, None, :]).any(-1)
    good = good | (there & (node == 0))
    stays = good & ~(up.bool() & ~good[:, None, :]).any(-1)
    depth = up.sum(-1)
    last = torch.argmax(torch.where(stays, depth, 0), 1)  # [B]
    n = torch.gather(torch.where(stays, depth, 0), 1, last[:, None])[:, 0]
    line = torch.gather(up, 1, last[:, None, None].expand(B, 1, N))[:, 0].bool()
    path = torch.sort(torch.where(line, node, N), 1).values
    here = torch.gather(row, 1, last[:, None])[:, 0]
    left = _units(s["p"][here])  # [B, V]
    kids = drafted & (parent == last[:, None])
    if s["q"] is None:
        out = torch.where(kids, tok, V)
        left = torch.cat([left, left[:, :1]], 1).scatter_(1, out, 0)[:, :V]
    else:
        left = torch.where(kids.any(1, keepdim=True),
                           (left - _units(s["q"][here])).clamp(min=0), left)
    to = ((s["u_next"] * (1 << 24)).long() * left.sum(1)) >> 24
    nxt = (left.cumsum(1) <= to[:, None]).sum(1)
    i = torch.arange(N, device=DEV)
    drawn = torch.gather(torch.cat([tok, tok[:, :1]], 1), 1, torch.roll(path, -1, 1))
    tokens = torch.where(i < (n - 1)[:, None], drawn, torch.where(i == (n - 1)[:, None], nxt[:, None], -1))
    return {"tokens": tokens.int(), "path": torch.where(path < N, path, -1).int(), "n": n.int()}


def _plain_compact(s):
    c = s["case"]
    i = torch.arange(c["N"], device=DEV)
    L = s["lengths"].long()[:, None]
    stays = i < s["keep"].long()[:, None]
    at = (L + torch.where(stays, s["path"].long(), i), L + i)
    table = s["table"].long()
    src, dst = ((torch.gather(table, 1, p // c["page"]) * c["page"] + p % c["page"]).view(-1) for p in at)
    for x in (s["k"], s["v"]):
        x = x.view(c["layers"], -1, c["Hkv"] * c["D"])
        x[:, dst] = x[:, src]
    torch.add(s["lengths"], s["keep"], out=s["new_lengths"])
    return {"k": s["k"], "v": s["v"], "lengths": s["new_lengths"]}


def _plain_pages(s):
    c = s["case"]
    page, table, refs, held, L = c["page"], s["table"], s["refs"], s["held"], s["lengths"]
    width = table.shape[1]
    col = torch.arange(width, device=DEV)

    def fresh(count):  # the lowest free pages, dealt out in order
        free = torch.argsort((refs > 0).int(), stable=True)
        start = torch.cumsum(count, 0) - count
        return free, start, start + count <= (refs == 0).sum()

    # fork
    src, dst = s["src"].long(), s["dst"].long()
    whole, part = L[src].long() // page, L[src].long() % page > 0
    free, start, fits = fresh(part.long())
    new = free[start.clamp(max=free.numel() - 1)]
    old = table[src].long()  # [f, width]
    rows = torch.where(col < whole[:, None], old, torch.where((col == whole[:, None]) & part[:, None],
                                                              new[:, None], -1))
    rows = torch.where(fits[:, None], rows, -1)
    refs.scatter_add_(0, rows.clamp(min=0).view(-1), (rows >= 0).int().view(-1))
    copied = part & fits
    last = torch.where(copied, torch.gather(old, 1, whole.clamp(max=width - 1)[:, None])[:, 0],
                       old[:, 0])  # a page of the parent's that stays as it is
    for x in (s["k"], s["v"]):  # only rows that are in use are copied
        used = copied[:, None] & (torch.arange(page, device=DEV) < (L[src].long() % page)[:, None])
        to = torch.where(copied, new, last)
        x[:, to] = torch.where(used[None, :, :, None, None], x[:, last], x[:, to])
    table[dst] = rows.int()
    held[dst] = (rows >= 0).sum(1).int()
    L[dst] = torch.where(fits, L[src], L[dst])
    s["fork_status"].copy_(fits)
    # reserve
    n = s["offsets"][1:] - s["offsets"][:-1]
    want = (L + n + page - 1) // page
    add = (want - held).clamp(min=0).long()
    free, start, fits = fresh(add)
    gets = (col >= held[:, None]) & (col < (held + add)[:, None]) & fits[:, None]
    at = (start[:, None] + col - held[:, None]).clamp(0, free.numel() - 1)
    table.copy_(torch.where(gets, free[at].int(), table))
    refs.scatter_add_(0, free[at].view(-1), gets.int().view(-1))
    held.add_(torch.where(fits, add, 0).int())
    s["status"].copy_(fits)
    r = torch.arange(s["slots"].numel(), device=DEV)
    b = torch.searchsorted(s["offsets"], r.int(), right=True) - 1
    p = L[b].long() + r - s["offsets"][b]
    s["slots"].copy_(torch.where(fits[b], table[b, p // page] * page + p % page, -1))
    # trim
    keep = (s["keep"] + page - 1) // page
    drop = (col >= keep[:, None]) & (col < held[:, None])
    refs.scatter_add_(0, table.long().clamp(min=0).view(-1), -drop.int().view(-1))
    table.masked_fill_(drop, -1)
    held.copy_(torch.minimum(held, keep))
    return _page_outputs(s)


# --------------------------------------------------------------------------
# What a pass cannot do without.
# --------------------------------------------------------------------------


def work(case):
    if case["op"] == "qk":
        n = case["T"] * (case["Hq"] + 2 * case["Hkv"]) * case["D"]
        return {"bytes": 4 * n + case["T"] * (4 * case["rot"] + 8) + 4 * case["D"], "flops": 10 * n}
    if case["op"] == "attn":
        L, N = _lengths(case)
        kv = sum(a + b for a, b in zip(L, N)) * case["Hkv"] * case["D"] * 4
        qo = sum(N) * case["Hq"] * case["D"] * 4
        flops = sum(4 * n * (a + 1) for a, n in zip(L, N)) * case["Hq"] * case["D"]
        return {"bytes": kv + qo + sum(-(-a // case["page"]) for a in L) * 4, "flops": flops}
    if case["op"] == "verify":
        rows = 2 if case["sampled"] else 1
        n = case["B"] * case["V"] * rows
        return {"bytes": 4 * n + 20 * case["B"] * case["N"], "flops": 2 * n}
    row = case["Hkv"] * case["D"] * 2 * 2 * case["layers"]  # K and V of one token, all layers
    if case["op"] == "compact":
        moved = sum(len(p) - 1 for p in _paths(case))
        return {"bytes": 2 * row * moved + 12 * case["B"], "flops": 0}
    L = _lengths(case)[0]
    part = sum(L[b] % case["page"] for b in _forks(case)[0])
    tables = sum(-(-(a + case["N"]) // case["page"]) for a in L)
    return {"bytes": 2 * row * part + 8 * tables + 8 * case["B"] * case["N"], "flops": 0}


# --------------------------------------------------------------------------
# The operators' definitions in 64 bits.
# --------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["op"]](case, s) if case["op"] in ("qk", "attn") else None


def _exact_qk(case, s):
    T, Hq, Hkv, rot = case["T"], case["Hq"], case["Hkv"], case["rot"]
    x = s["qkv"].double()
    rms = (x.square().sum(-1) / case["D"] + EPS).sqrt()[..., None]
    heads = torch.cat([s["qw"].double().expand(Hq, -1), s["kw"].double().expand(Hkv, -1)])
    y = x[:, :Hq + Hkv] / rms[:, :Hq + Hkv] * heads
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       torch.zeros((), dtype=torch.float64, device=DEV)).expand(T, 1, rot // 2).clone()
    table = s["cos_sin"].double()[s["positions"].long()]
    turn.real.copy_(table[:, None, :rot // 2])
    turn.imag.copy_(table[:, None, rot // 2:])
    if case["pairs"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    k, v = s["k"].double(), s["v"].double()
    at = s["slots"].long()
    k.view(-1, Hkv, case["D"])[at] = y[:, Hq:]
    v.view(-1, Hkv, case["D"])[at] = x[:, Hq + Hkv:]
    return {"q": y[:, :Hq].contiguous(), "k": k, "v": v}


def _exact_attn(case, s):
    L, N = _lengths(case)
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    masks, at = s["mask"][:, 0].tolist(), 0
    for b in range(case["B"]):
        n = L[b] + N[b]
        pages = s["table"][b, :-(-n // page)].long()
        ok = torch.ones((N[b], n), dtype=torch.bool)
        for j in range(N[b]):
            ok[j, L[b]:] = torch.tensor([bool(masks[at + j] >> i & 1) for i in range(N[b])])
        ok = ok.to(DEV)
        for h in range(Hkv):
            k = s["k"][0, pages, :, h].reshape(-1, D)[:n].double()
            v = s["v"][0, pages, :, h].reshape(-1, D)[:n].double()
            for i in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                e = (s["q"][at:at + N[b], i].double() @ k.t()) * D ** -0.5
                p = torch.softmax(e.masked_fill(~ok, -math.inf), -1)
                out[at:at + N[b], i] = p @ v
        at += N[b]
    return out

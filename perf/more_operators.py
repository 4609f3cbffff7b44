"""What is measured of the operators of a decode step whose requests go on from a
common prompt: few rows against much that is read.

A case is a dict of plain values; ``op`` names the operator:

* ``prefix``  attention of a batch whose groups of requests share the pages of a
              long prefix, each prefix read once for its whole group;
* ``few``     a whole mixture-of-experts layer (gate, routing table, experts,
              combine) for a few tokens, bf16 weights or 8-bit ones with a scale
              for each block of 128 x 128;
* ``sample``  the next tokens from logits and given random numbers, with
              temperature, top-k, top-p and min-p for each row, and the
              distribution that they were drawn from where it is wanted.

``own`` selects the framework's kernels; the plain form computes the same in
elementary torch operations. Sizes: the layers that ``synth.CONFIGS`` names (the
Mixtral-8x7B layer with its 32 query and 8 KV heads of 128; one expert-parallel
share of a DeepSeek-V3 layer) and generic ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
HEADS = dict(Hq=32, Hkv=8, D=128)
MIXTRAL = dict(d=4096, I=14336, E=8, k=2, n_local=8, shadows=1)
SHARE = dict(d=7168, I=2048, E=256, k=8, n_local=32, shadows=8)
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 128  # rows and columns of a weight block with one scale


def listed():
    return [
        # Four samples of one prompt of ordinary length: latency.
        dict(name="prefix_four", op="prefix", groups=1, B=4, N=1, P=1000, L=33, **HEADS,
             dtype="bf16", page=16),
        # A served batch behind one long system prompt.
        dict(name="prefix_batch", op="prefix", groups=1, B=128, N=1, P=8192, L=512, **HEADS,
             dtype="bf16", page=16),
        # Eight prompts of uneven popularity, small heads.
        dict(name="prefix_groups", op="prefix", groups=8, B=61, N=1, P=4099, L=700, Hq=24, Hkv=4,
             D=64, dtype="f16", page=32),
        # Drafted trees of requests that ask about one long document.
        dict(name="prefix_trees", op="prefix", groups=1, B=16, N=12, P=30000, L=300, **HEADS,
             dtype="bf16", page=64),
        # One token at one expert-parallel share: latency.
        dict(name="few_one", op="few", T=1, **SHARE, gate="logits", weights="f8"),
        # A small decode batch at the same share.
        dict(name="few_share", op="few", T=16, **SHARE, gate="logits", weights="bf16"),
        # One token of a layer with few, large experts, gate included.
        dict(name="few_large", op="few", T=1, **MIXTRAL, gate="weights", weights="bf16"),
        # The most tokens, which touch every expert of that layer.
        dict(name="few_most", op="few", T=32, **MIXTRAL, gate="weights", weights="f8"),
        # One row over a 32000-token vocabulary with every filter: latency.
        dict(name="sample_one", op="sample", T=1, V=32000, dtype="f32", filters="all", probs=False),
        # A batch over a large vocabulary by temperature alone.
        dict(name="sample_plain", op="sample", T=128, V=128000, dtype="bf16", filters="none",
             probs=False),
        # The same batch with each request's own filters.
        dict(name="sample_mixed", op="sample", T=128, V=128000, dtype="f32", filters="mixed",
             probs=False),
        # Rows of drafted trees, whose distributions the verification reads.
        dict(name="sample_probs", op="sample", T=192, V=32003, dtype="f16", filters="nucleus",
             probs=True),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(("prefix", "few", "sample"))
    if op == "prefix":
        D, Hkv = rng.choice((64, 128, 128, 256)), rng.choice((1, 2, 4, 8))
        Hq = Hkv * rng.choice((1, 2, 3, 4, 6, 8))
        B, N = _log(rng, 2, 128), rng.choice((1, 1, 1, _log(rng, 2, 16)))
        groups = rng.choice((1, 1, _log(rng, 1, B)))
        row = B * Hkv * D  # a position of every request
        P = _log(rng, 100, max(200, min(32768, 560_000_000 // row,
                                        2_000_000_000 // (B * N * Hq * D // 4))))
        return dict(op=op, groups=groups, B=B, N=N, P=P, L=_log(rng, 16, 700), Hq=Hq, Hkv=Hkv, D=D,
                    dtype=rng.choice(("bf16", "bf16", "f16")), page=rng.choice((8, 16, 32, 64, 128)))
    if op == "few":
        weights = rng.choice(("bf16", "f8"))
        step = 64 if weights == "bf16" else BLOCK
        d, I = (step * _log(rng, 512 // step, 7168 // step) for _ in range(2))
        n_local = rng.choice((4, 8, 16, 32))
        n_local = max(1, min(n_local, 1_600_000_000 // (3 * d * I) - 2))
        E = n_local * rng.choice((1, 1, 2, 8))
        return dict(op=op, T=_log(rng, 1, 32), d=d, I=I, E=E, k=min(E, rng.choice((1, 2, 4, 6, 8))),
                    n_local=n_local, shadows=rng.randint(0, 2), gate=rng.choice(("logits", "weights")),
                    weights=weights)
    V = _log(rng, 1000, 160000)
    return dict(op=op, T=_log(rng, 1, min(192, 16_000_000 // V)), V=V,
                dtype=rng.choice(("f32", "bf16", "f16")),
                filters=rng.choice(("none", "all", "nucleus", "mixed")), probs=rng.random() < 0.4)


# --------------------------------------------------------------------------
# What a program has in hand before the call.
# --------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) + 171)
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
    """What decides a case's work goes by the case, not by the seed."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _offsets(n):
    off = [0]
    for x in n:
        off.append(off[-1] + x)
    return off


def _requests(case):
    """(requests of each group, prefix of each group, cached tokens behind the
    prefix and rows of each request): the first of each is the largest, the
    others are ragged."""
    r, B, G = _shape_rng(case), case["B"], case["groups"]
    cuts = sorted(r.sample(range(1, B), G - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [B])]
    prefixes = [case["P"]] + [max(1, int(case["P"] * r.uniform(0.2, 1.0))) for _ in range(G - 1)]
    tails = [case["L"]] + [int(case["L"] * r.uniform(0.0, 1.0)) for _ in range(B - 1)]
    rows = [case["N"]] + [max(1, int(case["N"] * r.uniform(0.3, 1.0))) for _ in range(B - 1)]
    return sizes, prefixes, tails, rows


def _shared(case, prefix):
    """Tokens in whole pages: those are what forked requests share."""
    return prefix // case["page"] * case["page"]


def _trees(N, rng):
    """Ancestor bits of each node (its own among them), parents before children."""
    masks = []
    for n in N:
        m = [1]
        for j in range(1, n):
            m.append(m[rng.randrange(max(0, j - 6), j)] | 1 << j)
        masks += m
    return torch.tensor(masks, dtype=torch.int64, device=DEV)[:, None].contiguous()


def prepare(case, seed):
    s = globals()["_prepare_" + case["op"]](case, int(seed))
    s["case"] = case
    return s


def _prepare_prefix(case, seed):
    g, page = _gen(seed), case["page"]
    sizes, prefixes, tails, rows = _requests(case)
    shared = [_shared(case, p) for p in prefixes]
    of = [i for i, n in enumerate(sizes) for _ in range(n)]  # each request's group
    lengths = [prefixes[i] + t for i, t in zip(of, tails)]
    mine = [-(-(n + r) // page) - shared[i] // page for n, r, i in zip(lengths, rows, of)]
    n_pages = sum(s // page for s in shared) + sum(mine)
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["B"], max(s // page for s in shared) + max(mine) + 2), -1,
                       dtype=torch.int32, device=DEV)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    at, b = 0, 0
    for i, n in enumerate(sizes):
        common = order[at:at + shared[i] // page]
        at += len(common)
        refs[common.long()] = n
        for _ in range(n):
            pages = torch.cat([common, order[at:at + mine[b]]])
            refs[order[at:at + mine[b]].long()] = 1
            table[b, :len(pages)] = pages
            at, b = at + mine[b], b + 1
    dims, dtype = (1, n_pages, page, case["Hkv"], case["D"]), DTYPES[case["dtype"]]
    s = dict(k=_normal(dims, dtype, g), v=_normal(dims, dtype, g), table=table, refs=refs,
             held=_ints([shared[i] // page + m for i, m in zip(of, mine)]),
             q=_normal((sum(rows), case["Hq"], case["D"]), dtype, g),
             offsets=_ints(_offsets(rows)), lengths=_ints(lengths),
             group_offsets=_ints(_offsets(sizes)), shared=_ints(shared),
             mask=_trees(rows, random.Random(seed)) if case["N"] > 1 else None)
    if own:
        from paper_2601_01310_amd import spec
        cache = spec.KvCache(s["k"], s["v"], s["table"], s["held"], s["refs"])
        s["call"] = spec.PrefixAttention(cache, s["q"], s["offsets"], s["lengths"],
                                         s["group_offsets"], s["shared"], s["mask"],
                                         max_nodes=case["N"])
    return s


def _picks(case):
    """The experts of each token, the likeliest first: by the case, since they
    decide which weights are read. One of the first token's is served here."""
    r = _shape_rng(case)
    picks = [r.sample(range(case["E"]), case["k"]) for _ in range(case["T"])]
    if all(e >= case["n_local"] for e in picks[0]):
        picks[0][-1] = r.randrange(case["n_local"])
    return picks


def _prepare_few(case, seed):
    g, T, d, I, E, k = _gen(seed), case["T"], case["d"], case["I"], case["E"], case["k"]
    n, S = case["n_local"], case["n_local"] + case["shadows"]
    s = dict(x=_normal((T, d), torch.bfloat16, g), w_gate=None, logits=None)
    picks = torch.tensor(_picks(case), device=DEV)
    lift = (4.0 + 3.0 * torch.rand((T, k), generator=g, device=DEV)).sort(1, descending=True).values
    if case["gate"] == "weights":  # rows that lean towards their experts' gate rows
        s["w_gate"] = _normal((E, d), torch.bfloat16, g, 0.02)
        rows = s["w_gate"].float()
        lean = torch.zeros((T, E), device=DEV).scatter_(1, picks, lift * 2.0 + 2.0)
        s["x"] = (s["x"].float() + lean @ (rows / rows.square().sum(1, keepdim=True))).to(torch.bfloat16)
    else:
        s["logits"] = torch.rand((T, E), generator=g, device=DEV).scatter_(1, picks, lift)
    w13, w2 = _normal((S, 2 * I, d), torch.bfloat16, g, 0.02), _normal((S, d, I), torch.bfloat16, g, 0.02)
    table = torch.full((E, 2), -1, dtype=torch.int32)
    table[:n, 0] = torch.arange(n, dtype=torch.int32)
    alive = torch.ones(S, dtype=torch.uint8)
    for j in range(case["shadows"]):  # copies of some experts; the first one's primary has failed
        e = j * n // max(1, case["shadows"]) % n
        w13[n + j], w2[n + j], table[e, 1] = w13[e], w2[e], n + j
        alive[e] = 1 if j else 0
    s["table"], s["alive"] = table.to(DEV), alive.to(DEV)
    s["w13"], s["w2"], s["s13"], s["s2"] = w13, w2, None, None
    if case["weights"] == "f8":
        s["w13"], s["s13"] = _blocks(w13)
        s["w2"], s["s2"] = _blocks(w2)
    if own:
        from paper_2601_01310_amd import tg
        s["call"] = tg.EwFew(s["x"], s["w_gate"], s["logits"], s["table"], s["alive"], s["w13"],
                             s["w2"], k, w13_scale=s["s13"], w2_scale=s["s2"])
    return s


def _blocks(w):
    """8-bit values and one scale for each block of 128 x 128: its largest value
    becomes the type's, 448."""
    values = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=DEV)
    S, rows, cols = w.shape
    scale = torch.empty((S, rows // BLOCK, cols // BLOCK), device=DEV)
    for i in range(S):
        x = w[i].float().view(rows // BLOCK, BLOCK, cols // BLOCK, BLOCK)
        scale[i] = x.abs().amax((1, 3)) / 448.0
        values[i] = (x / scale[i][:, None, :, None]).view(rows, cols).to(torch.float8_e4m3fn)
    return values, scale


def _prepare_sample(case, seed):
    g, T, V = _gen(seed), case["T"], case["V"]
    logits = torch.randn((T, V), generator=g, device=DEV).mul_(2.5)
    # A few tokens stand out, as a trained model's do.
    at = torch.randint(0, V, (T, 8), generator=g, device=DEV)
    logits.scatter_(1, at, 8.0 + 4.0 * torch.rand((T, 8), generator=g, device=DEV))
    s = dict(logits=logits.to(DTYPES[case["dtype"]]), u=torch.rand(T, generator=g, device=DEV),
             temperature=0.6 + 0.7 * torch.rand(T, generator=g, device=DEV),
             top_k=None, top_p=None, min_p=None)
    f = case["filters"]
    if f in ("all", "mixed"):
        s["top_k"] = torch.randint(20, 200, (T,), generator=g, device=DEV).int()
        s["min_p"] = 0.02 + 0.08 * torch.rand(T, generator=g, device=DEV)
    if f != "none":
        s["top_p"] = 0.85 + 0.14 * torch.rand(T, generator=g, device=DEV)
    if f == "mixed":  # each request has its own: greedy, some of the filters, or none
        kind = torch.randint(0, 5, (T,), generator=g, device=DEV)
        s["temperature"][kind == 0] = 0.0
        s["top_k"][kind >= 2] = 0
        s["top_p"][kind == 1] = 1.0
        s["top_p"][kind == 4] = 1.0
        s["min_p"][kind != 3] = 0.0
    if own:
        from paper_2601_01310_amd import spec
        s["call"] = spec.SampleTokens(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"],
                                      s["min_p"], probs=case["probs"])
    return s


# --------------------------------------------------------------------------
# One pass.
# --------------------------------------------------------------------------


def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state)


def _own_prefix(s):
    return s["call"]()


def _own_few(s):
    c = s["call"]
    return {"out": c(), "ids": c.topk_ids, "weights": c.topk_w, "slots": c.pair_slot}


def _own_sample(s):
    if s["case"]["probs"]:
        tokens, probs = s["call"]()
        return {"tokens": tokens, "probs": probs}
    return {"tokens": s["call"]()}


def _plain_prefix(s):
    c, off, L = s["case"], s["offsets"].long(), s["lengths"].long()
    B, N, Hq, Hkv, D, page = c["B"], c["N"], c["Hq"], c["Hkv"], c["D"], c["page"]
    most = c["P"] + c["L"] + N
    at = torch.arange(most, device=DEV)
    of = s["table"].long()[:, (at // page).clamp(max=s["table"].shape[1] - 1)]
    rows = of.clamp(min=0) * page + at % page
    K = s["k"].view(-1, Hkv, D)[rows].permute(0, 2, 3, 1).float().contiguous()  # [B, Hkv, D, most]
    V = s["v"].view(-1, Hkv, D)[rows].permute(0, 2, 1, 3).float().contiguous()
    node = torch.arange(N, device=DEV)
    row = (off[:-1, None] + node).clamp(max=s["q"].shape[0] - 1)  # [B, N]
    q = s["q"][row].float().view(B, N, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4)
    S = torch.matmul(q.reshape(B, Hkv, -1, D), K) / math.sqrt(D)
    own_node = at - L[:, None]  # node that lies at a position
    there = own_node < (off[1:] - off[:-1])[:, None]
    if s["mask"] is None:
        sees = own_node[:, None, :] <= node[:, None]
    else:
        bits = (s["mask"][:, 0][row][:, :, None] >> own_node.clamp(0, 63)[:, None, :]) & 1
        sees = (own_node < 0)[:, None, :] | ((bits == 1) & (own_node < 64)[:, None, :])
    sees = (sees & there[:, None, :])[:, None, None].expand(B, 1, Hq // Hkv, N, most)
    S = S.masked_fill_(~sees.reshape(B, 1, -1, most), -math.inf)
    P = torch.exp(S - S.amax(-1, keepdim=True))
    O = torch.matmul(P, V) / P.sum(-1, keepdim=True)
    O = O.view(B, Hkv, Hq // Hkv, N, D).permute(0, 3, 1, 2, 4).reshape(B * N, Hq, D)
    r = torch.arange(s["q"].shape[0], device=DEV)
    b = torch.searchsorted(off, r, right=True) - 1
    return O[b * N + r - off[b]].to(s["q"].dtype)


def _weights32(w, scale):
    if scale is None:
        return w.float()
    S, rows, cols = w.shape
    w = w.float().view(S, rows // BLOCK, BLOCK, cols // BLOCK, BLOCK)
    return w.mul_(scale[:, :, None, :, None]).view(S, rows, cols)


def _plain_few(s):
    c, x = s["case"], s["x"]
    k, I = c["k"], c["I"]
    logits = s["logits"] if s["w_gate"] is None else torch.mm(
        x.double(), s["w_gate"].double().t()).float()
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    e = torch.exp(top - top[:, :1])
    weights = e / e.sum(1, keepdim=True)
    cand = s["table"].long()[ids]  # [T, k, R]
    ok = (cand >= 0) & (s["alive"][cand.clamp(min=0)] > 0)
    first = ok.int().argmax(-1, keepdim=True)
    slots = torch.where(ok.any(-1), torch.gather(cand, 2, first)[..., 0], -1)
    # Every expert over every token; a token's own are picked at the end.
    gu = torch.matmul(x.float(), _weights32(s["w13"], s["s13"]).transpose(1, 2))  # [S, T, 2I]
    h = gu[..., :I] * torch.sigmoid(gu[..., :I]) * gu[..., I:]
    y = torch.matmul(h, _weights32(s["w2"], s["s2"]).transpose(1, 2))  # [S, T, d]
    mine = y[slots.clamp(min=0), torch.arange(c["T"], device=DEV)[:, None]]  # [T, k, d]
    out = (torch.where(slots >= 0, weights, 0.0)[..., None] * mine).sum(1)
    return {"out": out.to(x.dtype), "ids": ids.int(), "weights": weights, "slots": slots.int()}


def _plain_sample(s):
    l, T, V = s["logits"].double(), s["case"]["T"], s["case"]["V"]
    hot = s["temperature"].double()[:, None]
    greedy = ~(hot > 0)
    w = torch.exp((l - l.amax(1, keepdim=True)) / torch.where(greedy, 1.0, hot))
    w = torch.where(w < 2.0 ** -64, 0.0, w)
    order = torch.sort(l, dim=1, descending=True, stable=True).indices
    ranked = torch.gather(w, 1, order)
    rank = torch.arange(V, device=DEV)
    most = torch.full((T, 1), V, device=DEV)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        most = torch.where(k > 0, k, most)
    keep = rank < torch.where(greedy, 1, most)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        left = ranked * keep
        before = left.cumsum(1) - left
        keep &= (before < p * left.sum(1, keepdim=True)) | (rank == 0) | (p >= 1)
    if s["min_p"] is not None:
        keep &= (ranked >= s["min_p"].double()[:, None]) | (rank == 0)
    left = torch.zeros_like(w).scatter_(1, order, ranked * keep)
    mass = left.sum(1, keepdim=True)
    tokens = (left.cumsum(1) <= s["u"].double()[:, None] * mass).sum(1).int()
    if not s["case"]["probs"]:
        return {"tokens": tokens}
    return {"tokens": tokens, "probs": (left / mass).float()}


# --------------------------------------------------------------------------
# What a pass cannot do without.
# --------------------------------------------------------------------------


def work(case):
    if case["op"] == "prefix":
        sizes, prefixes, tails, rows = _requests(case)
        of = [i for i, n in enumerate(sizes) for _ in range(n)]
        once = sum(_shared(case, p) for p in prefixes)
        rest = sum(prefixes[i] - _shared(case, prefixes[i]) + t + r
                   for i, t, r in zip(of, tails, rows))
        pages = sum(-(-(prefixes[i] + t + r) // case["page"]) for i, t, r in zip(of, tails, rows))
        flops = sum(4 * r * (prefixes[i] + t + 1) for i, t, r in zip(of, tails, rows))
        return {"bytes": (once + rest) * case["Hkv"] * case["D"] * 4 + 4 * pages +
                sum(rows) * case["Hq"] * case["D"] * 4, "flops": flops * case["Hq"] * case["D"]}
    if case["op"] == "few":
        T, d, I = case["T"], case["d"], case["I"]
        used = [e for p in _picks(case) for e in p if e < case["n_local"]]
        values = 3 * d * I * len(set(used))
        size = 2 * values if case["weights"] == "bf16" else values + values // BLOCK ** 2 * 4
        gate = 2 * case["E"] * d if case["gate"] == "weights" else 4 * T * case["E"]
        flops = 6 * d * I * len(used) + (2 * T * d * case["E"] if case["gate"] == "weights" else 0)
        return {"bytes": size + gate + 4 * T * d + 12 * T * case["k"], "flops": flops}
    n = case["T"] * case["V"]
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": n * (size + (4 if case["probs"] else 0)) + 24 * case["T"], "flops": 20 * n}


# --------------------------------------------------------------------------
# The operators' definitions in 64 bits.
# --------------------------------------------------------------------------


def exact(case, seed):
    if case["op"] == "sample" and not case["probs"]:
        return None  # whole numbers alone
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _exact_prefix(case, s):
    sizes, prefixes, tails, rows = _requests(case)
    of = [i for i, n in enumerate(sizes) for _ in range(n)]
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    masks = [1] * sum(rows) if s["mask"] is None else s["mask"][:, 0].tolist()
    at = 0
    for b in range(case["B"]):
        L, n = prefixes[of[b]] + tails[b], rows[b]
        pages = s["table"][b, :-(-(L + n) // page)].long()
        ok = torch.ones((n, L + n), dtype=torch.bool)
        for j in range(n):
            ok[j, L:] = torch.tensor([bool(masks[at + j] >> i & 1) for i in range(n)])
        ok = ok.to(DEV).repeat(Hq // Hkv, 1)
        for h in range(Hkv):
            k = s["k"][0, pages, :, h].reshape(-1, D)[:L + n].double()
            v = s["v"][0, pages, :, h].reshape(-1, D)[:L + n].double()
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            q = s["q"][at:at + n, heads].double().transpose(0, 1).reshape(-1, D)
            p = torch.softmax((q @ k.t() * D ** -0.5).masked_fill(~ok, -math.inf), -1)
            out[at:at + n, heads] = (p @ v).view(-1, n, D).transpose(0, 1)
        at += n
    return out


def _exact_few(case, s):
    T, d, I = case["T"], case["d"], case["I"]
    out = torch.zeros((T, d), dtype=torch.float64, device=DEV)
    weights = torch.zeros((T, case["k"]), dtype=torch.float64, device=DEV)
    table, alive = s["table"].tolist(), s["alive"].tolist()

    def whole(w, scale, slot):
        w = w[slot].double()
        if scale is not None:
            w = w * scale[slot].double().repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)
        return w

    by_slot = {}
    for t, picks in enumerate(_picks(case)):
        row = s["x"][t].double()
        l = torch.stack([row @ s["w_gate"][e].double() if s["logits"] is None
                         else s["logits"][t, e].double() for e in picks])
        order = sorted(range(len(picks)), key=lambda j: (-float(l[j]), picks[j]))
        weights[t] = torch.softmax(l[torch.tensor(order, device=DEV)], 0)
        for j, i in enumerate(order):
            slot = next((c for c in table[picks[i]] if c >= 0 and alive[c]), None)
            if slot is not None:
                by_slot.setdefault(slot, []).append((t, j))
    for slot, pairs in by_slot.items():
        t = torch.tensor([p[0] for p in pairs], device=DEV)
        x = s["x"][t].double()
        w13 = whole(s["w13"], s["s13"], slot)
        g, u = x @ w13[:I].t(), x @ w13[I:].t()
        y = (g / (1 + torch.exp(-g)) * u) @ whole(s["w2"], s["s2"], slot).t()
        for row, (i, j) in zip(y, pairs):
            out[i] += weights[i, j] * row
    return {"out": out, "ids": None, "weights": weights, "slots": None}


def _exact_sample(case, s):
    probs = torch.zeros((case["T"], case["V"]), dtype=torch.float64, device=DEV)
    for t in range(case["T"]):
        l, hot = s["logits"][t].double(), float(s["temperature"][t])
        kept, at = torch.sort(l, dim=0, descending=True, stable=True)
        k = int(s["top_k"][t]) if s["top_k"] is not None else 0
        if not hot > 0:
            k, hot = 1, 1.0
        if k > 0:
            kept, at = kept[:k], at[:k]
        p = torch.softmax(kept / hot, 0)
        if s["top_p"] is not None and float(s["top_p"][t]) < 1:
            n = 1 + int((torch.cumsum(p, 0)[:-1] < float(s["top_p"][t])).sum())
            p, at = p[:n], at[:n]
        if s["min_p"] is not None:
            n = max(1, int((p >= float(s["min_p"][t]) * p[0]).sum()))
            p, at = p[:n], at[:n]
        probs[t, at] = p / p.sum()
    return {"tokens": None, "probs": probs}

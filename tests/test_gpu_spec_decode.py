"""The paged-cache operators against the float64 oracle, through the binding.

Tolerances, from the number formats (u = half a unit in the last place of a
value, relative to it: 2^-8 for bf16, 2^-11 for f16):

* norms and rotation: float32 throughout and one rounding: u |ref| plus
  float32 errors of a dozen operations on terms of the size of the pair,
  2^-20 (|a| + |b|), plus f16's subnormal step 2^-25;
* attention: probabilities are rounded to the type before their product with
  v (float32 sums), and the output once: u * sum(p |v|) + u |ref|, with 1/16
  more of the first for the float32 errors of scores (|s| below 64: less than
  2^-14 relative) and of exp, plus 2^-25;
* everything of whole numbers: equal.
"""
import math

import numpy as np
import pytest
import torch

from oracle import spec_decode as S
from paper_2601_01310_amd import spec, tg

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def say(what):
    print(f"[gpu] {what}", flush=True)


def random_masks(sizes, rng, words=None):
    """Trees with parents before children: int64 [T, words]."""
    words = words or max(1, -(-max(list(sizes) + [1]) // 64))
    rows = []
    for n in sizes:
        m = []
        for j in range(n):
            m.append((m[rng.integers(max(0, j - 5), j)] if j else 0) | 1 << j)
        rows += [[x >> 64 * w & (2 ** 64 - 1) for w in range(words)] for x in m]
    a = np.array(rows, np.uint64).reshape(-1, words)
    return torch.from_numpy(a.view(np.int64)).to(DEV)


def make_pool(tokens, page, Hkv, D, dtype, rng, layers=1, fill=float("nan"), together=False,
              spare=2, extra=3):
    """Pages in no order; rows that no request owns hold ``fill``. Returns the
    cache and its page table (host)."""
    held = [-(-t // page) for t in tokens]
    n = sum(held) + spare
    order = rng.permutation(n)
    table = np.full((len(tokens), max(held + [1]) + extra), -1, np.int32)
    refs, at = np.zeros(n, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        at += h
    refs[order[:at]] = 1
    both = torch.full((layers, n, 2, page, Hkv, D), fill, dtype=dtype, device=DEV)
    if together:
        k, v = both[:, :, 0], both[:, :, 1]
    else:
        k, v = both[:, :, 0].contiguous(), both[:, :, 1].contiguous()
    for b, t in enumerate(tokens):
        for p in range(t):
            for x in (k, v):
                x[:, table[b, p // page], p % page] = torch.from_numpy(
                    rng.normal(size=(layers, Hkv, D)).astype(np.float32)).to(DEV).to(dtype)
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints(held),
                         torch.from_numpy(refs).to(DEV))
    return cache, table


# --------------------------------------------------------------------------
# Norms and rotation
# --------------------------------------------------------------------------

QK = [
    # T, Hq, Hkv, D, rot, interleaved, weights, dtype, page
    (1, 32, 8, 128, 128, False, True, torch.bfloat16, 16),
    (1, 1, 1, 64, 64, True, True, torch.float16, 1),
    (5, 6, 2, 64, 32, True, True, torch.float16, 8),
    (37, 3, 3, 128, 96, False, True, torch.bfloat16, 32),
    (7, 4, 1, 256, 256, False, True, torch.bfloat16, 4),
    (9, 4, 4, 256, 16, True, False, torch.float16, 4),
    (3, 5, 1, 64, 0, False, True, torch.bfloat16, 2),
    (1029, 7, 1, 64, 48, False, False, torch.bfloat16, 16),
    (1025, 2, 2, 128, 128, True, True, torch.bfloat16, 64),
]


@pytest.mark.parametrize("T,Hq,Hkv,D,rot,inter,weights,dtype,page", QK)
def test_qk_norm_rope(T, Hq, Hkv, D, rot, inter, weights, dtype, page):
    say(f"qk T={T} Hq={Hq} Hkv={Hkv} D={D} rot={rot} {dtype}")
    rng = np.random.default_rng(T + D + rot)
    cache, _ = make_pool([T], page, Hkv, D, dtype, rng, layers=2, fill=7.0)
    n_slots = cache.args.n_pages * page
    slots = rng.permutation(n_slots)[:T].astype(np.int32)
    if T > 2:
        slots[1], slots[2] = -1, n_slots + 5  # not cached
    wide = torch.randn((T, Hq + 2 * Hkv + 1, D), device=DEV).to(dtype)  # strided rows
    qkv = wide[:, :Hq + 2 * Hkv]
    places = 50
    pos = rng.integers(-2, places + 2, T).astype(np.int32)  # clamped
    angle = np.arange(places)[:, None] * 50.0 ** (-np.arange(max(rot // 2, 1)) / max(rot // 2, 1))
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    w = [(1 + 0.2 * torch.randn(D, device=DEV)).to(dtype) if weights else None for _ in range(2)]
    before_k, before_v = cache.k.clone(), cache.v.clone()
    call = spec.QkNormRope(cache, qkv, Hq, torch.from_numpy(pos).to(DEV),
                           torch.from_numpy(slots).to(DEV),
                           torch.from_numpy(table).to(DEV) if rot else None, *w, eps=1e-5,
                           interleaved=inter)
    q = f64(call(layer=1))
    x, host_w = f64(qkv), [None if t is None else f64(t) for t in w]
    K, V = f64(cache.k), f64(cache.v)
    assert torch.equal(cache.k[0], before_k[0]) and torch.equal(cache.v[0], before_v[0])
    written = set()
    for t in range(T):
        row = table[min(max(pos[t], 0), places - 1)] if rot else []
        for h in range(Hq + Hkv):
            ref = S.norm_rope(x[t, h], host_w[int(h >= Hq)], row, 1e-5, inter)
            size = np.abs(S.norm_rope(x[t, h], host_w[int(h >= Hq)], [], 1e-5, inter)).max() * 2
            tol = U[dtype] * np.abs(ref) + 2.0 ** -20 * size + 2.0 ** -25
            if h < Hq:
                assert (np.abs(q[t, h] - ref) <= tol).all(), (t, h)
            elif 0 <= slots[t] < n_slots:
                at = K[1, slots[t] // page, slots[t] % page, h - Hq]
                assert (np.abs(at - ref) <= tol).all(), (t, h)
        if 0 <= slots[t] < n_slots:
            written.add(int(slots[t]))
            assert np.array_equal(V[1, slots[t] // page, slots[t] % page], x[t, Hq + Hkv:])
    rest = [s for s in range(n_slots) if s not in written]
    for now, was in ((cache.k, before_k), (cache.v, before_v)):
        assert torch.equal(now[1].flatten(0, 1)[rest], was[1].flatten(0, 1)[rest])


def test_qk_norm_rope_in_place_gives_the_same_bits():
    rng = np.random.default_rng(0)
    cache, _ = make_pool([6], 4, 2, 128, torch.bfloat16, rng)
    qkv = torch.randn((6, 8, 128), device=DEV).to(torch.bfloat16)
    t = torch.randn((8, 128), device=DEV)
    w = torch.randn(128, device=DEV).to(torch.bfloat16)
    pos, slots = ints([0, 1, 2, 3, 4, 7]), ints([0, 1, 2, 3, 4, 5])
    a = spec.QkNormRope(cache, qkv.clone(), 4, pos, slots, t, w, w)().clone()
    ka = cache.k.clone()
    spec.QkNormRope(cache, qkv, 4, pos, slots, t, w, w, q_out=qkv[:, :4])()
    assert torch.equal(qkv[:, :4], a)
    assert torch.equal(cache.k.view(torch.int16), ka.view(torch.int16))
    spec.QkNormRope(cache, qkv[:0], 4, pos[:0], slots[:0], t, w, w)()  # no rows: nothing


# --------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------

ATTN = [
    # [(committed, rows)], Hq, Hkv, D, dtype, page, mask, together
    ([(1, 1)], 1, 1, 64, torch.bfloat16, 1, "tree", False),
    ([(0, 1)], 4, 1, 128, torch.bfloat16, 16, "tree", False),
    ([(31, 1)], 32, 8, 128, torch.bfloat16, 16, "tree", False),
    ([(32, 1), (33, 1), (127, 1), (128, 1), (129, 1)], 8, 2, 128, torch.float16, 8, "chain", True),
    ([(300, 5), (0, 0), (1, 9), (257, 1), (64, 3)], 8, 2, 128, torch.bfloat16, 32, "tree", False),
    ([(77, 17), (0, 16), (130, 4)], 3, 3, 64, torch.float16, 4, "tree", True),
    ([(200, 33)], 16, 2, 128, torch.bfloat16, 64, "tree", False),
    ([(45, 64), (90, 12)], 12, 2, 64, torch.bfloat16, 16, "chain", False),
    ([(100, 70), (3, 100)], 4, 1, 128, torch.float16, 16, "tree", False),
    ([(513, 2), (40, 7)], 6, 1, 256, torch.bfloat16, 16, "tree", False),
    ([(90, 31)], 8, 1, 256, torch.float16, 128, "chain", True),
    ([(1500, 1)], 40, 1, 128, torch.bfloat16, 16, "tree", False),
    ([(700, 3)] * 9, 4, 4, 64, torch.bfloat16, 2, "tree", False),
    # Tiles shared by the waves, with an address per lane (tiny pages), and 33
    # to 64 rows of a KV head.
    ([(90, 31), (64, 1)], 8, 2, 128, torch.bfloat16, 2, "tree", True),
    ([(70, 12)], 8, 1, 256, torch.float16, 1, "tree", False),
    ([(129, 9), (0, 7)], 12, 2, 128, torch.bfloat16, 4, "chain", False),
    ([(65, 40)], 2, 1, 64, torch.bfloat16, 4, "tree", False),
    # More requests than a wave has lanes, some without rows.
    ([(i % 37, i % 3) for i in range(150)], 4, 2, 64, torch.bfloat16, 8, "tree", False),
    ([(i % 61, 1 + i % 9) for i in range(70)], 8, 1, 128, torch.float16, 16, "tree", False),
    # One context over many blocks.
    ([(9000, 2)], 4, 1, 128, torch.bfloat16, 16, "tree", False),
    ([(5000, 20)], 6, 1, 64, torch.bfloat16, 64, "tree", False),
]


def check_attention(out, q, cache, table, layer, offsets, lengths, mask, scale, dtype):
    host = None if mask is None else mask.cpu().numpy().view(np.uint64)
    k, v = f64(cache.k[layer]), f64(cache.v[layer])
    ref = S.tree_attention(q, k, v, table, offsets, lengths, host, scale)
    size = S.tree_attention(q, k, np.abs(v), table, offsets, lengths, host, scale)
    tol = U[dtype] * (size * (1 + 1 / 16) + np.abs(ref)) + 2.0 ** -25
    got = f64(out)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], tol[bad][:3])


@pytest.mark.parametrize("requests,Hq,Hkv,D,dtype,page,mask,together", ATTN)
def test_tree_attention(requests, Hq, Hkv, D, dtype, page, mask, together):
    say(f"attention {requests} Hq={Hq} Hkv={Hkv} D={D} {dtype} page={page} {mask}")
    rng = np.random.default_rng(len(requests) * 1000 + D + page)
    L, N = [r[0] for r in requests], [r[1] for r in requests]
    cache, table = make_pool([a + b for a, b in zip(L, N)], page, Hkv, D, dtype, rng, layers=2,
                             together=together)
    off = np.concatenate([[0], np.cumsum(N)]).astype(np.int32)
    T = int(off[-1])
    wide = torch.randn((T, Hq + 1, D), device=DEV).to(dtype)
    q, out = wide[:, 1:], torch.full((T, Hq + 2, D), 3.0, dtype=dtype, device=DEV)
    m = random_masks(N, rng) if mask == "tree" else None
    call = spec.TreeAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L), m,
                              out=out[:, :Hq], max_nodes=max(N))
    got = call(layer=1)
    check_attention(got, f64(q), cache, table, 1, off, L, m, 1 / math.sqrt(D), dtype)
    assert (out[:, Hq:] == 3.0).all()
    again = got.clone()
    call(layer=1)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16)), "two runs differ"


@pytest.mark.parametrize("Hq,D", [(2, 64), (8, 128), (40, 128), (2, 256), (16, 128), (40, 64),
                                  (16, 256)])
def test_rows_that_see_nothing_and_masked_nan(Hq, D):
    """Rows without a set bit and without context give zeros; nodes that a row
    does not see hold NaN and infinities and stay out of it."""
    say(f"attention, masked NaN, Hq={Hq} D={D}")
    rng = np.random.default_rng(5)
    n = 7
    for L in (0, 50):
        cache, table = make_pool([L + n], 16, 2, D, torch.bfloat16, rng)
        bits = [1, 0, 0b101, 0b1001, 0, 0b100001, 0b1]
        poison = {1: float("nan"), 4: float("inf"), 6: -float("inf")}  # seen by no row
        for j, x in poison.items():
            for c in (cache.k, cache.v):
                c[0, table[0, (L + j) // 16], (L + j) % 16] = x
        mask = torch.tensor([[x] for x in bits], device=DEV)
        q = torch.randn((n, Hq, D), device=DEV).to(torch.bfloat16)
        out = spec.TreeAttention(cache, q, ints([0, n]), ints([L]), mask)()
        assert torch.isfinite(out).all()
        check_attention(out, f64(q), cache, table, 0, [0, n], [L], mask, 1 / math.sqrt(D),
                        torch.bfloat16)
        if L == 0:
            assert (out[[1, 4]] == 0).all()
        # A node's own NaN or infinity reaches the rows that see it, and no other.
        j = 2
        cache.v[0, table[0, (L + j) // 16], (L + j) % 16] = float("inf")
        out = spec.TreeAttention(cache, q, ints([0, n]), ints([L]), mask)()
        assert not torch.isfinite(out[2]).any()
        assert torch.isfinite(out[[0, 1, 3, 4, 5, 6]]).all()


def test_attention_positions_without_a_page_are_not_there():
    rng = np.random.default_rng(6)
    cache, table = make_pool([100], 16, 1, 64, torch.float16, rng, extra=0, fill=0.5)
    table[0, 2], table[0, 4] = -1, cache.args.n_pages + 3
    cache.page_table.copy_(torch.from_numpy(table))
    q = torch.randn((3, 2, 64), device=DEV).half()
    for L in (97, 500):  # 500: past the table
        out = spec.TreeAttention(cache, q, ints([0, 3]), ints([L]))()
        check_attention(out, f64(q), cache, table, 0, [0, 3], [L], None, 0.125, torch.float16)


def test_attention_large_scores_and_scale():
    """Scores far beyond exp's range: the running maximum keeps them in it."""
    rng = np.random.default_rng(7)
    cache, table = make_pool([260], 16, 1, 64, torch.bfloat16, rng)
    cache.k.nan_to_num_().mul_(8)
    q = (torch.randn((4, 4, 64), device=DEV) * 8).to(torch.bfloat16)
    call = spec.TreeAttention(cache, q, ints([0, 4]), ints([256]), scale=1.0)
    got = f64(call())
    k, v = f64(cache.k[0]), f64(cache.v[0])
    ref = S.tree_attention(f64(q), k, v, table, [0, 4], [256], None, 1.0)
    # |s| up to 4096 in float32: 64 products of at most 2^10 each, added in
    # float32 (2^-24 * 64 * 4096 = 2^-6 at most): e^(2^-6) on each p.
    size = S.tree_attention(f64(q), k, np.abs(v), table, [0, 4], [256], None, 1.0)
    assert (np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -4) * size + 2.0 ** -8 * np.abs(ref)).all()


def test_attention_offsets_past_32_bits():
    """Pages more than 2^31 elements apart."""
    say("attention, pages 2.4e9 bytes apart")
    page, Hkv, D, stride = 16, 1, 64, 1_200_000_000
    pool = torch.empty(2 * stride + 4096, dtype=torch.bfloat16, device=DEV)
    k, v = (torch.as_strided(pool, (1, 3, page, Hkv, D), (0, stride, Hkv * D, D, 1), o)
            for o in (0, 2048))
    rng = np.random.default_rng(8)
    for x in (k, v):
        x.copy_(torch.randn((1, 3, page, Hkv, D), device=DEV))
    table = np.array([[2, 0, 1]], np.int32)
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints([3]), ints([1, 1, 1]))
    q = torch.randn((2, 3, D), device=DEV).to(torch.bfloat16)
    out = spec.TreeAttention(cache, q, ints([0, 2]), ints([45]))()
    check_attention(out, f64(q), cache, table, 0, [0, 2], [45], None, 0.125, torch.bfloat16)
    qkv = torch.randn((1, 5, D), device=DEV).to(torch.bfloat16)
    spec.QkNormRope(cache, qkv, 3, None, ints([2 * page + 5]))()
    assert torch.equal(k[0, 2, 5, 0], qkv[0, 3]) and torch.equal(v[0, 2, 5, 0], qkv[0, 4])


def test_attention_on_another_stream_and_in_a_graph():
    say("attention in a graph")
    rng = np.random.default_rng(9)
    cache, table = make_pool([1200 + 9, 30 + 2], 16, 2, 128, torch.bfloat16, rng)
    L, off = ints([1200, 30]), ints([0, 9, 11])
    q = torch.randn((11, 8, 128), device=DEV).to(torch.bfloat16)
    mask = random_masks([9, 2], rng)
    call = spec.TreeAttention(cache, q, off, L, mask)
    lengths = [[1200, 30], [5, 29], [700, 0], [1200, 30]]
    eager = []
    for x in lengths:
        L.copy_(ints(x))
        eager.append(call().clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    side.synchronize()
    assert torch.equal(got, eager[3])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="thread_local"):
        call()
    for x, ref in zip(lengths, eager):
        L.copy_(ints(x))
        call.out.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(call.out, ref)
        torch.randn(1000, device=DEV).sum().item()  # eager work between replays


# --------------------------------------------------------------------------
# Verification
# --------------------------------------------------------------------------

VERIFY = [
    # rows of each request, V, sampled, max_path
    ([1], 5, False, 1),
    ([4], 300, True, 4),
    ([8, 1, 0, 5], 32000, False, 8),
    ([6, 6, 2, 0, 6], 4099, True, 6),
    ([33, 64, 17], 1000, False, 4),
    ([130, 3], 257, False, 20),
    ([7] * 40, 70001, True, 7),
    ([5], 128000, True, 3),
    ([9] * 3, 128000, False, 9),
]


def verify_inputs(sizes, V, sampled, seed):
    rng = np.random.default_rng(seed)
    T = sum(sizes)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    logits = torch.randn((T, V), generator=g, device=DEV) * 3
    p = torch.softmax(logits, 1)
    q = torch.softmax(logits + torch.randn((T, V), generator=g, device=DEV) * 0.5, 1) if sampled \
        else None
    mask = None if sampled else random_masks(sizes, rng)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    tokens = rng.integers(0, V, T).astype(np.int32)
    top = torch.topk(p, min(4, V), 1).indices.cpu().numpy()
    for b in range(len(sizes)):  # mostly likely tokens after each node's parent
        for j in range(1, sizes[b]):
            up = j - 1 if mask is None else (
                S.mask_bits(mask[off[b] + j].cpu().numpy().view(np.uint64)) & ((1 << j) - 1)
            ).bit_length() - 1
            if rng.random() < 0.9:
                tokens[off[b] + j] = rng.choice(top[off[b] + up])
            if rng.random() < 0.05:
                tokens[off[b] + j] = rng.choice([-1, V, V + 9])
    u, un = rng.random(T).astype(np.float32), rng.random(len(sizes)).astype(np.float32)
    if T > 3:
        u[1], u[2], un[0] = 0.0, 1.0, 0.99999997
    return p, q, mask, off, tokens, u, un


@pytest.mark.parametrize("sizes,V,sampled,max_path", VERIFY)
def test_verify_tree(sizes, V, sampled, max_path):
    say(f"verify {sizes[:5]} V={V} sampled={sampled}")
    for seed in range(4):
        p, q, mask, off, tokens, u, un = verify_inputs(sizes, V, sampled, seed + V)
        if seed == 3:  # strided rows, unaligned
            wide = torch.zeros((p.shape[0], V + 3), device=DEV)
            wide[:, 1:V + 1] = p
            p = wide[:, 1:V + 1]
        call = spec.VerifyTree(p, *(torch.from_numpy(x).to(DEV) for x in (tokens, u, un, off)),
                               tree_mask=mask, max_path=max_path, draft_probs=q)
        got = [t.cpu().numpy() for t in call()]
        ref = S.verify(p.cpu().numpy(), None if q is None else q.cpu().numpy(), tokens, u, un, off,
                       None if mask is None else mask.cpu().numpy().view(np.uint64), max_path)
        for name, a, b in zip(("tokens", "path", "n"), got, ref):
            assert np.array_equal(a, b), (seed, name, a, b)


def _verify(p, tokens, u, un, q=None, mask=None):
    p = torch.tensor(p, dtype=torch.float32, device=DEV)
    T = p.shape[0]
    mask = None if mask is None else torch.tensor([[m] for m in mask], device=DEV)
    q = None if q is None else torch.tensor(q, dtype=torch.float32, device=DEV)
    call = spec.VerifyTree(p, ints(tokens), torch.tensor(u, device=DEV), torch.tensor([un], device=DEV),
                           ints([0, T]), tree_mask=mask, draft_probs=q)
    t, path, n = (x.cpu().tolist() for x in call())
    return path[0][:n[0]], t[0][:n[0]]


@pytest.mark.parametrize("V", [1000, 160000, 300001])
def test_rows_that_are_no_distributions_give_a_token_of_theirs(V):
    """Rows of ones and infinities: sums far beyond exact float64."""
    p = torch.ones((6, V), device=DEV)
    p[2:4] = float("inf")
    p[4:] = 1e30
    u = torch.tensor([0.0, 0.3, 0.5, 0.7, 0.999, 0.99999997], device=DEV)
    call = spec.VerifyTree(p, ints([V - 1] * 6), u, u, ints(range(7)), max_path=1)
    tokens, path, n = (t.cpu().numpy() for t in call())
    assert (n == 1).all() and (path == 0).all()
    assert ((tokens >= 0) & (tokens < V)).all()
    if V == 1000:
        assert tokens[:, 0].tolist() == (np.floor(u.cpu().double().numpy() * 2 ** 24) * V
                                         // 2 ** 24).astype(int).tolist()


def test_a_whole_step_in_a_graph():
    """Reserve, norms and rotation, attention (heads of 256), verification,
    compaction and trim, captured once and replayed on new inputs."""
    say("a step in a graph")
    B, n, Hq, Hkv, D, V = 3, 5, 4, 1, 256, 900
    T = B * n
    rng = np.random.default_rng(4)
    cache = spec.KvCache.empty(2, 40, 8, Hkv, D, B, 10, device=DEV)
    lengths, new, keep = ints([0] * B), ints([0] * B), ints([0] * B)
    off, slots, status = ints([0, n, 2 * n, T]), ints([0] * T), ints([0] * B)
    qkv = torch.zeros((T, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device=DEV)
    mask, tokens = random_masks([n] * B, rng), ints([0] * T)
    p, u, un = torch.zeros((T, V), device=DEV), torch.zeros(T, device=DEV), torch.zeros(B, device=DEV)
    rope = spec.QkNormRope(cache, qkv, Hq, None, slots)
    attend = spec.TreeAttention(cache, rope.q_out, off, lengths, mask)
    check = spec.VerifyTree(p, tokens, u, un, off, mask, max_path=n)

    def step():
        cache.reserve(lengths, off, slots, status)
        for layer in range(2):
            rope(layer=layer)
        attend(layer=1)
        tok, path, kept = check()
        cache.compact(path, kept, lengths, new)
        lengths.copy_(new)
        cache.trim(lengths)

    state = [cache.k, cache.v, cache.page_table, cache.held, cache.refcount, lengths, slots,
             attend.out, check.tokens_out, check.path, check.n_out]

    def inputs(seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        qkv.copy_(torch.randn(qkv.shape, generator=g, device=DEV))
        p.copy_(torch.softmax(torch.randn(p.shape, generator=g, device=DEV) * 3, 1))
        tokens.copy_(torch.topk(p, 1).indices[:, 0].roll(1))
        u.copy_(torch.rand(u.shape, generator=g, device=DEV))
        un.copy_(torch.rand(un.shape, generator=g, device=DEV))

    def reset():
        for t in (cache.k, cache.v, cache.held, cache.refcount, lengths):
            t.zero_()
        cache.page_table.fill_(-1)

    step()
    torch.cuda.synchronize()
    reset()
    eager = []
    for seed in range(5):
        inputs(seed)
        step()
        eager.append([t.clone() for t in state])
    reset()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, capture_error_mode="thread_local"):
        step()
    reset()
    for seed in range(5):
        inputs(seed)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(state, eager[seed]):
            assert torch.equal(a, b), seed
        torch.randn(1000, device=DEV).sum().item()
    assert int(lengths.min()) >= 5


def test_verify_edges():
    nan = float("nan")
    half = [0.5, 0.5, 0.0]
    # A draft equal to the target is always kept, one without mass never.
    assert _verify([half, [0, 0, 1.0]], [0, 1], [0.0, 0.999], 0.3, q=[half, half]) == ([0, 1], [1, 2])
    assert _verify([half, half], [0, 2], [0.0, 0.0], 0.75, q=[half, half])[0] == [0]
    # Refused with p == q elsewhere: nothing is left, p as it is.
    assert _verify([half, half], [0, 2], [0.0, 0.0], 0.75, q=[half, half])[1] == [1]
    # Every child refused and all mass with them: p as it is.
    assert _verify([half] * 3, [0, 0, 0], [0.0] * 3, 0.2, mask=[1, 3, 5])[1][0] == 0
    # No mass at all, NaN among it.
    assert _verify([[nan, 0.0, -1.0]], [0], [0.5], 0.5) == ([0], [0])
    assert _verify([[nan, 0.0, 1.0]], [0], [nan], nan) == ([0], [2])
    # Two children with one token: the second is not kept.
    assert _verify([[0.5, 0.5, 0.0]] * 3, [0, 1, 1], [0.0, 0.99, 0.0], 0.0, mask=[1, 3, 5]) == \
        ([0], [0])


# --------------------------------------------------------------------------
# Pages
# --------------------------------------------------------------------------


def state_of(cache):
    return [t.cpu().numpy() for t in (cache.page_table, cache.held, cache.refcount)]


@pytest.mark.parametrize("B,page,n_pages,width,seed", [
    (1, 16, 4, 4, 0), (5, 4, 60, 12, 1), (7, 1, 40, 20, 2), (64, 16, 9000, 40, 3),
    (3, 8, 20000, 16, 4), (1500, 2, 2500, 6, 5)])
def test_pages_follow_the_oracle(B, page, n_pages, width, seed):
    """Reserve, fork and trim in a seeded order, running out of pages and of
    table rows; tables, counts, slots and statuses equal after every call."""
    say(f"pages B={B} page={page} n={n_pages}")
    rng = np.random.default_rng(seed)
    cache = spec.KvCache.empty(2, n_pages, page, 1, 64, B, width, device=DEV)
    cache.k.copy_(torch.randn(cache.k.shape, device=DEV))
    cache.v.copy_(torch.randn(cache.k.shape, device=DEV))
    if n_pages > 8192:  # free pages far up
        cache.refcount[:n_pages - 700] = 1
    ref = S.Pages(*state_of(cache), page, [cache.k.float().cpu().numpy(),
                                           cache.v.float().cpu().numpy()])
    lengths = np.zeros(B, np.int32)
    dev_len = ints(lengths.tolist())
    for step in range(8):
        n = rng.integers(0, 3 * page + 2, B)
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        T = int(off[-1])
        slots, status = torch.full((T,), 77, dtype=torch.int32, device=DEV), ints([9] * B)
        cache.reserve(dev_len, torch.from_numpy(off).to(DEV), slots, status)
        r_slots, r_status = ref.reserve(lengths, off, T)
        assert np.array_equal(status.cpu().numpy(), r_status)
        assert np.array_equal(slots.cpu().numpy(), r_slots)
        lengths = (lengths + n * r_status).astype(np.int32)
        keep = np.where(rng.random(B) < 0.3, 0, np.maximum(0, lengths - rng.integers(0, 3, B)))
        if step % 3 == 2:
            keep = lengths.copy()
        cache.trim(ints(keep.tolist()))
        ref.trim(keep)
        lengths = keep.astype(np.int32)
        dev_len.copy_(torch.from_numpy(lengths))
        k = min(B, 12)
        src, dst = rng.integers(-1, B + 1, k).astype(np.int32), rng.integers(0, B, k).astype(np.int32)
        st = ints([9] * k)
        cache.fork(dev_len, torch.from_numpy(src).to(DEV), torch.from_numpy(dst).to(DEV), st)
        r_st = ref.fork(lengths, src.tolist(), dst.tolist())
        assert np.array_equal(st.cpu().numpy(), r_st), (src, dst)
        assert np.array_equal(dev_len.cpu().numpy(), lengths)
        for a, b in zip(state_of(cache), (ref.table, ref.held, ref.ref)):
            assert np.array_equal(a, b), step
    for t, c in zip((cache.k, cache.v), ref.caches):
        assert np.array_equal(t.float().cpu().numpy(), c)


@pytest.mark.parametrize("B,page,Hkv,D,layers,dtype,together", [
    (1, 16, 1, 64, 1, torch.bfloat16, False), (5, 4, 3, 128, 3, torch.float16, True),
    (9, 1, 2, 256, 2, torch.bfloat16, False), (3, 64, 8, 128, 5, torch.bfloat16, False)])
def test_compaction(B, page, Hkv, D, layers, dtype, together):
    say(f"compact B={B} page={page} layers={layers}")
    rng = np.random.default_rng(B + page)
    L, n = rng.integers(0, 40, B).tolist(), 30
    cache, table = make_pool([x + n for x in L], page, Hkv, D, dtype, rng, layers=layers, fill=2.0,
                             together=together)
    paths = [sorted(rng.choice(np.arange(1, n), rng.integers(0, n - 1), replace=False).tolist())
             for _ in range(B)]
    paths = [[0] + p for p in paths]
    path = np.array([p + [-1] * (n - len(p)) for p in paths], np.int32)
    keep = np.array([len(p) for p in paths], np.int32)
    keep[0] = min(keep[0], 1)  # nothing moves
    ref = S.Pages(table, cache.held.cpu().numpy(), cache.refcount.cpu().numpy(), page,
                  [cache.k.float().cpu().numpy(), cache.v.float().cpu().numpy()])
    r_new = ref.compact(path, keep, L)
    new = ints([-5] * B)
    cache.compact(torch.from_numpy(path).to(DEV), torch.from_numpy(keep).to(DEV), ints(L), new)
    assert np.array_equal(new.cpu().numpy(), r_new)
    for t, c in zip((cache.k, cache.v), ref.caches):
        assert np.array_equal(t.float().cpu().numpy(), c)


def test_compaction_skips_what_has_no_page():
    rng = np.random.default_rng(1)
    cache, table = make_pool([20], 4, 1, 64, torch.bfloat16, rng, fill=2.0)
    before = cache.k.clone()
    new = ints([0])
    path = ints([[0, 3, 900, 1 << 30, -4]])
    cache.compact(path, ints([5]), ints([17]), new)  # rows 20, 917, ...: no page
    assert torch.equal(cache.k, before) and int(new[0]) == 22
    cache.compact(path, ints([9]), ints([-3]), new)  # clamped: 5 rows from position 0
    assert int(new[0]) == 5
    assert torch.equal(cache.k[0, table[0, 0], 1], before[0, table[0, 0], 3])

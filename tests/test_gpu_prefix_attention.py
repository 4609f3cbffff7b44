"""tg_prefix_attention on the GPU against the float64 oracle, which knows nothing of
groups: it reads every request's own table. Tolerances: those of attention in
test_gpu_spec_decode (the parts are joined in float32: within its 1/16)."""
import math

import numpy as np
import pytest
import torch

from paper_2601_01310_amd import spec
from tests.test_gpu_spec_decode import DEV, U, check_attention, f64, ints, random_masks, say

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def room(B, Hkv, D, page):
    """Pages per request from which on a call of B requests reads shared pages once:
    tables that hold less are left to tree attention."""
    return -(-4096 * 8 * 128 // (max(1, B - 1) * Hkv * D * page))


def make(requests, groups, Hq, Hkv, D, dtype, page, seed, layers=2, mask=True, fill=float("nan"),
         wide=True):
    """requests [(committed tokens, rows)], groups [(first request, requests, shared
    positions)]; pages in no order, those of the shared positions held by all of the
    group, rows that nobody owns ``fill``; tables for ``room`` or (wide False) little
    more than the requests have."""
    rng = np.random.default_rng(seed)
    L, N = [r[0] for r in requests], [r[1] for r in requests]
    held = [-(-(a + b) // page) for a, b in requests]
    order = rng.permutation(sum(held) + 3)
    width = max(max(held + [1]) + 2, room(len(requests), Hkv, D, page) if wide else 0)
    table = np.full((len(requests), width), -1, np.int32)
    own, at = np.zeros(sum(held) + 3, np.int64), 0  # rows in use of a page
    for b, h in enumerate(held):
        table[b, :h] = order[at:at + h]
        for i in range(h):
            own[order[at + i]] = min(page, L[b] + N[b] - i * page)
        at += h
    for first, n, shared in groups:
        for b in range(first + 1, first + n):
            whole = min(shared // page, held[b])
            table[b, :whole] = table[first, :whole]
    k, v = ((torch.randn((layers, len(own), page, Hkv, D), device=DEV,
                         generator=torch.Generator(DEV).manual_seed(seed + i))).to(dtype) for i in (1, 2))
    gone = torch.arange(page, device=DEV)[None, :] >= torch.from_numpy(own).to(DEV)[:, None]
    for x in (k, v):
        x.masked_fill_(gone[None, :, :, None, None], fill)
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints(held),
                         torch.zeros(len(own), dtype=torch.int32, device=DEV))
    off = np.concatenate([[0], np.cumsum(N)]).astype(np.int32)
    q = torch.randn((int(off[-1]), Hq, D), device=DEV,
                    generator=torch.Generator(DEV).manual_seed(seed)).to(dtype)
    return cache, table, off, L, q, random_masks(N, rng) if mask else None


def tensors(groups):
    """group_offsets and shared of groups that lie one behind the other."""
    edges = [groups[0][0]] if groups else [0]
    for first, n, _ in groups:
        assert first == edges[-1]
        edges.append(first + n)
    return ints(edges), ints([g[2] for g in groups])


def run(x, groups, Hq, D, layer=1, **kw):
    cache, table, off, L, q, m = x
    call = spec.PrefixAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L), *tensors(groups), m,
                                **kw)
    call.out.fill_(3.0)
    got = call(layer=layer)
    check_attention(got, f64(q), cache, table, layer, off, L, m, 1 / math.sqrt(D), q.dtype)
    again = got.clone()
    call(layer=layer)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16)), "two runs differ"
    return call


CASES = [
    # requests, groups, Hq, Hkv, D, dtype, page, mask, max_nodes
    ([(200, 1), (201, 1)], [(0, 2, 192)], 1, 1, 64, BF, 16, False, 1),
    ([(128, 1)] * 3, [(0, 3, 128)], 4, 1, 128, BF, 16, False, 1),  # nothing of their own but the row
    ([(300, 1), (290, 1), (513, 1), (256, 1)], [(0, 4, 256)], 32, 8, 128, BF, 16, False, 1),
    ([(300, 2), (290, 7), (513, 1)], [(0, 3, 288)], 8, 2, 128, F16, 32, True, 7),
    # Several groups, some of one request, requests outside, too short prefixes.
    ([(40, 1), (400, 1), (400, 1), (50, 1), (50, 1), (600, 1), (700, 1), (640, 1), (9, 1)],
     [(1, 2, 384), (3, 2, 48), (5, 1, 600), (6, 2, 640)], 6, 2, 64, BF, 16, False, 1),
    # Requests without rows, the first of a group and a short one among them.
    ([(400, 0), (420, 3), (5, 0), (390, 1), (0, 0)], [(0, 5, 384)], 8, 2, 64, F16, 64, True, 3),
    # A length below what is said to be shared: less counts.
    ([(500, 1), (200, 1), (450, 1)], [(0, 3, 448)], 4, 2, 128, BF, 16, False, 1),
    ([(500, 1), (0, 1), (450, 1)], [(0, 3, 448)], 4, 2, 128, BF, 16, False, 1),
    # Trees: tails of the shared kernel, groups of many rows.
    ([(260, 33), (300, 12), (270, 20)], [(0, 3, 256)], 8, 1, 128, BF, 16, True, 33),
    ([(260, 20), (300, 9), (280, 14)], [(0, 3, 256)], 4, 1, 256, F16, 32, True, 20),
    ([(150, 2)] * 9, [(0, 4, 128), (4, 5, 144)], 2, 2, 256, BF, 8, True, 2),
    # Tiny and large pages.
    ([(333, 1), (340, 2), (350, 1)], [(0, 3, 332)], 8, 2, 64, BF, 4, True, 2),
    ([(333, 1), (340, 2), (350, 1)], [(0, 3, 330)], 8, 2, 128, F16, 2, True, 2),
    ([(300, 1), (280, 1)], [(0, 2, 280)], 4, 1, 64, BF, 1, False, 1),
    ([(1500, 1), (1400, 1), (1300, 1)], [(0, 3, 1024)], 4, 1, 128, BF, 512, False, 1),
    # Few rows in a long prefix, many rows of a group.
    ([(9000, 1), (9001, 1)], [(0, 2, 8990)], 4, 1, 128, BF, 16, False, 1),
    ([(520 + i % 7, 1) for i in range(70)], [(0, 70, 512)], 8, 2, 64, BF, 16, False, 1),
    ([(400 + i % 31, 1 + i % 3) for i in range(90)], [(0, 30, 400), (30, 1, 9), (31, 59, 390)], 6, 1,
     128, F16, 16, True, 3),
]


@pytest.mark.parametrize("requests,groups,Hq,Hkv,D,dtype,page,mask,nodes", CASES)
def test_against_float64(requests, groups, Hq, Hkv, D, dtype, page, mask, nodes):
    say(f"prefix {requests[:4]} {groups} Hq={Hq} Hkv={Hkv} D={D} page={page}")
    x = make(requests, groups, Hq, Hkv, D, dtype, page, len(requests) + D + page, mask=mask)
    run(x, groups, Hq, D, max_nodes=nodes)
    run(x, groups, Hq, D, layer=0)  # without max_nodes: the kernels for the mean rows


@pytest.mark.parametrize("requests,groups,Hq,Hkv,D,dtype,page,mask,nodes", CASES[1:6])
def test_small_tables(requests, groups, Hq, Hkv, D, dtype, page, mask, nodes):
    """So few positions that the call is tree attention: the same bits."""
    x = make(requests, groups, Hq, Hkv, D, dtype, page, 5, mask=mask, wide=False)
    got = run(x, groups, Hq, D, max_nodes=nodes).out
    cache, _, off, L, q, m = x
    ref = spec.TreeAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L), m,
                             max_nodes=nodes)(layer=1)
    assert torch.equal(got.view(torch.int16), ref.view(torch.int16))


def test_no_groups_and_no_shared_positions():
    requests = [(300, 1), (270, 2), (0, 1)]
    x = make(requests, [], 4, 2, 128, BF, 16, 1)
    run(x, [], 4, 128)
    run(x, [(0, 3, 0)], 4, 128)
    run(x, [(0, 0, 100), (0, 2, 100), (2, 0, 5), (2, 1, 0)], 4, 128)
    cache, table, off, L, q, m = x
    none = spec.PrefixAttention(cache, q[:0], ints([0, 0, 0, 0]), ints(L), *tensors([(0, 3, 0)]))
    assert none().shape == (0, 4, 128)


def test_positions_without_a_page_are_not_there():
    requests, groups = [(400, 1), (420, 1), (410, 3)], [(0, 3, 400)]
    x = make(requests, groups, 4, 1, 64, F16, 16, 2)
    cache, table = x[0], x[1]
    table[:, 3] = -1
    table[:, 17] = cache.args.n_pages + 7
    table[1, 25] = -1  # of its own
    cache.page_table.copy_(torch.from_numpy(table))
    run(x, groups, 4, 64)


@pytest.mark.parametrize("length", [400, 0])
def test_a_request_without_rows_says_nothing_of_the_prefix(length):
    """A sample that has ended: its pages given back, its length still there or not."""
    requests, groups = [(400, 0), (420, 1), (0, 0), (410, 2)], [(0, 4, 400)]
    x = make(requests, groups, 4, 2, 128, BF, 16, 4)
    cache, table, off, L, q, m = x
    table[[0, 2]] = -1
    L[0] = length
    cache.page_table.copy_(torch.from_numpy(table))
    run(x, groups, 4, 128)


def test_infinities_stay_with_the_rows_that_see_them():
    requests, groups = [(300, 4), (310, 2)], [(0, 2, 288)]
    x = make(requests, groups, 4, 2, 128, BF, 16, 3, fill=float("inf"))
    cache, table, off, L, q, _ = x
    # A node of the first request that only itself sees.
    m = torch.tensor([[1], [0b11], [0b101], [0b1001], [1], [0b11]], device=DEV)
    x = (cache, table, off, L, q, m)
    run(x, groups, 4, 128)
    at = L[0] + 2
    cache.v[1, table[0, at // 16], at % 16] = float("inf")
    out = spec.PrefixAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L), *tensors(groups),
                               m)(layer=1)
    assert not torch.isfinite(out[2]).any()
    assert torch.isfinite(out[[0, 1, 3, 4, 5]]).all()


def test_strided_rows_and_large_scores():
    requests, groups = [(300, 1), (280, 2), (290, 1)], [(0, 3, 272)]
    cache, table, off, L, q, m = make(requests, groups, 4, 1, 64, BF, 16, 4)
    wide = torch.zeros((4, 6, 64), dtype=BF, device=DEV)
    wide[:, 1:5] = q * 8
    cache.k.mul_(8)
    out = torch.full((4, 6, 64), 3.0, dtype=BF, device=DEV)
    args = (torch.from_numpy(off).to(DEV), ints(L))
    got = spec.PrefixAttention(cache, wide[:, 1:5], *args, *tensors(groups), m, scale=1.0,
                               out=out[:, :4])(layer=1)
    assert (out[:, 4:] == 3.0).all()
    ref = spec.TreeAttention(cache, wide[:, 1:5], *args, m, scale=1.0)(layer=1)
    # |s| up to 2^12: e^(2^-6) on each p in either (see test_gpu_spec_decode), of
    # values below 5, and the roundings of both.
    assert float((got.float() - ref.float()).abs().max()) < 5 * (2 * 2.0 ** -6 + 4 * U[BF])


@pytest.mark.parametrize("B,groups", [(4096, 1), (4096, 4096), (1500, 37)])
def test_many_requests(B, groups):
    say(f"prefix, {B} requests in {groups} groups")
    cut = np.linspace(0, B, groups + 1).astype(int)
    shape = [(int(a), int(b - a), 256) for a, b in zip(cut, cut[1:])]
    g = torch.Generator(DEV).manual_seed(B + groups)
    k, v = (torch.randn((1, 64, 16, 1, 64), generator=g, device=DEV).to(BF) for _ in range(2))
    table = torch.randint(0, 64, (groups, 18), generator=g, device=DEV).int()
    of = torch.repeat_interleave(torch.arange(groups, device=DEV),
                                 torch.tensor([s[1] for s in shape], device=DEV))
    table = table[of].contiguous()
    table[:, 16:] = torch.randint(0, 64, (B, 2), generator=g, device=DEV).int()
    cache = spec.KvCache(k, v, table, torch.full((B,), 18, dtype=torch.int32, device=DEV),
                         torch.ones(64, dtype=torch.int32, device=DEV))
    L = (257 + torch.arange(B, device=DEV) % 20).int()
    q = torch.randn((B, 2, 64), generator=g, device=DEV).to(BF)
    off = torch.arange(B + 1, device=DEV).int()
    got = spec.PrefixAttention(cache, q, off, L, *tensors(shape), max_nodes=1)().clone()
    # Against the formula in float64, all requests at once.
    pos = torch.arange(288, device=DEV)
    rows = table.long()[:, pos // 16] * 16 + pos % 16
    K, V = k.view(-1, 64).double()[rows], v.view(-1, 64).double()[rows]
    s = torch.einsum("bhd,bpd->bhp", q.double(), K) / 8
    s.masked_fill_(pos[None, None] > L[:, None, None], -math.inf)
    p = torch.softmax(s, -1)
    ref, size = torch.einsum("bhp,bpd->bhd", p, V), torch.einsum("bhp,bpd->bhd", p, V.abs())
    tol = U[BF] * (size * (1 + 1 / 16) + ref.abs()) + 2.0 ** -25
    assert ((got.double() - ref).abs() <= tol).all()


def test_offsets_past_32_bits():
    """Pages more than 2^31 elements apart."""
    say("prefix, pages 2.4e9 bytes apart")
    page, D, stride = 16, 64, 1_200_000_000
    pool = torch.empty(2 * stride + 4096, dtype=BF, device=DEV)
    k, v = (torch.as_strided(pool, (1, 3, page, 1, D), (0, stride, D, D, 1), o) for o in (0, 2048))
    for i, x in enumerate((k, v)):
        x.copy_(torch.randn((1, 3, page, 1, D), generator=torch.Generator(DEV).manual_seed(i),
                            device=DEV))
    table = np.tile(np.array([[2, 0, 1, 2, 1, 0, 2, 2, 0, 1]], np.int32), (2, 1))
    table = np.pad(table, ((0, 0), (0, room(2, 1, D, page))), constant_values=-1)
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints([10, 10]), ints([2, 2, 2]))
    q = torch.randn((2, 3, D), generator=torch.Generator(DEV).manual_seed(5), device=DEV).to(BF)
    x = (cache, table, np.array([0, 1, 2], np.int32), [150, 140], q, None)
    run(x, [(0, 2, 130)], 3, D, layer=0)


def test_after_forks_it_gives_what_tree_attention_gives():
    """The pages that KvCache.fork shares, with rows of the requests' own behind."""
    B, P, page = 6, 333, 16
    cache = spec.KvCache.empty(2, 200, page, 2, 128, B, room(B, 2, 128, page))
    lengths, status = ints([0] * B), ints([0] * B)
    slots = ints([0] * P)
    cache.reserve(lengths, ints([0] + [P] * B), slots, status)
    g = torch.Generator(DEV).manual_seed(9)
    rope = spec.QkNormRope(cache, torch.randn((P, 12, 128), generator=g, device=DEV).to(BF), 8, None,
                           slots)
    rope(layer=0)
    lengths.copy_(ints([P] + [0] * (B - 1)))
    done = ints([0] * (B - 1))
    cache.fork(lengths, ints([0] * (B - 1)), ints(list(range(1, B))), done)
    assert done.tolist() == [1] * (B - 1) and lengths.tolist() == [P] * B
    shared = P // page * page
    for step in range(3):
        off, slots = ints(list(range(B + 1))), ints([0] * B)
        cache.reserve(lengths, off, slots, status)
        qkv = torch.randn((B, 12, 128), generator=g, device=DEV).to(BF)
        rope = spec.QkNormRope(cache, qkv, 8, None, slots)
        q = rope(layer=0)
        got = spec.PrefixAttention(cache, q, off, lengths, ints([0, B]), ints([shared]))(layer=0)
        check_attention(got, f64(q), cache, cache.page_table.cpu().numpy(), 0, list(range(B + 1)),
                        lengths.tolist(), None, 1 / math.sqrt(128), BF)
        lengths += 1


def test_streams_and_graphs():
    """Two objects on two streams, and captured calls replayed with other lengths and
    groups."""
    groups = [(0, 3, 256), (3, 3, 384)]
    requests = [(300, 1), (310, 1), (290, 1), (500, 1), (400, 1), (444, 1)]
    xs = [make(requests, groups, 8, 2, 128, BF, 16, 20, mask=False),
          make(requests, groups, 4, 1, 64, F16, 16, 21, mask=False)]
    live = [(ints(x[3]), *tensors(groups)) for x in xs]
    calls = [spec.PrefixAttention(x[0], x[4], torch.from_numpy(x[2]).to(DEV), *t, max_nodes=1)
             for x, t in zip(xs, live)]
    ref = [c().clone() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for c, s in zip(calls, streams):
            c.out.fill_(0)
            s.wait_stream(torch.cuda.current_stream())
            c(stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(c.out, r) for c, r in zip(calls, ref))
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, capture_error_mode="thread_local"):
            c()
        graphs.append(g)
    for lengths, shared in (([299, 260, 290, 490, 385, 444], [256, 128]), ([300] * 6, [0, 256]),
                            (xs[0][3], [100, 384])):
        for t in live:
            t[0].copy_(ints(lengths))
            t[2].copy_(ints(shared))
        want = [spec.PrefixAttention(x[0], x[4], torch.from_numpy(x[2]).to(DEV), *t, max_nodes=1)()
                for x, t in zip(xs, live)]
        torch.cuda.synchronize()
        for c, g in zip(calls, graphs):
            c.out.fill_(0)
            g.replay()
        torch.cuda.synchronize()
        for c, r in zip(calls, want):  # (a length past its rows reads NaN)
            assert torch.equal(c.out.view(torch.int16), r.view(torch.int16))

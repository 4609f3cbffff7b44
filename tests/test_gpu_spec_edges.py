"""The paged-cache operators where they were once wrong, against the float64
oracle (tolerances as derived in ``test_gpu_spec_decode``, or where they are
used)."""
import math

import numpy as np
import pytest
import torch

from oracle import spec_decode as S
from paper_2601_01310_amd import spec
from tests.test_gpu_spec_decode import (DEV, check_attention, f64, ints, make_pool, random_masks,
                                        say, verify_inputs)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,Hq,Hkv,D,dtype,page", [
    (33, 4, 1, 128, torch.bfloat16, 16), (64, 2, 1, 64, torch.float16, 4),
    (64, 2, 2, 256, torch.bfloat16, 32), (40, 8, 2, 128, torch.float16, 64)])
def test_trees_that_fill_their_mask_words(n, Hq, Hkv, D, dtype, page):
    """Contexts after which a tile's second half lies past the mask's last
    word, the last request's row among them."""
    say(f"attention, {n} nodes in one word, Hq={Hq} D={D}")
    rng = np.random.default_rng(n + D)
    L = [64, 31, 28, 32]
    cache, table = make_pool([x + n for x in L], page, Hkv, D, dtype, rng)
    off = [n * b for b in range(len(L) + 1)]
    q = torch.randn((n * len(L), Hq, D), device=DEV).to(dtype)
    mask = random_masks([n] * len(L), rng)
    out = spec.TreeAttention(cache, q, ints(off), ints(L), mask, max_nodes=n)()
    check_attention(out, f64(q), cache, table, 0, off, L, mask, 1 / math.sqrt(D), dtype)


@pytest.mark.parametrize("page,together,trim", [(16, False, True), (8, True, False)])
def test_rows_after_a_rollback_below_a_fork_leave_the_parent_alone(page, together, trim):
    """A child goes back to fewer tokens than it shares and writes new rows:
    the parent's rows keep their bits, and so do the child's remaining ones."""
    say(f"rollback below a fork, page {page}")
    rng = np.random.default_rng(page)
    n, back = 2 * page, 2 * page - page // 2 - 1
    cache, _ = make_pool([n, 0], page, 2, 64, torch.bfloat16, rng, layers=3, together=together,
                         spare=6)
    lengths, status = ints([n, 0]), ints([7])
    cache.fork(lengths, ints([0]), ints([1]), status)
    assert status.tolist() == [1] and lengths.tolist() == [n, n]
    lengths.copy_(ints([n, back]))
    if trim:
        cache.trim(lengths)

    def tokens(b, m):
        table = cache.page_table[b].tolist()
        return torch.stack([x[:, table[p // page], p % page] for x in (cache.k, cache.v)
                            for p in range(m)])

    parent, child = tokens(0, n), tokens(1, back)
    rows = page + 3
    off, slots, status = ints([0, 0, rows]), ints([9] * rows), ints([9, 9])
    cache.reserve(lengths, off, slots, status)
    assert status.tolist() == [1, 1]
    refs = cache.refcount.tolist()
    assert all(refs[s // page] == 1 for s in slots.tolist())
    qkv = torch.randn((rows, 8, 64), device=DEV).to(torch.bfloat16)
    rope = spec.QkNormRope(cache, qkv, 4, None, slots)
    for layer in range(3):
        rope(layer=layer)
    assert torch.equal(tokens(0, n), parent)
    assert torch.equal(tokens(1, back), child)
    new = tokens(1, back + rows).view(2, back + rows, 3, 2, 64)[:, back:]
    assert torch.equal(new[0], qkv[:, None, 4:6].expand(-1, 3, -1, -1))
    assert torch.equal(new[1], qkv[:, None, 6:].expand(-1, 3, -1, -1))


def test_a_decode_batch_takes_the_kernel_of_single_rows_by_default():
    say("attention, decode batch without max_nodes")
    rng = np.random.default_rng(11)
    L = rng.integers(0, 90, 130).tolist()
    cache, table = make_pool([x + 1 for x in L], 16, 2, 128, torch.bfloat16, rng)
    q = torch.randn((130, 8, 128), device=DEV).to(torch.bfloat16)
    off = list(range(131))
    by_default = spec.TreeAttention(cache, q, ints(off), ints(L))
    told = spec.TreeAttention(cache, q, ints(off), ints(L), max_nodes=1)
    assert by_default.ws_bytes == told.ws_bytes
    assert torch.equal(by_default(), told())
    check_attention(told.out, f64(q), cache, table, 0, off, L, None, 1 / math.sqrt(128),
                    torch.bfloat16)


@pytest.mark.parametrize("Hq,Hkv,D,dtype,page", [
    (4, 1, 128, torch.bfloat16, 16), (6, 1, 64, torch.float16, 32), (2, 1, 256, torch.bfloat16, 4),
    (40, 2, 64, torch.bfloat16, 8)])
def test_a_long_request_among_short_ones_without_max_nodes(Hq, Hkv, D, dtype, page):
    """Many row tiles of a kernel that is chosen for few rows."""
    say(f"attention, one request of 90 rows among 40 of one, Hq={Hq} D={D}")
    rng = np.random.default_rng(D)
    N = [1] * 20 + [90, 0] + [1] * 20
    L = rng.integers(0, 200, len(N)).tolist()
    cache, table = make_pool([a + b for a, b in zip(L, N)], page, Hkv, D, dtype, rng)
    off = np.concatenate([[0], np.cumsum(N)]).astype(np.int32)
    q = torch.randn((int(off[-1]), Hq, D), device=DEV).to(dtype)
    mask = random_masks(N, rng)
    for m in (mask, None):
        call = spec.TreeAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L), m)
        check_attention(call(), f64(q), cache, table, 0, off, L, m, 1 / math.sqrt(D), dtype)


@pytest.mark.parametrize("rows,Hq,D", [(1, 2, 64), (12, 4, 128), (40, 2, 64), (9, 4, 256)])
def test_f16_keeps_a_long_context_behind_one_large_score(rows, Hq, D):
    """The first token scores about 18 above all others, whose values alone
    make the output: each of their probabilities is 2^-26 of the largest.

    f16's subnormal step limits a probability to 2^-25 / 2^7 of the largest
    score's: up to 2^-32 |v| for each position, over the sum of e^(s - max).
    """
    say(f"attention, f16 behind a large score, {rows} rows, D={D}")
    rng = np.random.default_rng(rows)
    L = 6000
    k = torch.zeros((1, (L + rows + 63) // 64, 64, 1, D), dtype=torch.float16, device=DEV)
    v = torch.zeros_like(k)
    table = rng.permutation(k.shape[1]).astype(np.int32)[None]
    at = torch.from_numpy(table[0].astype(np.int64)).to(DEV)
    q = torch.randn((rows, Hq, D), device=DEV).half()
    q[..., 0] = 4.0
    K = torch.randn((k.shape[1] * 64, D), device=DEV) * 0.1
    V = 1 + 0.5 * torch.randn((k.shape[1] * 64, D), device=DEV)
    K[:, 0] = 0
    K[0], V[0] = 0, 0
    K[0, 0] = 18 * math.sqrt(D) / 4
    k[0, at, :, 0], v[0, at, :, 0] = K.half().view(-1, 64, D), V.half().view(-1, 64, D)
    ones = torch.ones(k.shape[1], dtype=torch.int32, device=DEV)
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints([k.shape[1]]), ones)
    got = f64(spec.TreeAttention(cache, q, ints([0, rows]), ints([L]))())
    hk, hv, hq = f64(k[0, at].flatten(0, 1)[:, 0]), f64(v[0, at].flatten(0, 1)[:, 0]), f64(q)
    for r in range(rows):
        n = L + r + 1
        for h in range(Hq):
            s = hk[:n] @ hq[r, h] / math.sqrt(D)
            p = np.exp(s - s.max())
            ref, size = p @ hv[:n] / p.sum(), p @ np.abs(hv[:n]) / p.sum()
            tol = (2.0 ** -11 * (size * (1 + 1 / 16) + np.abs(ref)) + 2.0 ** -25
                   + 2.0 ** -32 * np.abs(hv[:n]).sum(0) / p.sum())
            assert s[0] - s[1:].max() > 17 and ref.min() > 20 * tol.max()
            assert (np.abs(got[r, h] - ref) <= tol).all(), (r, h, got[r, h][:4], ref[:4], tol[:4])


@pytest.mark.parametrize("sampled", [False, True])
def test_requests_without_pages_keep_nothing(sampled):
    """Pages for two of three requests: the third one's rows are not cached, so
    it keeps none of them, and its length stays until it gets pages."""
    say(f"verify with a status, sampled={sampled}")
    n, V, page = 6, 500, 4
    cache = spec.KvCache.empty(1, 4, page, 1, 64, 3, 3, device=DEV)
    lengths, new, off = ints([0, 0, 0]), ints([-1] * 3), ints([0, n, 2 * n, 3 * n])
    slots, status = ints([9] * 3 * n), ints([9] * 3)
    p, q, mask, off_h, tokens, u, un = verify_inputs([n] * 3, V, sampled, 5)
    p.zero_()
    p[:, 7] = 1.0
    tokens[:] = 7  # every draft would stay
    if sampled:
        q.copy_(p)
    say("  reserve, verify, compact")
    check = spec.VerifyTree(p, *(torch.from_numpy(x).to(DEV) for x in (tokens, u, un)), off, mask,
                            max_path=n, draft_probs=q, status=status)
    cache.reserve(lengths, off, slots, status)
    assert status.tolist() == [1, 1, 0] and set(slots.tolist()[2 * n:]) == {-1}
    got = [x.cpu().numpy() for x in check()]
    ref = S.verify(p.cpu().numpy(), None if q is None else q.cpu().numpy(), tokens, u, un, off_h,
                   None if mask is None else mask.cpu().numpy().view(np.uint64), n, [1, 1, 0])
    for a, b in zip(got, ref):
        assert np.array_equal(a, b)
    assert got[2].tolist()[0] > 1 and got[2].tolist()[2] == 0
    cache.compact(check.path, check.n_out, lengths, new)
    assert new.tolist() == got[2].tolist()
    cache.trim(ints([0, 0, 0]))
    cache.reserve(lengths, off, slots, status)  # all pages free: still two of three
    assert status.tolist() == [1, 1, 0]
    status.copy_(ints([0, 1, 1]))
    assert check()[2].tolist()[0] == 0


def test_a_batch_without_requests_gets_no_slots():
    """Slots kept from another batch must not lead rows into the cache."""
    say("reserve without requests")
    cache = spec.KvCache.empty(1, 4, 16, 1, 64, 0, 2, device=DEV)
    slots = ints([5] * 70)
    cache.reserve(ints([]), ints([0]), slots, ints([]))
    assert slots.tolist() == [-1] * 70
    cache.reserve(ints([]), ints([0]), slots[:0], ints([]))
    assert cache.refcount.tolist() == [0] * 4


def test_one_row_may_come_with_any_stride():
    """A slice of one row keeps the stride of what it was cut from."""
    say("one row, odd strides")
    rng = np.random.default_rng(12)
    cache, table = make_pool([40], 16, 1, 64, torch.bfloat16, rng)
    wide = torch.randn((1, 4 * 64 + 3), device=DEV).to(torch.bfloat16)
    q = torch.as_strided(wide, (1, 4, 64), (4 * 64 + 3, 64, 1))
    off, L = ints([0, 1]), ints([39])
    a = spec.TreeAttention(cache, q, off, L)()
    assert torch.equal(a, spec.TreeAttention(cache, q.contiguous().view(1, 4, 64), off, L)())
    qkv = torch.as_strided(wide, (1, 4, 64), (4 * 64 + 3, 64, 1))
    slots, w = ints([39]), torch.ones(64, dtype=torch.bfloat16, device=DEV)
    want = spec.QkNormRope(cache, qkv, 2, None, slots, None, w, w)().clone()
    spec.QkNormRope(cache, qkv, 2, None, slots, None, w, w, q_out=qkv[:, :2])()  # in place
    assert torch.equal(qkv[:, :2], want)


def test_norms_and_rotation_either_side_of_the_choice_of_grid():
    """A row takes a wave or several, by the number of rows: the same bits."""
    say("qk, 2559 to 2561 rows of 20 heads")
    rng = np.random.default_rng(13)
    T, D = 2561, 128
    cache, _ = make_pool([1], 16, 4, D, torch.bfloat16, rng, spare=T // 16 + 1, fill=0.0)
    qkv = torch.randn((T, 20, D), device=DEV).to(torch.bfloat16)
    w = torch.randn((2, D), device=DEV).to(torch.bfloat16)
    t = torch.randn((T, D), device=DEV)
    pos, slots = ints(rng.permutation(T).tolist()), ints(rng.permutation(T).tolist())
    got = []
    for n in (T, T - 1, T - 2, 7):
        for x in (cache.k, cache.v):
            x.zero_()
        q = spec.QkNormRope(cache, qkv[:n], 12, pos[:n], slots[:n], t, *w)()
        k, v = (x[0].flatten(0, 1)[slots.long()] for x in (cache.k, cache.v))
        got.append((n, q, k, v))
    for n, *parts in got[1:]:
        for a, b in zip(parts, got[0][1:]):
            assert torch.equal(a[:n], b[:n]), n
            assert (a[n:] == 0).all()


@pytest.mark.parametrize("nodes,Hq,D,dtype", [
    (1, 4, 128, torch.bfloat16), (40, 2, 64, torch.float16), (40, 2, 128, torch.bfloat16),
    (40, 1, 256, torch.bfloat16), (1, 4, 256, torch.float16)])
def test_the_most_requests_of_a_batch(nodes, Hq, D, dtype):
    """4096 requests: the sums of their work take their whole place in LDS."""
    say(f"attention, 4096 requests, kernel of {nodes} rows, D={D}")
    rng = np.random.default_rng(D + nodes)
    B, page = 4096, 4
    L = rng.integers(0, 4, B)
    L[[5, 4095]] = 130
    N = rng.integers(0, 3, B)
    N[[5, 4095]] = nodes
    held = -(-(L + N) // page)
    table = np.full((B, int(held.max())), -1, np.int32)
    order = rng.permutation(int(held.sum())).astype(np.int32)
    for b, at in enumerate(np.cumsum(held) - held):
        table[b, :held[b]] = order[at:at + held[b]]
    k, v = (torch.randn((1, len(order), page, 1, D), device=DEV).to(dtype) for _ in range(2))
    cache = spec.KvCache(k, v, torch.from_numpy(table).to(DEV), ints(held.tolist()),
                         torch.ones(len(order), dtype=torch.int32, device=DEV))
    off = np.concatenate([[0], np.cumsum(N)]).astype(np.int32)
    q = torch.randn((int(off[-1]), Hq, D), device=DEV).to(dtype)
    out = spec.TreeAttention(cache, q, torch.from_numpy(off).to(DEV), ints(L.tolist()),
                             max_nodes=max(nodes, 2))()
    some = sorted({0, 5, 63, 64, 4095, *rng.integers(0, B, 60).tolist()})
    rows = np.concatenate([np.arange(off[b], off[b + 1]) for b in some])
    part = np.concatenate([[0], np.cumsum(N[some])]).astype(np.int32)
    check_attention(out[rows], f64(q[rows]), cache, table[some], 0, part, L[some], None,
                    1 / math.sqrt(D), dtype)


@pytest.mark.parametrize("Hq,D,dtype,page,masked,L", [
    (2, 128, torch.bfloat16, 16, False, 70), (1, 64, torch.float16, 64, True, 0),
    (1, 256, torch.bfloat16, 32, True, 33)])
def test_the_most_rows_of_a_request(Hq, D, dtype, page, masked, L):
    """A prompt's chunk of 1024 rows, and one row more, which is not written."""
    say(f"attention, 1024 rows, D={D} masked={masked}")
    rng = np.random.default_rng(D)
    n = 1024
    cache, table = make_pool([L + n], page, 1, D, dtype, rng)
    q = torch.randn((n + 1, Hq, D), device=DEV).to(dtype)
    mask = random_masks([n + 1], rng, words=17)[:, :16].contiguous() if masked else None
    out = torch.full((n + 1, Hq, D), 3.0, dtype=dtype, device=DEV)
    spec.TreeAttention(cache, q, ints([0, n + 1]), ints([L]), mask, out=out)()
    assert (out[n] == 3.0).all()
    check_attention(out[:n], f64(q[:n]), cache, table, 0, [0, n], [L],
                    None if mask is None else mask[:n], 1 / math.sqrt(D), dtype)


@pytest.mark.parametrize("sampled", [False, True])
def test_verification_of_the_most_nodes(sampled):
    say(f"verify 1024 nodes, sampled={sampled}")
    for seed in range(3):
        p, q, mask, off, tokens, u, un = verify_inputs([1024, 3], 40, sampled, seed)
        u *= 0.05  # long paths
        u[1] = 0.0
        call = spec.VerifyTree(p, *(torch.from_numpy(x).to(DEV) for x in (tokens, u, un, off)),
                               tree_mask=mask, max_path=1024, draft_probs=q)
        got = [t.cpu().numpy() for t in call()]
        ref = S.verify(p.cpu().numpy(), None if q is None else q.cpu().numpy(), tokens, u, un, off,
                       None if mask is None else mask.cpu().numpy().view(np.uint64), 1024)
        for a, b in zip(got, ref):
            assert np.array_equal(a, b), seed

"""Pins of the oracle of the paged-cache operators (CPU): closed forms,
invariants and exhaustive enumeration."""
import itertools
import math

import numpy as np
import pytest

from oracle import spec_decode as S


def test_rotation_keeps_norms_and_depends_on_relative_positions():
    rng = np.random.default_rng(1)
    D, rot = 64, 32
    q, k = rng.normal(size=(2, D))
    angle = 100.0 ** (-np.arange(rot // 2) / (rot // 2))
    for inter in (False, True):
        def at(x, pos):
            t = np.concatenate([np.cos(angle * pos), np.sin(angle * pos)])
            return S.norm_rope(x, None, t, 1e-6, inter)
        assert abs(np.linalg.norm(at(q, 17)) - np.linalg.norm(q)) < 1e-12
        assert np.array_equal(at(q, 5)[rot:], q[rot:])
        assert abs(at(q, 12) @ at(k, 5) - at(q, 107) @ at(k, 100)) < 1e-10
    y = S.norm_rope(q, np.full(D, 2.0), [], 0.0, False)
    assert abs(np.mean(y * y) - 4.0) < 1e-12


def test_attention_of_a_chain_is_causal_attention():
    rng = np.random.default_rng(2)
    size, L, n, D = 4, 6, 3, 8
    k, v = rng.normal(size=(2, 5, size, 1, D))
    table = np.array([[3, 1, 4, -1]], np.int32)
    q = rng.normal(size=(n, 2, D))
    out = S.tree_attention(q, k, v, table, [0, n], [L], None, 0.3)
    K, V = (t[[3, 1, 4], :, 0].reshape(-1, D) for t in (k, v))
    for i in range(n):
        e = np.exp(q[i] @ K[:L + i + 1].T * 0.3)
        assert np.allclose(out[i], e @ V[:L + i + 1] / e.sum(1, keepdims=True), atol=1e-13)
    mask = np.array([[1], [2 | 1], [4 | 1]], np.uint64)  # two children of the root
    tree = S.tree_attention(q, k, v, table, [0, n], [L], mask, 0.3)
    assert np.allclose(tree[:2], out[:2]) and not np.allclose(tree[2], out[2])
    none = S.tree_attention(q, k, v, table, [0, n], [0], np.zeros((n, 1), np.uint64), 0.3)
    assert np.array_equal(none, np.zeros_like(none))


GRID = 8  # probabilities in eighths, random numbers at the middles of eighths


def _law(p, q, tokens, masks, n_u):
    """Exact law of the first token that comes out, over a grid of random
    numbers on which every decision of these inputs is exact."""
    us = [(i + 0.5) / GRID for i in range(GRID)]
    law = np.zeros(p.shape[1])
    for u in itertools.product(us, repeat=n_u):
        r = S.verify_request(p, q, tokens, [0.0] + list(u[1:]) + [0.0] * len(tokens), u[0], masks, 9)
        law[r["tokens"][0]] += 1
    return law / GRID ** n_u


def test_verified_chains_follow_the_target():
    """Token x drafted from q, kept with min(1, p/q), else from max(p - q, 0):
    over q's draws the first token follows p."""
    p = np.array([[4, 2, 2, 0], [2, 2, 2, 2]], np.float32) / GRID
    q = np.array([[2, 4, 0, 2], [2, 2, 2, 2]], np.float32) / GRID
    law = sum(q[0, x] * _law(p, q, [0, x], [1, 3], 2) for x in range(4))
    assert np.allclose(law, p[0], atol=1e-12), law


def test_verified_trees_follow_the_target():
    """Children of the root, chosen without chance: kept with the mass that the
    refused ones left. With p = 4/8, 2/8, 2/8 the tests and the draw divide the
    grid evenly."""
    p = np.array([[4, 2, 2, 0]] + [[2, 2, 2, 2]] * 3, np.float32) / GRID
    for tokens in ([9, 0], [9, 0, 1], [9, 3, 0], [9, 0, 0, 2]):
        masks = [1] + [1 | 1 << j for j in range(1, len(tokens))]
        law = _law(p[:len(tokens)], None, tokens, masks, len(tokens))
        assert np.allclose(law, p[0], atol=1e-12), (tokens, law)


def test_verification_walks_the_tree():
    V = 6
    p = np.zeros((5, V), np.float32)
    # root -> {1: token 2, 2: token 3}, 2 -> {3: token 4}, 3 -> {4: token 5}
    for row, x in ((0, 3), (1, 0), (2, 4), (3, 1), (4, 0)):
        p[row, x] = 1.0
    masks = [0b1, 0b11, 0b101, 0b1101, 0b11101]
    tok, u = [0, 2, 3, 4, 5], [0.9] * 5
    r = S.verify_request(p, None, tok, u, 0.5, masks, 9)
    assert r == dict(path=[0, 2, 3], tokens=[3, 4, 1])
    assert S.verify_request(p, None, tok, u, 0.5, masks, 2) == dict(path=[0, 2], tokens=[3, 4])
    assert S.verify_request(p, None, tok, u, 0.5, masks, 1) == dict(path=[0], tokens=[3])
    assert S.verify_request(p[:1], None, tok[:1], u, 0.0, None, 4) == dict(path=[0], tokens=[3])


def test_draw_takes_the_lowest_token_past_the_mass():
    assert S.draw([0, 3, 0, 1], 0) == 1
    assert S.draw([0, 3, 0, 1], (3 << 22) - 1) == 1
    assert S.draw([0, 3, 0, 1], 3 << 22) == 3
    assert S.draw([0, 0], 5) is None
    assert S.units(np.nan) == 0 and S.units(2.0) == 1 << 36 and S.units(-1.0) == 0
    assert S.units24(1.0) == (1 << 24) - 1 and S.units24(np.nan) == 0


def test_pages_are_conserved():
    rng = np.random.default_rng(3)
    B, size, n = 5, 4, 40
    pages = S.Pages(np.full((B, 12), -1), np.zeros(B), np.zeros(n), size,
                    [rng.normal(size=(2, n, size, 3))])
    lengths = np.zeros(B, np.int64)
    for step in range(30):
        add = rng.integers(0, 6, B)
        off = np.concatenate([[0], np.cumsum(add)])
        slots, status = pages.reserve(lengths, off, off[-1])
        lengths = np.minimum(lengths + add * status, 30)
        used = slots[slots >= 0]
        assert len(set(used)) == len(used)
        b = int(rng.integers(B))
        keep = lengths.copy()
        keep[b] = 0
        pages.trim(keep)
        lengths = keep
        src = int(rng.integers(B))
        before = pages.table[src].copy()
        if src != b:
            st = pages.fork(lengths, [src], [b])
            if st[0]:
                L = int(lengths[b])
                c = pages.caches[0]
                for pos in range(L):
                    x, y = pages.table[b, pos // size], pages.table[src, pos // size]
                    assert np.array_equal(c[:, x, pos % size], c[:, y, pos % size])
        assert np.array_equal(before, pages.table[src]) or src == b
        held = [p for row in pages.table for p in row if p >= 0]
        assert np.array_equal(np.bincount(held, minlength=n), pages.ref)
        assert [int((row >= 0).sum()) for row in pages.table] == pages.held.tolist()


@pytest.mark.parametrize("path", [[0], [0, 1, 2], [0, 2, 5], [0, 1, 4, 7]])
def test_compaction_moves_the_path_together(path):
    size, L = 4, 6
    c = np.arange(2 * 6 * size).reshape(2, 6, size, 1).astype(float)
    before = c.copy()
    table = np.array([[5, 0, 3, 2]])
    pages = S.Pages(table, [4], [1] * 6, size, [c])
    new = pages.compact(np.array([path]), [len(path)], [L])
    assert new.tolist() == [L + len(path)]
    for i, j in enumerate(path):
        src, dst = (before[:, table[0, (L + x) // size], (L + x) % size] for x in (j, i))
        assert np.array_equal(c[:, table[0, (L + i) // size], (L + i) % size], src)
    assert math.isfinite(c.sum())

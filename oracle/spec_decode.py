"""Oracle of the operators around the paged KV cache (numpy, float64, one
request, row and node at a time).

Test infrastructure like ``moe_ew``: it shares no code with the HIP path and
follows the definitions of ``include/tg.h`` directly. Probabilities are whole
numbers of 2**-36 and random numbers whole numbers of 2**-24 there, so the
verification is done in Python's integers and has one answer.
"""
from __future__ import annotations

import math
from typing import Dict, List, Optional

import numpy as np


def mask_bits(words: np.ndarray) -> int:
    """One row of a uint64 tree mask as a Python integer."""
    return sum(int(w) << (64 * i) for i, w in enumerate(np.asarray(words).astype(np.uint64)))


# --------------------------------------------------------------------------
# Norms and rotation
# --------------------------------------------------------------------------


def norm_rope(x, weight, cos_sin_row, eps, interleaved) -> np.ndarray:
    """One head [D]: RMS norm (``weight`` None: as it is), then its first
    rot = len(cos_sin_row) elements turned."""
    y = np.array(x, np.float64)
    if weight is not None:
        y = y / math.sqrt(float(np.mean(y * y)) + eps) * np.asarray(weight, np.float64)
    rot = len(cos_sin_row)
    out = y.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = float(cos_sin_row[i]), float(cos_sin_row[rot // 2 + i])
        out[a], out[b] = y[a] * c - y[b] * s, y[b] * c + y[a] * s
    return out


# --------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------


def positions_seen(length, n_nodes, node, bits: Optional[int]) -> List[int]:
    """Positions that a row sees; ``bits`` None: a chain."""
    own = range(node + 1) if bits is None else [j for j in range(n_nodes) if bits >> j & 1]
    return list(range(length)) + [length + j for j in own]


def attend(q, k, v, scale) -> np.ndarray:
    """One row and head: q [D] over k, v [positions, D] (those it sees)."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros(q.shape[0])
    s = k @ q * scale
    p = np.exp(s - s.max())
    return p @ v / p.sum()


def tree_attention(q, k_pages, v_pages, table, q_offsets, lengths, tree_mask, scale) -> np.ndarray:
    """q [T, Hq, D]; pages [n_pages, page_size, Hkv, D]; out [T, Hq, D]."""
    T, Hq, D = q.shape
    n_pages, size, Hkv, _ = k_pages.shape
    out = np.zeros((T, Hq, D))
    for b in range(len(lengths)):
        n = q_offsets[b + 1] - q_offsets[b]
        L = max(0, int(lengths[b]))
        for node in range(n):
            r = q_offsets[b] + node
            bits = None if tree_mask is None else mask_bits(tree_mask[r])
            at = []
            for p in positions_seen(L, n, node, bits):
                if p // size < table.shape[1] and 0 <= table[b, p // size] < n_pages:
                    at.append((table[b, p // size], p % size))
            pages, rows = (np.array([a[i] for a in at], np.int64) for i in (0, 1))
            for h in range(Hq):
                g = h // (Hq // Hkv)
                out[r, h] = attend(q[r, h], k_pages[pages, rows, g], v_pages[pages, rows, g], scale)
    return out


# --------------------------------------------------------------------------
# Verification
# --------------------------------------------------------------------------


def units(p) -> int:
    """A probability in units of 2**-36."""
    p = float(p)
    return 0 if not p > 0 else int(math.floor(min(p, 1.0) * 2 ** 36))


def units24(u) -> int:
    u = float(u)
    return 0 if not u > 0 else min(int(math.floor(u * 2 ** 24)), 2 ** 24 - 1)


def draw(weights: List[int], u24: int) -> Optional[int]:
    """The lowest index whose cumulative weight exceeds u * the whole."""
    whole = sum(weights)
    if whole == 0:
        return None
    to, run = u24 * whole >> 24, 0
    for i, w in enumerate(weights):
        run += w
        if run > to:
            return i
    raise AssertionError("u < 1")


def verify_request(p, q, tokens, u_accept, u_next, masks, max_path) -> Dict[str, list]:
    """One request: p (and q, or None) [n, V], tokens [n], masks [n] integers
    (None: a chain). A walk from the root, child by child."""
    n, V = len(tokens), p.shape[1]
    if n == 0:
        return dict(path=[], tokens=[])
    masks = [(1 << (j + 1)) - 1 for j in range(n)] if masks is None else masks
    children: List[List[int]] = [[] for _ in range(n)]
    for j in range(1, n):
        up = masks[j] & ((1 << j) - 1)
        if up and bin(up).count("1") + 1 <= max_path:
            children[up.bit_length() - 1].append(j)
    path, out = [0], []
    while True:
        at = path[-1]
        left, seen, kept = 1 << 36, set(), None
        for j in children[at] if q is None else children[at][:1]:
            x = int(tokens[j])
            w = units(p[at, x]) if 0 <= x < V else 0
            u = units24(u_accept[j])
            if q is not None:
                if u * (units(q[at, x]) if 0 <= x < V else 0) < w << 24:
                    kept = j
                break
            if x in seen:
                continue
            if u * max(left, 0) < w << 24:
                kept = j
                break
            left -= w
            seen.add(x)
        if kept is None:
            break
        path.append(kept)
        out.append(int(tokens[kept]))
    at = path[-1]
    whole = [units(x) for x in p[at]]
    weights = list(whole)
    if children[at]:
        if q is None:
            for j in children[at]:
                if 0 <= int(tokens[j]) < V:
                    weights[int(tokens[j])] = 0
        else:
            weights = [max(a - units(b), 0) for a, b in zip(whole, q[at])]
    u = units24(u_next)
    x = draw(weights, u)
    if x is None:
        x = draw(whole, u)
    return dict(path=path, tokens=out + [0 if x is None else x])


def verify(p, q, tokens, u_accept, u_next, q_offsets, tree_mask, max_path, status=None):
    """(tokens_out [B, max_path], path [B, max_path], n_out [B])."""
    B = len(u_next)
    tok, path = (np.full((B, max_path), -1, np.int32) for _ in range(2))
    n_out = np.zeros(B, np.int32)
    for b in range(B):
        if status is not None and status[b] == 0:
            continue
        s = slice(q_offsets[b], q_offsets[b + 1])
        masks = None if tree_mask is None else [mask_bits(m) for m in tree_mask[s]]
        r = verify_request(p[s], None if q is None else q[s], tokens[s], u_accept[s], u_next[b],
                           masks, max_path)
        n_out[b] = len(r["path"])
        path[b, :n_out[b]] = r["path"]
        tok[b, :n_out[b]] = r["tokens"]
    return tok, path, n_out


# --------------------------------------------------------------------------
# Pages
# --------------------------------------------------------------------------


class Pages:
    """Page bookkeeping one request and page at a time, and the cache's rows
    ([layers, pages, page_size, width] arrays, changed in place)."""

    def __init__(self, table, held, refcount, page_size, caches=()):
        self.table, self.held, self.ref = (np.array(a, np.int32) for a in (table, held, refcount))
        self.size, self.caches = page_size, caches

    def _take(self) -> int:
        p = int(np.flatnonzero(self.ref == 0)[0])
        self.ref[p] = 1
        return p

    def pages_of(self, tokens) -> int:
        return -(-max(0, int(tokens)) // self.size)

    def reserve(self, lengths, q_offsets, T):
        B, width = self.table.shape
        slots, status = np.full(T, -1, np.int32), np.zeros(B, np.int32)
        free, short = int((self.ref == 0).sum()), False
        before, dropped = self.ref.copy(), []
        for b in range(B):
            n, L = max(0, int(q_offsets[b + 1] - q_offsets[b])), max(0, int(lengths[b]))
            want = self.pages_of(L + n)
            if want > width:
                continue
            # Held pages that new rows would lie in and that others hold too.
            shared = [j for j in range(L // self.size, min(int(self.held[b]), want))
                      if n and 0 <= self.table[b, j] < len(before) and before[self.table[b, j]] > 1]
            new = max(0, want - int(self.held[b]))
            short = short or len(shared) + new > free
            if shared + [0] * new and short:
                continue
            free -= len(shared) + new
            for j in shared:
                old, p = int(self.table[b, j]), self._take()
                used = L % self.size if j == L // self.size else 0
                for c in self.caches:
                    c[:, p, :used] = c[:, old, :used]
                self.table[b, j] = p
                dropped.append(old)
            for _ in range(new):
                self.table[b, self.held[b]] = self._take()
                self.held[b] += 1
            status[b] = 1
            for i in range(n):
                p = self.table[b, (L + i) // self.size]
                if p >= 0:
                    slots[q_offsets[b] + i] = p * self.size + (L + i) % self.size
        for p in dropped:
            self.ref[p] -= 1
        return slots, status

    def fork(self, lengths, src, dst):
        B, n = self.table.shape[0], len(src)
        status = np.zeros(n, np.int32)
        held0, free, short = self.held.copy(), int((self.ref == 0).sum()), False
        for i in range(n):
            s, d = int(src[i]), int(dst[i])
            if not (0 <= s < B and 0 <= d < B) or s in dst or d in dst[:i] or held0[d]:
                continue
            L = max(0, int(lengths[s]))
            if held0[s] < self.pages_of(L):
                continue
            need = int(L % self.size > 0)
            short = short or need > free
            if need and short:
                continue
            free -= need
            whole = L // self.size
            for j in range(whole):
                self.table[d, j] = self.table[s, j]
                self.ref[self.table[s, j]] += 1
            if need:
                p = self._take()
                self.table[d, whole] = p
                for c in self.caches:
                    c[:, p, :L % self.size] = c[:, self.table[s, whole], :L % self.size]
            self.held[d], lengths[d], status[i] = whole + need, L, 1
        return status

    def trim(self, keep):
        for b in range(self.table.shape[0]):
            for j in range(self.pages_of(keep[b]), int(self.held[b])):
                self.ref[self.table[b, j]] -= 1
                self.table[b, j] = -1
            self.held[b] = min(int(self.held[b]), self.pages_of(keep[b]))

    def compact(self, path, n_keep, lengths):
        for b in range(self.table.shape[0]):
            L = int(lengths[b])
            for c in self.caches:
                rows = []
                for i in range(int(n_keep[b])):
                    pos = L + int(path[b, i])
                    rows.append(c[:, self.table[b, pos // self.size], pos % self.size].copy())
                for i, row in enumerate(rows):
                    c[:, self.table[b, (L + i) // self.size], (L + i) % self.size] = row
        return np.asarray(lengths) + np.asarray(n_keep)

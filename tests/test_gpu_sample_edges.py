"""tg_sample on the GPU at the edges of its range: rows whose border holds more tokens
than the lists, logits of every bit pattern, tails of small weights. Expected values
follow from the definition in whole numbers and float64."""
import math
from fractions import Fraction

import pytest
import torch

from paper_2601_01310_amd import spec

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def border(k, p, m, n, ratio):
    """How many of m tokens of weight 1 and n of weight ``ratio`` (Fraction) behind
    them top-k and then top-p keep, from the definition in whole numbers."""
    m, n = min(k, m), min(max(k - m, 0), n)
    if p >= 1:
        return m + n
    to = p * (m + n * ratio)  # a token stays if the mass before it is less
    if to <= m:
        return math.ceil(to)
    if ratio < 1:  # weights are rounded: not at a border (see the test)
        at = (to - m) / ratio
        assert 2.0 ** -8 < at - math.floor(at) < 1 - 2.0 ** -8
    return m + min(n, math.ceil((to - m) / ratio))


@pytest.mark.parametrize("filters", ["k", "p", "kp"])
@pytest.mark.parametrize("V,dtype", [(1 << 20, "f32"), (1 << 20, "bf16"), ((1 << 20) + 5, "f32"),
                                     (3 << 20, "f16"), (1 << 24, "f32"), (1 << 24, "bf16")])
def test_flat_rows_of_256_parts_and_more(V, dtype, filters):
    """Rows of one and of two levels, all of whose parts have more tokens at the
    border than they can list.

    Weights of one level are equal, and so whatever is counted is exact. Those of the
    lower level are within half a unit of 2^-s and 2^-42 of themselves, s >= 38 and
    e^-1 > 2^-2: 2^-36 together. Up to 2^24 of them move a border by less than 2^-8
    tokens, and a probability by less than 2^-34 of itself beside its rounding."""
    print(f"[gpu] sample, flat rows, V={V} {dtype} {filters}", flush=True)
    low = Fraction(math.exp(-1.0))  # of the upper level's weight, to 2^-53
    logits = torch.full((4, V), 0.5, device=DEV, dtype=DTYPES[dtype])
    logits[1] -= 1.0  # and rows of two levels:
    logits[2:] = 0.0
    logits[2, 13::97] = 1.0
    logits[3, V - 3:] = 1.0
    ks = [3, V - 1, V // 2, 5000] if "k" in filters else [V] * 4
    ps = [0.5, 0.3, 0.7, 0.999] if "p" in filters else [1.0] * 4
    us = [0.75, 0.999, 0.4, 0.6]
    k = torch.tensor(ks, dtype=torch.int32, device=DEV) if "k" in filters else None
    p, u = (torch.tensor(x, device=DEV) for x in (ps, us))
    s = spec.SampleTokens(logits, u, None, k, p if "p" in filters else None, probs=True)
    s.tokens.fill_(-7)
    s.probs.fill_(float("nan"))
    tokens, probs = s()
    for t in range(4):
        top = logits[t] == logits[t].max()
        m, ratio = int(top.sum()), low if t >= 2 else Fraction(1)
        n = border(ks[t], Fraction(float(p[t])), m, V - m, ratio)
        at = torch.where(top, torch.cumsum(top, 0), m + torch.cumsum(~top, 0))  # from 1
        kept = at <= n
        w = torch.where(top, 1.0, float(ratio)).double() * kept
        whole = float(w.sum())
        assert torch.equal(probs[t] > 0, kept), (t, n, int((probs[t] > 0).sum()))
        err = (probs[t].double() * whole - w).abs()
        assert bool((err <= w * (2.0 ** -24 + 2.0 ** -33)).all()), (t, float(err.max()))
        x, i = float(u[t]), int(tokens[t])
        if t < 2:
            assert i == math.floor(Fraction(x) * n), (t, i, n)
        else:
            upto, slack = torch.cumsum(w, 0), V * 2.0 ** -36
            assert bool(kept[i]) and float(upto[i]) > x * whole - slack, (t, i)
            assert float(upto[i] - w[i]) <= x * whole + slack, (t, i)


BITS = {  # NaN: signalling and quiet ones, of both signs, least and largest payloads
    "f32": (torch.int32, (0x7F800001, 0x7FBFFFFF, 0xFF800001, 0xFFBFFFFF, 0x7FC00000, 0xFFFFFFFF)),
    "bf16": (torch.int16, (0x7F81, 0x7FBF, 0xFF81, 0xFFBF, 0x7FC0, 0xFFFF)),
    "f16": (torch.int16, (0x7C01, 0x7DFF, 0xFC01, 0xFDFF, 0x7E00, 0xFFFF)),
}


@pytest.mark.parametrize("dtype", list(BITS))
@pytest.mark.parametrize("V", [3, 1000, 9001])
def test_no_nan_is_a_token(V, dtype):
    """A logit of any NaN's bits counts as -infinity's does, in whole vectors and at a
    row's end, with and without filters and for the likeliest token."""
    print(f"[gpu] sample, NaN, V={V} {dtype}", flush=True)
    kind, codes = BITS[dtype]
    bits = 8 * torch.empty((), dtype=kind).element_size()
    codes = [c - (1 << bits) if c >> (bits - 1) else c for c in codes]
    T, g = len(codes) + 1, torch.Generator(DEV).manual_seed(V)
    logits = torch.randn((T, V), generator=g, device=DEV).to(DTYPES[dtype])
    ref = logits.clone()
    gone = torch.rand((T, V), generator=g, device=DEV) < 0.3
    gone[:, -1] = True
    gone[:, 1] = False
    gone[T - 1] = True
    ref[gone] = -math.inf
    for t in range(T):
        logits[t].view(kind)[gone[t]] = codes[t % len(codes)]
    assert bool(logits[gone].isnan().all()) and not logits[~gone].isnan().any()
    u = torch.rand(T, generator=g, device=DEV)
    full = lambda x, kind=torch.float32: torch.full((T,), x, dtype=kind, device=DEV)  # noqa: E731
    for f in ((None,) * 4, (full(0.0), None, None, None), (full(0.7), full(20, torch.int32), None, None),
              (None, None, full(0.8), None), (None, None, None, full(0.1)),
              (full(1.3), full(30, torch.int32), full(0.9), full(0.01))):
        a, b = (spec.SampleTokens(x, u, *f, probs=True)() for x in (logits, ref))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert not a[1][gone].any() and int(a[0][T - 1]) == -1
        assert bool((~gone[:T - 1].gather(1, a[0][:T - 1, None].long())).all())


def test_nothing_stays_behind_the_border():
    """A long tail of weights of a few units: rounded to these, the tokens of the
    border's step come to less than the share that their masses before the rounding
    gave, and all of them stay. Those behind them do not.

    V = 2^19, s = 43, and the likeliest token's weight is 2^43 units. n tokens have 4.4
    units (4, rounded) and n, less likely, 2.4 (2). top_p = 1 - 2^-24 leaves out
    2^19 = 524288 units, more than the latter have together (483958), so none of them
    stays."""
    print("[gpu] sample, tails of small weights", flush=True)
    V, n = 1 << 19, 201649
    logits = torch.full((1, V), -math.inf, device=DEV)
    at = torch.randperm(V, generator=torch.Generator(DEV).manual_seed(3), device=DEV)
    top, some, rest = at[:1], at[1:n + 1], at[n + 1:2 * n + 1]
    logits[0, top] = 0.0
    logits[0, some] = -math.log(2.0) * (43 - math.log2(4.4))
    logits[0, rest] = -math.log(2.0) * (43 - math.log2(2.4))
    p = torch.full((1,), 1 - 2.0 ** -24, device=DEV)
    for u in (0.5, 1 - 2.0 ** -24):
        token, probs = spec.SampleTokens(logits, torch.full((1,), u, device=DEV), top_p=p, probs=True)()
        assert not probs[0, rest].any(), int(probs[0, rest].count_nonzero())
        assert float(probs[0, top]) > 0.5 and probs[0, some].any()
        assert float(probs[0, int(token)]) > 0

"""tg_sample on the GPU against its definition in float64: the drawn token, the
tokens that stay and their probabilities.

Tolerances. A weight is e^((l - max) / temperature), of the largest 1. The kernel's
have a relative error of at most 2^-42 (a polynomial to 2^-44, float64 products, and
t = l log2 e / temperature, whose rounding at |t| < 512 is 2^-44) and are rounded
to units of at most 2^(1 - s), s = min(45, 62 - ceil(log2 V)). Sums over V weights
that come to M are therefore within V 2^(1 - s) + 2^-42 M (SLACK below), and so are
the borders that go by them. A token whose border is nearer than that may be on
either side."""
import math

import pytest
import torch

from paper_2601_01310_amd import spec, tg

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def row_of(l, hot, k, p, m):
    """(weights in token order, kept for sure, kept maybe, slack) of one row in
    float64 on the CPU; None for a row without tokens."""
    l = l.double().cpu()
    l = torch.where(l.isnan(), -math.inf, l).clamp(max=3.4028234663852886e38)
    V = l.numel()
    if l.max() == -math.inf:
        return None
    if not hot > 0:
        w = torch.zeros(V, dtype=torch.float64)
        w[int((l == l.max()).nonzero()[0])] = 1.0
        return w, w > 0, w > 0, 0.0
    w = torch.where(l == -math.inf, 0.0, torch.exp((l - l.max()) / hot))
    s = min(45, 62 - math.ceil(math.log2(V))) if V > 1 else 45
    order = torch.sort(l, dim=0, descending=True, stable=True).indices
    ranked = w[order]
    sure = ranked > 2.0 ** (1 - s)
    maybe = ranked > 0
    if k > 0:
        sure[k:] = False
        maybe[k:] = False
    mass = float(ranked[maybe].sum())
    slack = V * 2.0 ** (1 - s) + 2.0 ** -42 * mass
    if p < 1:
        before = torch.cumsum(ranked * maybe, 0) - ranked * maybe
        first = torch.arange(V) == 0
        sure &= (before < p * mass - slack) | first
        maybe &= (before < p * mass + slack) | first
    if m > 0:
        first = torch.arange(V) == 0
        sure &= (ranked >= min(m, 1.0) * (1 + 2.0 ** -40) + 2.0 ** (1 - s)) | first
        maybe &= (ranked >= min(m, 1.0) * (1 - 2.0 ** -40) - 2.0 ** (1 - s)) | first
    a, b = torch.zeros(V, dtype=torch.bool), torch.zeros(V, dtype=torch.bool)
    a[order], b[order] = sure, maybe
    return w, a, b, slack


def check(s, logits, u, hot=None, k=None, p=None, m=None, what=""):
    """Runs ``s`` (with probs) and checks every row."""
    T, V = logits.shape
    s.tokens.fill_(-7)
    s.probs.fill_(float("nan"))
    tokens, probs = s()
    tokens, probs = tokens.cpu(), probs.cpu()
    for t in range(T):
        get = lambda x, d: d if x is None else float(x[t])  # noqa: E731
        nan = lambda x, d: d if x != x else x  # noqa: E731
        ref = row_of(logits[t], get(hot, 1.0), int(get(k, 0)), nan(get(p, 1.0), 1.0),
                     nan(get(m, 0.0), 0.0))
        if ref is None:
            assert int(tokens[t]) == -1 and not probs[t].any(), (what, t)
            continue
        w, sure, maybe, slack = ref
        got = probs[t] > 0
        # (a probability may be too small for float32)
        assert not (got & ~maybe).any(), (what, t, "kept too many")
        tiny = w < 1e-37 * float(w[maybe].sum())
        assert not (sure & ~got & ~tiny).any(), (what, t, "kept too few")
        kept = got | (sure & tiny)
        mass = float(w[kept].sum())
        err = (probs[t].double() - w * kept / mass).abs()
        assert float(err.max()) <= 2.0 ** -24 + 2 * slack / mass, (what, t, float(err.max()))
        i = int(tokens[t])
        assert 0 <= i < V and (kept[i] or maybe[i]), (what, t, i)
        at = float(u[t])
        at = min(max(at, 0.0), 1.0 - 2.0 ** -53) if at == at else 0.0  # clamped into [0, 1)
        upto = torch.cumsum(w * kept, 0)
        lo = float(upto[i] - w[i])
        assert lo <= at * mass + slack and (float(upto[i]) > at * mass - slack), (what, t, i)
    return tokens


def make(logits, u, hot=None, k=None, p=None, m=None, probs=True):
    return spec.SampleTokens(logits, u, hot, k, p, m, probs=probs)


def batch(T, V, dtype, seed, filters):
    g = gen(seed)
    logits = torch.randn((T, V), generator=g, device=DEV).mul_(3.0)
    logits = logits.to(DTYPES[dtype])
    u = torch.rand(T, generator=g, device=DEV)
    hot = 0.4 + torch.rand(T, generator=g, device=DEV)
    k = p = m = None
    if "k" in filters:
        k = torch.randint(1, 60, (T,), generator=g, device=DEV).int()
        k[0] = min(V, 7)
    if "p" in filters:
        p = 0.3 + 0.69 * torch.rand(T, generator=g, device=DEV)
    if "m" in filters:
        m = 0.3 * torch.rand(T, generator=g, device=DEV)
    return logits, u, hot, k, p, m


@pytest.mark.parametrize("V", [1, 2, 5, 63, 1000, 1023, 1024, 1025, 8191, 8193, 32003, 70001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("filters", ["", "k", "p", "m", "kp", "pm", "kpm"])
def test_against_float64(V, dtype, filters):
    print(f"[gpu] sample V={V} {dtype} {filters}", flush=True)
    a = batch(5, V, dtype, V + len(filters), filters)
    tokens = check(make(*a), *a)
    # Without the distribution, and each row alone: the same token.
    assert torch.equal(make(*a, probs=False)().cpu(), tokens)
    for t in (0, 4):
        one = [None if x is None else x[t:t + 1].contiguous() for x in a]
        assert int(make(*one, probs=False)()) == int(tokens[t])


@pytest.mark.parametrize("V", [(1 << 20) + 5, 3_000_001, 1 << 24])
@pytest.mark.parametrize("filters", ["", "kp", "p"])
def test_large_vocabularies(V, filters):
    print(f"[gpu] sample V={V} {filters}", flush=True)
    a = batch(2, V, "f32", 3, filters)
    check(make(*a), *a)


@pytest.mark.parametrize("filters", ["", "k", "p", "kp", "pm"])
@pytest.mark.parametrize("V", [40, 4099, 20000, 131073])
def test_ties(V, filters):
    """Equal logits are ordered by their index, however many there are (more than
    any list holds)."""
    T = 6
    logits = torch.zeros((T, V), device=DEV)
    logits[1] = torch.randint(0, 3, (V,), generator=gen(1), device=DEV).float()
    logits[2, V // 2:] = 1.0
    logits[3] = -0.0
    logits[3, ::2] = 0.0
    logits[4] = torch.arange(V, device=DEV).float() * 1e-6
    logits[5] = -torch.arange(V, device=DEV).float() * 1e-6
    u = torch.rand(T, generator=gen(2), device=DEV)
    k = torch.tensor([3, V // 3, 1, V - 1, V // 2 + 1, 39], dtype=torch.int32, device=DEV) \
        if "k" in filters else None
    p = torch.tensor([0.5, 0.25, 0.999, 0.1, 0.7, 0.5], device=DEV) if "p" in filters else None
    m = torch.tensor([0.5, 0.5, 0.1, 1.0, 0.999, 0.99], device=DEV) if "m" in filters else None
    a = (logits, u, None, k, p, m)
    check(make(*a), *a)


def test_top_k_beyond_the_tokens_that_have_a_weight():
    """Cold rows, most of whose tokens are too small to count."""
    V = 9000
    logits = torch.randn((6, V), generator=gen(4), device=DEV).mul_(4)
    u = torch.rand(6, generator=gen(5), device=DEV)
    hot = torch.tensor([0.05, 0.1, 0.02, 1e-3, 0.2, 0.3], device=DEV)
    k = torch.tensor([500, 8999, 3000, 50, 2000, 4000], dtype=torch.int32, device=DEV)
    for p in (None, torch.full((6,), 0.99, device=DEV)):
        a = (logits, u, hot, k, p, None)
        check(make(*a), *a)


def test_rows_of_equal_logits_keep_the_first_ones():
    V = 6000
    logits = torch.full((2, V), 2.5, device=DEV)
    u = torch.tensor([0.999999, 0.0], device=DEV)
    s = make(logits, u, None, None, torch.tensor([0.5, 0.5], device=DEV))
    tokens, probs = s()
    assert tokens.tolist() == [2999, 0]  # 3000 tokens have half of the mass
    assert (probs[:, :3000] == torch.tensor(1 / 3000, dtype=torch.float32)).all()
    assert not probs[:, 3000:].any()


def test_masked_and_odd_logits():
    inf, nan = math.inf, math.nan
    V = 9000
    logits = torch.randn((8, V), generator=gen(5), device=DEV)
    logits[0] = -inf
    logits[1] = nan
    logits[2, 1:] = -inf
    logits[3, ::3] = nan
    logits[3, 1::3] = -inf
    logits[4, 77] = inf
    logits[4, 8999] = inf
    logits[5] = -3e38
    logits[5, 5:9] = 3e38
    logits[6, :] = -inf
    logits[6, 8998:] = 1.0
    logits[7] = logits[7] * 1e30
    u = torch.rand(8, generator=gen(6), device=DEV)
    for f in (dict(), dict(k=torch.full((8,), 4, dtype=torch.int32, device=DEV)),
              dict(p=torch.full((8,), 0.9, device=DEV)),
              dict(m=torch.full((8,), 0.5, device=DEV), p=torch.full((8,), 0.5, device=DEV))):
        a = (logits, u, None, f.get("k"), f.get("p"), f.get("m"))
        tokens = check(make(*a), *a)
        assert tokens[:2].tolist() == [-1, -1] and int(tokens[2]) == 0
        assert int(tokens[4]) in (77, 8999)
    half = logits[:5].to(torch.float16)
    a = (half, u[:5].contiguous(), None, None, None, None)
    check(make(*a), *a)


def test_odd_parameters():
    inf, nan = math.inf, math.nan
    V, T = 3000, 9
    logits = torch.randn((1, V), generator=gen(7), device=DEV).expand(T, V).contiguous()
    f = lambda *v: torch.tensor(v, device=DEV)  # noqa: E731
    u = f(0.0, 1.0, 1.0 - 2.0 ** -24, nan, -1.0, 0.5, 0.5, 0.5, 2.0)
    hot = f(0.0, -1.0, nan, 1e-6, 1e6, 1.0, 1.0, 1e-38, 1.0)
    k = torch.tensor([0, -5, V, V + 7, 1, 0, 2, 0, V - 1], dtype=torch.int32, device=DEV)
    p = f(1.0, 0.0, nan, 1.5, -1.0, 0.0, 0.999999, 0.5, nan)
    m = f(0.0, 2.0, nan, -1.0, 0.3, nan, 0.0, 1.0, 5.0)
    a = (logits, u, hot, k, p, m)
    tokens = check(make(*a), *a)
    best = int(logits[0].argmax())
    for t in (0, 1, 2, 4, 5, 8):  # greedy, or nothing but the likeliest stays
        assert int(tokens[t]) == best, t
    # An infinite temperature: every token that is one, alike.
    logits[0, 5] = -inf
    s = make(logits[:1].contiguous(), f(0.5), f(inf))
    token, probs = s()
    assert int(probs.count_nonzero()) == V - 1 and float(probs[0, 5]) == 0.0
    assert abs(float(probs.max()) * (V - 1) - 1) < 1e-6 and abs(int(token) - V // 2) <= 1


def test_the_law_of_the_draw():
    """Over evenly spaced random numbers a token comes as often as its probability
    says, up to one."""
    N, V = 4096, 50
    for f in (dict(), dict(p=0.8), dict(k=10), dict(m=0.2)):
        logits = torch.randn((1, V), generator=gen(11), device=DEV).mul_(2).expand(N, V).contiguous()
        u = (torch.arange(N, device=DEV) + 0.5) / N
        full = lambda n, dt: None if n not in f else torch.full((N,), f[n], dtype=dt, device=DEV)  # noqa: E731
        s = make(logits, u, None, full("k", torch.int32), full("p", torch.float32),
                 full("m", torch.float32))
        tokens, probs = s()
        counts = torch.bincount(tokens.long(), minlength=V).double()
        assert float((counts - N * probs[0].double()).abs().max()) <= 1.001


def test_strides_and_alignment():
    V, T = 5003, 4
    base = torch.randn((T, V + 13), generator=gen(8), device=DEV).mul_(3)
    u = torch.rand(T, generator=gen(9), device=DEV)
    p = torch.full((T,), 0.9, device=DEV)
    for dtype in DTYPES.values():
        for off in (0, 1, 3, 8):
            logits = base.to(dtype)[:, off:off + V]
            store = torch.full((T, V + 9), -1.0, device=DEV)
            s = spec.SampleTokens(logits, u, None, None, p, None, probs=store[:, 2:2 + V])
            check(s, logits, u, None, None, p, None)
            assert (store[:, :2] == -1).all() and (store[:, 2 + V:] == -1).all()
            ref = make(logits.contiguous(), u, None, None, p)
            assert torch.equal(s.tokens, ref()[0])


def test_rows_that_overlap_are_refused():
    """Expanded rows have a stride of 0 (and a store of them has no place of its own)."""
    one, u = torch.zeros((1, 50), device=DEV), torch.zeros(3, device=DEV)
    with pytest.raises(tg.TgError):
        spec.SampleTokens(one.expand(3, 50), u)
    with pytest.raises(tg.TgError):
        spec.SampleTokens(one.expand(3, 50).contiguous(), u, probs=one.expand(3, 50))
    # Of one row the stride says nothing.
    assert spec.SampleTokens(one, u[:1])().tolist() == [0]


def test_no_rows():
    s = make(torch.zeros((0, 50), device=DEV), torch.zeros(0, device=DEV))
    tokens, probs = s()
    assert tokens.shape == (0,) and probs.shape == (0, 50)


def test_streams_and_graphs():
    """Two objects on two streams, and captured calls replayed with other logits."""
    cases = [batch(3, 20000, "f32", 1, "kpm"), batch(40, 50000, "bf16", 2, "p")]
    ss = [make(*a) for a in cases]
    ref = [[x.clone() for x in s()] for s in ss]
    streams = [torch.cuda.Stream() for _ in ss]
    for _ in range(5):
        for s, st in zip(ss, streams):
            s.tokens.fill_(-9)
            st.wait_stream(torch.cuda.current_stream())
            s(st)
        torch.cuda.synchronize()
        for s, r in zip(ss, ref):
            assert torch.equal(s.tokens, r[0]) and torch.equal(s.probs, r[1])
    graphs = []
    for s in ss:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, capture_error_mode="thread_local"):
            s()
        graphs.append(g)
    for i in range(4):
        for a in cases:
            a[0].copy_(torch.roll(a[0], 17 + i, 1))
        want = [[x.clone() for x in make(*a)()] for a in cases]
        torch.cuda.synchronize()
        for s, g in zip(ss, graphs):
            s.tokens.fill_(-9)
            g.replay()
        torch.cuda.synchronize()
        for s, r in zip(ss, want):
            assert torch.equal(s.tokens, r[0]) and torch.equal(s.probs, r[1]), i

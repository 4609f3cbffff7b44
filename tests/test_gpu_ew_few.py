"""The forward of a few tokens (tg_ew_few) on the GPU: against the formula in
float64, against tg_ew_forward's routing bit for bit, and on its own: a token's
result depends neither on its batch nor on the slot that serves it."""
import dataclasses

import pytest
import torch

from paper_2601_01310_amd import synth, tg

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = 2.0 ** -8  # a bf16 rounding, relative


def few(wl, weights=None, alive=None, valid=None, x=None, logits=None):
    w13, s13, w2, s2 = weights or (wl.w13, None, wl.w2, None)
    return tg.EwFew(wl.x if x is None else x, wl.wg, wl.logits if logits is None else logits, wl.ert,
                    wl.alive if alive is None else alive, w13, w2, wl.k, w13_scale=s13, w2_scale=s2,
                    token_valid=valid)


def f8_weights(wl, seed):
    """8-bit weights with every finite code in them and scales over many powers
    of two; shadows are copies."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def one(w):
        S, rows, cols = w.shape
        codes = torch.randint(0, 256, w.shape, generator=g, device=DEV).to(torch.uint8)
        codes = torch.where(codes & 127 == 127, 0, codes)  # no NaN
        scale = 1e-4 * torch.exp2(torch.randint(-6, 7, (S, rows // 128, cols // 128), generator=g,
                                                device=DEV).float())
        for s in range(S):
            e = wl.slot_expert[s]
            codes[s], scale[s] = codes[e], scale[e]
        return codes.view(torch.float8_e4m3fn), scale.contiguous()

    return (*one(wl.w13), *one(wl.w2))


def plain(w, scale):
    w = w.double()
    if scale is not None:
        w = w * scale.double().repeat_interleave(128, 0).repeat_interleave(128, 1)
    return w


def check(f, wl, weights=None, x=None, what=""):
    """Every element against the formula in float64.

    h is rounded to bf16 (BF of it) after float32 sums of d products (each of at
    most d 2^-24 of the products' absolute sum; 2^-20 of h for the exponential and
    the reciprocal), out is rounded once more after I products."""
    w13, s13, w2, s2 = weights or (wl.w13, None, wl.w2, None)
    x = (wl.x if x is None else x).double()
    T, I, d = f.out.shape[0], wl.I, wl.d
    ref = torch.zeros((T, d), dtype=torch.float64, device=DEV)
    room = torch.zeros_like(ref)
    slots, w = f.pair_slot.cpu(), f.topk_w.double()
    for s in range(w13.shape[0]):
        pairs = [(t, j) for t in range(T) for j in range(wl.k) if int(slots[t, j]) == s]
        if not pairs:
            continue
        t = torch.tensor([p[0] for p in pairs], device=DEV)
        W13, W2 = plain(w13[s], None if s13 is None else s13[s]), plain(w2[s], None if s2 is None else s2[s])
        g, u = (x[t] @ W13.t()).split(I, 1)
        eg, eu = (d * 2.0 ** -24 * (x[t].abs() @ W13.abs().t())).split(I, 1)
        h = g * torch.sigmoid(g) * u
        eh = (BF + 2.0 ** -20) * h.abs() + 1.1 * u.abs() * eg + (g * torch.sigmoid(g)).abs() * eu \
            + 1.1 * eg * eu
        y, ey = h @ W2.t(), (eh + I * 2.0 ** -24 * h.abs()) @ W2.abs().t()
        for i, (a, j) in enumerate(pairs):
            ref[a] += w[a, j] * y[i]
            room[a] += w[a, j] * ey[i]
    got = f.out.double()
    limit = 1.01 * room + BF * ref.abs() + 1e-30
    bad = (got - ref).abs() > limit
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / limit).max()))
    # Two roundings of at most BF, evenly spread: 0.82 BF in the mean square.
    if ref.norm() > 0:
        assert float((got - ref).norm() / ref.norm()) < BF, what


CASES = [  # T, d, E, k, I, local, shadows, gate
    (1, 128, 4, 1, 128, 4, [], "weights"),
    (1, 256, 8, 2, 512, 8, [0, 3], "weights"),
    (2, 192, 8, 2, 320, 8, [1], "logits"),
    (3, 4096, 8, 2, 1024, 8, [0], "weights"),
    (4, 1024, 32, 8, 256, 8, [0, 1], "logits"),
    (5, 448, 16, 4, 704, 16, [2], "weights"),
    (8, 7168, 256, 8, 256, 32, [3, 4, 5], "logits"),
    (16, 2048, 64, 6, 512, 32, [0], "weights"),
    (17, 576, 8, 2, 192, 8, [5], "logits"),
    (24, 256, 300, 9, 128, 40, [0], "logits"),
    (31, 1152, 6, 3, 640, 3, [0, 0], "logits"),
    (32, 512, 8, 8, 256, 8, [7], "weights"),
    (32, 128, 1000, 8, 128, 200, [], "logits"),
]


@pytest.mark.parametrize("T,d,E,k,I,local,shadows,gate", CASES)
@pytest.mark.parametrize("kind", ["bf16", "f8"])
def test_against_float64(T, d, E, k, I, local, shadows, gate, kind):
    print(f"[gpu] few T={T} d={d} E={E} k={k} I={I} {gate} {kind}", flush=True)
    if kind == "f8" and (d % 128 or I % 128):
        d, I = (d + 127) // 128 * 128, (I + 127) // 128 * 128
    wl = synth.make_custom(T=T, d=d, E=E, k=k, I=I, n_local=local, shadow_experts=shadows, gate=gate,
                           seed=T + d, device=DEV, fail_experts=shadows[:1])
    weights = f8_weights(wl, 5) if kind == "f8" else None
    f = few(wl, weights)
    f.out.fill_(float("nan"))
    f()
    torch.cuda.synchronize()
    r = tg.EwForward(wl)
    r()
    for name in ("topk_ids", "topk_w", "pair_slot", "n_unserved"):
        assert torch.equal(getattr(f, name), getattr(r, name)), name
    check(f, wl, weights)
    # Its first expert's primary fails: the shadow gives the same bits.
    if shadows:
        g = few(wl, weights, alive=wl.alive_after_failure())
        assert torch.equal(g(), f.out)
        assert not torch.equal(g.pair_slot, f.pair_slot) or not (f.pair_slot == shadows[0]).any()
    # Each token alone, and in another batch.
    for t in sorted({0, T // 2, T - 1}):
        one = few(dataclasses.replace(wl, T=1), weights, x=wl.x[t:t + 1],
                  logits=None if wl.logits is None else wl.logits[t:t + 1])
        assert torch.equal(one()[0], f.out[t]), t


def test_tokens_outside_the_batch_and_without_an_expert():
    wl = synth.make_custom(T=9, d=256, E=16, k=2, I=256, n_local=4, shadow_experts=[1], gate="logits",
                           seed=3, device=DEV)
    whole = few(wl)()
    valid = torch.tensor([1, 0, 1, 1, 0, 1, 1, 0, 1], dtype=torch.uint8, device=DEV)
    alive = wl.alive.clone()
    alive[2] = 0  # an expert without a shadow
    f = few(wl, alive=alive, valid=valid)
    f()
    r = tg.EwForward(wl, alive, token_valid=valid)
    r()
    assert torch.equal(f.pair_slot, r.pair_slot) and torch.equal(f.n_unserved, r.n_unserved)
    check(f, wl)
    for t in range(9):
        slots = f.pair_slot[t].tolist()
        if all(s < 0 for s in slots):  # +0, whatever was there
            assert (f.out[t].view(torch.int16) == 0).all()
        elif 2 not in wl.ert[f.topk_ids[t].long(), 0].tolist():
            assert torch.equal(f.out[t], whole[t])
    none = few(wl, alive=torch.zeros_like(wl.alive))
    none.out.fill_(float("nan"))
    assert (none().view(torch.int16) == 0).all()


@pytest.mark.parametrize("T,k", [(3, 8), (4, 32), (32, 8)])
def test_many_pairs_of_one_slot(T, k):
    """Experts that share a slot: more pairs than an operand has columns."""
    wl = synth.make_custom(T=T, d=256, E=40, k=k, I=192, n_local=3, shadow_experts=[], gate="logits",
                           seed=9, device=DEV)
    wl.ert.copy_(torch.arange(40, device=DEV)[:, None] % 5 // 4)  # slots 0 and 1
    f = few(wl)
    f()
    assert int((f.pair_slot == 0).sum()) > 16
    check(f, wl)
    one = few(dataclasses.replace(wl, T=1), x=wl.x[T - 1:], logits=wl.logits[T - 1:])
    assert torch.equal(one()[0], f.out[T - 1])


def test_a_large_routing_table():
    wl = synth.make_custom(T=4, d=128, E=512, k=4, I=128, n_local=8, shadow_experts=[], gate="logits",
                           seed=4, device=DEV)
    ert = torch.full((512, 16), -1, dtype=torch.int32, device=DEV)
    ert[:, 7] = torch.arange(512, device=DEV) % 8
    ert[:, 3] = 9999  # not a slot
    wl = dataclasses.replace(wl, ert=ert, R=16)
    f, r = few(wl), tg.EwForward(wl)
    f()
    r()
    assert torch.equal(f.pair_slot, r.pair_slot) and (f.pair_slot >= 0).all()
    check(f, wl)


def test_other_tokens_and_slots_do_not_matter():
    """Infinities and NaN in other tokens and in slots that nothing is sent to."""
    wl = synth.make_custom(T=6, d=512, E=8, k=2, I=256, n_local=8, shadow_experts=[0], gate="logits",
                           seed=12, device=DEV)
    ref = few(wl)().clone()
    x = wl.x.clone()
    x[1], x[4] = float("nan"), float("inf")
    out = few(wl, x=x)()
    for t in (0, 2, 3, 5):
        assert torch.equal(out[t], ref[t])
    f8 = f8_weights(wl, 2)
    a = few(wl, f8)
    ref = a().clone()
    used = set(a.pair_slot.flatten().tolist())
    idle = [s for s in range(wl.S) if s not in used]
    assert idle
    for s in idle:
        f8[0].view(torch.uint8)[s] = 0x7F
        f8[3][s] = float("nan")
    assert torch.equal(a(), ref)


def test_equal_logits_and_infinities_choose_as_the_gate_does():
    wl = synth.make_custom(T=8, d=128, E=130, k=5, I=128, n_local=130, shadow_experts=[],
                           gate="logits", seed=1, device=DEV)
    wl.logits.round_()  # many ties
    wl.logits[1] = 0.0
    wl.logits[2, ::2] = -0.0
    wl.logits[2, 1::2] = 0.0
    wl.logits[3] = -2.5
    wl.logits[4, 7:] = float("-inf")
    f, r = few(wl), tg.EwForward(wl)
    f()
    r()
    assert torch.equal(f.topk_ids, r.topk_ids) and torch.equal(f.topk_w, r.topk_w)


def test_no_tokens():
    wl = synth.make_custom(T=1, d=128, E=4, k=2, I=128, n_local=4, shadow_experts=[], gate="logits",
                           seed=1, device=DEV)
    f = few(wl, x=wl.x[:0], logits=wl.logits[:0])
    f.n_unserved.fill_(7)
    assert f().shape == (0, 128)
    assert int(f.n_unserved) == 0


def test_streams_and_graphs():
    """Two objects on two streams, and captured calls replayed with new inputs
    between eager ones."""
    wls = [synth.make_custom(T=T, d=512, E=8, k=2, I=512, n_local=8, shadow_experts=[1], gate=gate,
                             seed=T, device=DEV) for T, gate in ((2, "logits"), (20, "weights"))]
    fs = [few(w) for w in wls]
    ref = [f().clone() for f in fs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in fs]
    for _ in range(5):
        for f, s in zip(fs, streams):
            f.out.fill_(0)
            s.wait_stream(torch.cuda.current_stream())
            f(s)
        torch.cuda.synchronize()
        assert all(torch.equal(f.out, r) for f, r in zip(fs, ref))
    graphs = []
    for f in fs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, capture_error_mode="thread_local"):
            f()
        graphs.append(g)
    for i in range(4):
        for w in wls:
            w.x.copy_(torch.randn(w.x.shape, device=DEV, generator=torch.Generator(DEV).manual_seed(i)))
            if w.logits is not None:
                w.logits.copy_(torch.roll(w.logits, 1, 1))
        want = [few(w)().clone() for w in wls]
        torch.cuda.synchronize()
        for f, g in zip(fs, graphs):
            f.out.fill_(0)
            g.replay()
        torch.cuda.synchronize()
        for f, r in zip(fs, want):
            assert torch.equal(f.out, r), i

"""Refusals of the operators of a decode step behind a common prompt (prefix
attention, the forward of a few tokens, sampling): checked on the host, before
anything reaches the GPU (CPU-only tests)."""
import ctypes

import pytest
import torch

from paper_2601_01310_amd import spec, tg
from tests.test_spec_abi import P, attn_args, cache, lib  # noqa: F401 (a fixture)
from tests.test_spec_edges import _Machine

BIG = 1 << 40


def fill(a, values):
    for n, v in values.items():
        setattr(a, n, v)
    return a


def prefix_args(attn=None, **kw):
    a = tg.PrefixAttnArgs()
    a.attn = attn or attn_args()
    return fill(a, {**dict(n_groups=2, group_offsets=P, shared=P), **kw})


def few_args(ew=None, **kw):
    a = tg.EwFewArgs()
    fill(a.ew, {**dict(T=4, d=256, E=8, k=2, I=512, S=10, R=2, x=P, w_gate=P, ert=P, slot_alive=P,
                       w13=P, w2=P, out=P), **(ew or {})})
    return fill(a, kw)


F8 = dict(weights=tg.WEIGHTS_F8, w13_scale=P, w2_scale=P)


def sample_args(**kw):
    return fill(tg.SampleArgs(), {**dict(dtype=tg.F32, T=4, V=1000, logits_stride=1000,
                                         probs_stride=1000, logits=P, u=P, temperature=P, top_k=P,
                                         top_p=P, min_p=P, tokens=P, probs=P), **kw})


@pytest.mark.parametrize("bad,status", [
    (dict(n_groups=-1), tg.TG_ERR_BAD_DIM), (dict(n_groups=5000), tg.TG_ERR_UNSUPPORTED),
    (dict(group_offsets=None), tg.TG_ERR_NULL_ARG), (dict(shared=None), tg.TG_ERR_NULL_ARG),
    (dict(attn=attn_args(Hq=5)), tg.TG_ERR_BAD_DIM), (dict(attn=attn_args(layer=9)), tg.TG_ERR_BAD_DIM),
    (dict(attn=attn_args(q=None)), tg.TG_ERR_NULL_ARG),
    (dict(attn=attn_args(c=cache(D=96))), tg.TG_ERR_UNSUPPORTED),
    (dict(attn=attn_args(scale=0.0)), tg.TG_ERR_BAD_DIM),
    (dict(attn=attn_args(c=cache(B=1, Hkv=1, max_pages=1), T=1 << 23, max_nodes=1, Hq=1)),
     tg.TG_ERR_UNSUPPORTED),
    # By the requests it could be, as one group it could not.
    (dict(attn=attn_args(c=cache(B=1, max_pages=1 << 20), T=1 << 16, max_nodes=1)),
     tg.TG_ERR_UNSUPPORTED)])
def test_prefix_attention_refuses(lib, bad, status):  # noqa: F811
    a = ctypes.byref(prefix_args(**bad))
    assert lib.tg_prefix_attention(a, P, BIG, None) == status
    assert lib.tg_prefix_attention_workspace(a) == 0
    assert lib.tg_last_error()


@pytest.mark.parametrize("ew,bad,status", [
    (dict(T=33), {}, tg.TG_ERR_UNSUPPORTED), (dict(T=32, E=16, k=9), {}, tg.TG_ERR_UNSUPPORTED),
    (dict(T=-1), {}, tg.TG_ERR_BAD_DIM), (dict(k=9), {}, tg.TG_ERR_BAD_DIM),
    (dict(d=200), {}, tg.TG_ERR_UNSUPPORTED), (dict(I=64), {}, tg.TG_ERR_UNSUPPORTED),
    (dict(S=0), {}, tg.TG_ERR_BAD_DIM), (dict(S=1025), {}, tg.TG_ERR_UNSUPPORTED),
    (dict(x=None), {}, tg.TG_ERR_NULL_ARG), (dict(out=None), {}, tg.TG_ERR_NULL_ARG),
    (dict(w_gate=None), {}, tg.TG_ERR_NULL_ARG), (dict(logits_in=P), {}, tg.TG_ERR_NULL_ARG),
    (dict(slot_counts=P), {}, tg.TG_ERR_UNSUPPORTED), (dict(slot_offsets=P), {}, tg.TG_ERR_UNSUPPORTED),
    (dict(pair_row=P), {}, tg.TG_ERR_UNSUPPORTED), (dict(y=P), {}, tg.TG_ERR_UNSUPPORTED),
    (dict(w13=P + 8), {}, tg.TG_ERR_UNSUPPORTED), (dict(x=P + 2), {}, tg.TG_ERR_UNSUPPORTED),
    ({}, dict(weights=2), tg.TG_ERR_BAD_DIM), ({}, dict(w13_scale=P), tg.TG_ERR_NULL_ARG),
    ({}, dict(weights=tg.WEIGHTS_F8), tg.TG_ERR_NULL_ARG),
    ({}, dict(F8, w2_scale=None), tg.TG_ERR_NULL_ARG),
    (dict(d=192), F8, tg.TG_ERR_UNSUPPORTED), (dict(I=320), F8, tg.TG_ERR_UNSUPPORTED)])
def test_ew_few_refuses(lib, ew, bad, status):  # noqa: F811
    a = ctypes.byref(few_args(ew, **bad))
    assert lib.tg_ew_few(a, P, BIG, None) == status
    assert lib.tg_ew_few_workspace(a) == 0
    assert lib.tg_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(dtype=3), tg.TG_ERR_BAD_DIM), (dict(T=-1), tg.TG_ERR_BAD_DIM), (dict(V=0), tg.TG_ERR_BAD_DIM),
    (dict(V=(1 << 24) + 1, logits_stride=1 << 25, probs_stride=1 << 25), tg.TG_ERR_UNSUPPORTED),
    (dict(T=(1 << 31) - 1, V=1 << 24, logits_stride=1 << 24, probs_stride=1 << 24),
     tg.TG_ERR_UNSUPPORTED),
    (dict(T=1 << 23, V=1), tg.TG_ERR_UNSUPPORTED), (dict(T=1 << 22, V=4097, logits_stride=5000,
                                                         probs_stride=5000), tg.TG_ERR_UNSUPPORTED),
    (dict(logits_stride=999), tg.TG_ERR_BAD_DIM), (dict(probs_stride=999), tg.TG_ERR_BAD_DIM),
    (dict(logits=None), tg.TG_ERR_NULL_ARG), (dict(u=None), tg.TG_ERR_NULL_ARG),
    (dict(tokens=None), tg.TG_ERR_NULL_ARG), (dict(logits=P + 2), tg.TG_ERR_UNSUPPORTED),
    (dict(dtype=tg.F16, logits=P + 1), tg.TG_ERR_UNSUPPORTED),
    (dict(probs=P + 2), tg.TG_ERR_UNSUPPORTED)])
def test_sample_refuses(lib, bad, status):  # noqa: F811
    a = ctypes.byref(sample_args(**bad))
    assert lib.tg_sample(a, P, BIG, None) == status
    assert lib.tg_sample_workspace(a) == 0
    assert lib.tg_last_error()


def test_what_is_allowed(lib):  # noqa: F811
    """Workspaces of calls at the limits, which are not refused."""
    assert lib.tg_prefix_attention_workspace(ctypes.byref(prefix_args(n_groups=0, group_offsets=None,
                                                                      shared=None))) > 0
    assert lib.tg_prefix_attention_workspace(ctypes.byref(prefix_args(n_groups=4096))) > 0
    for ew in (dict(T=0, x=None, out=None, w_gate=None), dict(T=32, k=8), dict(T=8, E=32, k=32),
               dict(d=128, I=128), dict(topk_ids=P, topk_w=P, pair_slot=P, n_unserved=P, token_valid=P)):
        assert lib.tg_ew_few_workspace(ctypes.byref(few_args(ew))) > 0, ew
    assert lib.tg_ew_few_workspace(ctypes.byref(few_args(**F8))) > 0
    for kw in (dict(T=0, logits=None, u=None, tokens=None), dict(V=1), dict(probs=None, probs_stride=0),
               dict(temperature=None, top_k=None, top_p=None, min_p=None),
               dict(dtype=tg.BF16, logits=P + 2), dict(V=1 << 24, logits_stride=1 << 24, probs=None),
               dict(T=(1 << 23) - 1, V=1)):
        assert lib.tg_sample_workspace(ctypes.byref(sample_args(**kw))) > 0, kw


def test_null_arguments_and_workspaces(lib):  # noqa: F811
    for name, a in (("tg_prefix_attention", prefix_args()), ("tg_ew_few", few_args()),
                    ("tg_sample", sample_args())):
        need, call = getattr(lib, name + "_workspace"), getattr(lib, name)
        assert call(None, P, BIG, None) == tg.TG_ERR_NULL_ARG and need(None) == 0
        n = need(ctypes.byref(a))
        assert n > 0
        assert call(ctypes.byref(a), P, n - 1, None) == tg.TG_ERR_WORKSPACE
        assert call(ctypes.byref(a), None, n, None) == tg.TG_ERR_WORKSPACE
        assert call(ctypes.byref(a), P + 16, n, None) == tg.TG_ERR_WORKSPACE


@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_on_the_device_of_their_tensors(monkeypatch, current):
    m = _Machine(monkeypatch, current)
    for kind in (spec.PrefixAttention, spec.SampleTokens, tg.EwFew):
        x = kind.__new__(kind)
        x.args, x._ref, x._device, x._ws, x.ws_bytes = tg.PrefixAttnArgs(), None, 1, 0, 0
        x._call, x._run = m.lib.anything, spec._run
        x.out = x.tokens = torch.zeros(1)
        x.probs = None
        x()
    assert [(d, s) for _, d, s in m.calls] == [(1, 1001)] * 3 and m.current == current


def test_the_binding_refuses_tensors_that_do_not_fit():
    """Host tensors stand in: the checks of shapes and types come first."""
    z = torch.zeros
    x, w13, w2 = z((2, 128), dtype=torch.bfloat16), z((4, 256, 128)), z((4, 128, 128))
    ert, alive, logits = z((8, 1), dtype=torch.int32), z(4, dtype=torch.uint8), z((2, 8))
    with pytest.raises(ValueError, match="w13 is"):
        tg.EwFew(x, None, logits, ert, alive, w13, w2, 2)
    w13, w2 = w13.to(torch.bfloat16), w2.to(torch.bfloat16)
    for bad, name in ((dict(logits=z((3, 8))), "logits"), (dict(alive=z(5, dtype=torch.uint8)), "alive"),
                      (dict(w2=w2[:, :64]), "w2"), (dict(token_valid=z(2)), "token_valid"),
                      (dict(w13_scale=z((4, 1, 1))), "w13_scale")):
        a = {**dict(x=x, w_gate=None, logits=logits, ert=ert, alive=alive, w13=w13, w2=w2, k=2), **bad}
        with pytest.raises(ValueError, match=name):
            tg.EwFew(**a)
    for bad in (dict(logits=z(5)), dict(logits=z((2, 5), dtype=torch.float64))):
        with pytest.raises(ValueError):
            spec.SampleTokens(**{**dict(logits=z((2, 5)), u=z(2)), **bad})
    with pytest.raises(ValueError, match="device tensors"):
        spec.SampleTokens(z((2, 5)), z(2))

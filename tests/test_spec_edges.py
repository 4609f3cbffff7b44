"""Arguments of the paged-cache operators that were once refused or taken
wrongly (CPU-only: checked on the host, before anything reaches the GPU)."""
import ctypes

import pytest
import torch

from paper_2601_01310_amd import spec, tg
from tests.test_spec_abi import attn_args, cache, lib  # noqa: F401 (a fixture)


def test_the_limit_of_attention_goes_by_the_rows_that_there_are(lib):  # noqa: F811
    """A decode batch of 1024 requests over tables of 32768 positions, whose
    caller only knows that no request has more rows than there are."""
    c = dict(B=1024, n_pages=1 << 21, Hkv=8, max_pages=2048, page_stride=16 * 8 * 128,
             layer_stride=0)
    a = dict(T=1024, Hq=32, q_stride=4096, out_stride=4096, tree_mask=None, mask_words=0)

    def need(**kw):
        return lib.tg_tree_attention_workspace(ctypes.byref(attn_args(cache(**c), **{**a, **kw})))

    assert need(max_nodes=1024, typical_nodes=1) == need(max_nodes=1) > 0
    assert need(max_nodes=1024) > need(max_nodes=1)  # chosen for requests of 1024 rows
    assert need(max_nodes=4, T=1 << 20) > 0  # by the requests: 1024 x 4 rows
    assert need(max_nodes=1024, T=1 << 20) == 0  # 2^20 rows of 8 KV heads over 512 tiles
    assert need(max_nodes=1, typical_nodes=-1) == 0
    bad = attn_args(cache(**c), **{**a, "max_nodes": 1, "typical_nodes": -1})
    assert lib.tg_tree_attention(ctypes.byref(bad), 0x10000, 1 << 40, None) == tg.TG_ERR_BAD_DIM


@pytest.mark.parametrize("max_nodes", [1, 7, 64])
def test_more_typical_rows_than_the_bound_change_nothing(lib, max_nodes):  # noqa: F811
    def need(typical):
        return lib.tg_tree_attention_workspace(ctypes.byref(
            attn_args(max_nodes=max_nodes, typical_nodes=typical)))
    assert need(0) == need(max_nodes) == need(1000) > 0


class _Machine:
    """Several devices, each with its streams, and a library that notes what
    was current when it was called."""

    def __init__(self, monkeypatch, current):
        self.current, self.calls = current, []

        class device:
            def __init__(_, d):
                _.d = d

            def __enter__(_):
                _.was, self.current = self.current, _.d

            def __exit__(_, *exc):
                self.current = _.was

        class Lib:
            def __getattr__(_, name):
                def call(*args):
                    self.calls.append((name, self.current, args[-1]))
                    return tg.TG_OK
                return call

        self.lib = Lib()
        monkeypatch.setattr(spec, "_current_device", lambda: self.current)
        monkeypatch.setattr(spec, "_current_stream", lambda d: 1000 + d)
        monkeypatch.setattr(torch.cuda, "device", device)
        monkeypatch.setattr(spec, "_int32", lambda t, name, d, n, dim=1: 0)


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("stream,raw", [(None, 1001), (0, 0), (77, 77)])
def test_calls_run_on_the_device_of_their_tensors(monkeypatch, current, stream, raw):
    """Whatever device is current: the null stream, which torch's default
    stream is, belongs to the current one."""
    m = _Machine(monkeypatch, current)
    i = torch.zeros((3, 3), dtype=torch.int32)
    c = spec.KvCache.__new__(spec.KvCache)
    c.args, c._ref, c._device, c._lib = tg.KvCacheArgs(), None, 1, m.lib
    c.reserve(i, i, i, i, stream=stream)
    c.fork(i, i, i, i, stream=stream)
    c.trim(i, stream=stream)
    c.compact(i, i, i, i, stream=stream)
    for kind in (spec.QkNormRope, spec.TreeAttention, spec.VerifyTree):
        x = kind.__new__(kind)
        x.args, x._ref, x._device, x._ws, x.ws_bytes = tg.QkArgs(), None, 1, 0, 0
        x._call = m.lib.anything
        x.q_out = x.out = x.tokens_out = x.path = x.n_out = i
        x(stream=stream)
    assert len(m.calls) == 7
    assert {(d, s) for _, d, s in m.calls} == {(1, raw)}, m.calls
    assert m.current == current

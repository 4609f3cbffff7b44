"""Arguments of the paged-cache operators that were once refused or taken
wrongly (CPU-only: checked on the host, before anything reaches the GPU)."""
import ctypes

import pytest

from paper_2601_01310_amd import tg
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

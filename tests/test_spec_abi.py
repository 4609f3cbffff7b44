"""Refusals of the paged-cache operators: checked on the host, before anything
reaches the GPU (CPU-only tests)."""
import ctypes
import os

import pytest
import torch

from paper_2601_01310_amd import spec, tg

P = 0x10000  # bogus, aligned; every call below is refused before it is used


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(tg._LIB_PATH):
        from paper_2601_01310_amd import build
        build.build()
    return tg.load()


def cache(**kw):
    c = tg.KvCacheArgs()
    a = dict(dtype=tg.BF16, n_layers=2, n_pages=64, page_size=16, Hkv=2, D=128, B=3, max_pages=8,
             layer_stride=64 * 16 * 256, page_stride=16 * 256, k=P, v=P, page_table=P, held=P,
             refcount=P)
    a.update(kw)
    for n, v in a.items():
        setattr(c, n, v)
    return c


CACHE = [
    (dict(dtype=2), tg.TG_ERR_BAD_DIM), (dict(n_layers=0), tg.TG_ERR_BAD_DIM),
    (dict(n_pages=0), tg.TG_ERR_BAD_DIM), (dict(page_size=0), tg.TG_ERR_BAD_DIM),
    (dict(page_size=24), tg.TG_ERR_UNSUPPORTED), (dict(page_size=2048), tg.TG_ERR_UNSUPPORTED),
    (dict(D=96), tg.TG_ERR_UNSUPPORTED), (dict(B=-1), tg.TG_ERR_BAD_DIM),
    (dict(B=5000), tg.TG_ERR_UNSUPPORTED), (dict(Hkv=0), tg.TG_ERR_BAD_DIM),
    (dict(Hkv=2000, page_stride=1 << 30), tg.TG_ERR_UNSUPPORTED),
    (dict(max_pages=0), tg.TG_ERR_BAD_DIM),
    (dict(n_pages=1 << 27), tg.TG_ERR_UNSUPPORTED),
    (dict(max_pages=1 << 27), tg.TG_ERR_UNSUPPORTED),
    (dict(n_layers=20000), tg.TG_ERR_UNSUPPORTED),
    (dict(B=4096, max_pages=1 << 19, page_size=1, page_stride=256), tg.TG_ERR_UNSUPPORTED),
    (dict(page_stride=16 * 256 - 8), tg.TG_ERR_BAD_DIM),
    (dict(page_stride=16 * 256 + 4), tg.TG_ERR_UNSUPPORTED),
    (dict(layer_stride=-8), tg.TG_ERR_UNSUPPORTED),
    (dict(k=None), tg.TG_ERR_NULL_ARG), (dict(page_table=None), tg.TG_ERR_NULL_ARG),
    (dict(v=P + 8), tg.TG_ERR_UNSUPPORTED),
]


def qk_args(c=None, **kw):
    a = tg.QkArgs()
    a.cache = c or cache()
    v = dict(layer=1, T=4, Hq=4, rot=128, interleaved=0, max_pos=100, eps=1e-6, qkv_stride=1024,
             q_out_stride=512, qkv=P, q_weight=P, k_weight=P, cos_sin=P, positions=P, slots=P,
             q_out=2 * P)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return a


def attn_args(c=None, **kw):
    a = tg.TreeAttnArgs()
    a.cache = c or cache()
    v = dict(layer=1, T=4, Hq=4, max_nodes=64, mask_words=1, scale=0.1, q_stride=512, out_stride=512,
             q=P, q_offsets=P, lengths=P, tree_mask=P, out=P)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return a


def verify_args(**kw):
    a = tg.VerifyArgs()
    v = dict(B=2, T=8, V=1000, max_path=4, max_nodes=8, mask_words=1, target_stride=1000,
             draft_stride=1000, target_probs=P, draft_probs=P, tokens=P, u_accept=P, u_next=P,
             q_offsets=P, tree_mask=P, tokens_out=P, path=P, n_out=P)
    v.update(kw)
    for n, x in v.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("bad,status", CACHE)
def test_every_call_refuses_a_bad_cache(lib, bad, status):
    c = cache(**bad)
    r = ctypes.byref(c)
    assert lib.tg_kv_pages_trim(r, P, None) == status
    assert lib.tg_kv_pages_reserve(r, P, P, 4, P, P, None) == status
    assert lib.tg_kv_pages_fork(r, P, P, P, 2, P, None) == status
    assert lib.tg_kv_compact(r, P, 4, P, P, 2 * P, None) == status
    if bad.get("Hkv", 1) > 0:
        assert lib.tg_qk_norm_rope(ctypes.byref(qk_args(c)), None) == status
        assert lib.tg_tree_attention(ctypes.byref(attn_args(c)), P, 1 << 40, None) == status
        assert lib.tg_tree_attention_workspace(ctypes.byref(attn_args(c))) == 0
    assert lib.tg_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(layer=2), tg.TG_ERR_BAD_DIM), (dict(layer=-1), tg.TG_ERR_BAD_DIM),
    (dict(T=-1), tg.TG_ERR_BAD_DIM), (dict(Hq=3), tg.TG_ERR_BAD_DIM),
    (dict(Hq=2048, qkv_stride=1 << 20, q_out_stride=1 << 20), tg.TG_ERR_UNSUPPORTED),
    (dict(rot=130), tg.TG_ERR_BAD_DIM), (dict(rot=24), tg.TG_ERR_UNSUPPORTED),
    (dict(max_pos=0), tg.TG_ERR_BAD_DIM), (dict(eps=-1.0), tg.TG_ERR_BAD_DIM),
    (dict(eps=float("nan")), tg.TG_ERR_BAD_DIM), (dict(qkv_stride=1016), tg.TG_ERR_BAD_DIM),
    (dict(qkv_stride=1028), tg.TG_ERR_UNSUPPORTED), (dict(q_out_stride=100), tg.TG_ERR_BAD_DIM),
    (dict(qkv=None), tg.TG_ERR_NULL_ARG), (dict(slots=None), tg.TG_ERR_NULL_ARG),
    (dict(cos_sin=None), tg.TG_ERR_NULL_ARG), (dict(k_weight=None), tg.TG_ERR_NULL_ARG),
    (dict(q_out=P + 8), tg.TG_ERR_UNSUPPORTED), (dict(q_out=P), tg.TG_ERR_BAD_DIM)])
def test_qk_norm_rope_refuses(lib, bad, status):
    assert lib.tg_qk_norm_rope(ctypes.byref(qk_args(**bad)), None) == status
    assert lib.tg_qk_norm_rope(None, None) == tg.TG_ERR_NULL_ARG


@pytest.mark.parametrize("bad,status", [
    (dict(layer=2), tg.TG_ERR_BAD_DIM), (dict(Hq=5), tg.TG_ERR_BAD_DIM),
    (dict(max_nodes=0), tg.TG_ERR_BAD_DIM), (dict(max_nodes=65), tg.TG_ERR_BAD_DIM),
    (dict(max_nodes=2000, mask_words=40), tg.TG_ERR_UNSUPPORTED),
    (dict(mask_words=0), tg.TG_ERR_BAD_DIM), (dict(tree_mask=P + 4), tg.TG_ERR_UNSUPPORTED),
    (dict(c=cache(B=4096, max_pages=1 << 20)), tg.TG_ERR_UNSUPPORTED),
    (dict(scale=0.0), tg.TG_ERR_BAD_DIM), (dict(scale=float("nan")), tg.TG_ERR_BAD_DIM),
    (dict(scale=float("inf")), tg.TG_ERR_BAD_DIM), (dict(q_stride=504), tg.TG_ERR_BAD_DIM),
    (dict(out_stride=516), tg.TG_ERR_UNSUPPORTED), (dict(q=None), tg.TG_ERR_NULL_ARG),
    (dict(lengths=None), tg.TG_ERR_NULL_ARG), (dict(out=P + 2), tg.TG_ERR_UNSUPPORTED)])
def test_tree_attention_refuses(lib, bad, status):
    a = ctypes.byref(attn_args(**bad))
    assert lib.tg_tree_attention(a, P, 1 << 40, None) == status
    assert lib.tg_tree_attention_workspace(a) == 0


def test_workspaces_are_checked(lib):
    a, v = attn_args(), verify_args()
    for need, call, x in ((lib.tg_tree_attention_workspace, lib.tg_tree_attention, a),
                          (lib.tg_verify_tree_workspace, lib.tg_verify_tree, v)):
        n = need(ctypes.byref(x))
        assert n > 0
        assert call(ctypes.byref(x), P, n - 1, None) == tg.TG_ERR_WORKSPACE
        assert call(ctypes.byref(x), None, n, None) == tg.TG_ERR_WORKSPACE
        assert call(ctypes.byref(x), P + 16, n, None) == tg.TG_ERR_WORKSPACE


@pytest.mark.parametrize("bad,status", [
    (dict(B=-1), tg.TG_ERR_BAD_DIM), (dict(T=-1), tg.TG_ERR_BAD_DIM), (dict(V=0), tg.TG_ERR_BAD_DIM),
    (dict(max_path=0), tg.TG_ERR_BAD_DIM), (dict(B=5000), tg.TG_ERR_UNSUPPORTED),
    (dict(V=(1 << 24) + 1, target_stride=1 << 25, draft_stride=1 << 25), tg.TG_ERR_UNSUPPORTED),
    (dict(max_nodes=100), tg.TG_ERR_BAD_DIM), (dict(target_stride=999), tg.TG_ERR_BAD_DIM),
    (dict(draft_stride=999), tg.TG_ERR_BAD_DIM), (dict(tokens=None), tg.TG_ERR_NULL_ARG),
    (dict(target_probs=None), tg.TG_ERR_NULL_ARG), (dict(n_out=None), tg.TG_ERR_NULL_ARG)])
def test_verify_tree_refuses(lib, bad, status):
    a = ctypes.byref(verify_args(**bad))
    assert lib.tg_verify_tree(a, P, 1 << 40, None) == status
    assert lib.tg_verify_tree_workspace(a) == 0


def test_page_calls_refuse(lib):
    c = ctypes.byref(cache())
    assert lib.tg_kv_compact(c, P, 0, P, P, 2 * P, None) == tg.TG_ERR_BAD_DIM
    assert lib.tg_kv_compact(c, P, 4, P, P, P, None) == tg.TG_ERR_UNSUPPORTED
    assert lib.tg_kv_compact(c, None, 4, P, P, 2 * P, None) == tg.TG_ERR_NULL_ARG
    assert lib.tg_kv_pages_reserve(c, P, P, -1, P, P, None) == tg.TG_ERR_BAD_DIM
    assert lib.tg_kv_pages_reserve(c, P, P, 4, None, P, None) == tg.TG_ERR_NULL_ARG
    assert lib.tg_kv_pages_fork(c, P, P, P, -1, P, None) == tg.TG_ERR_BAD_DIM
    assert lib.tg_kv_pages_fork(c, P, P, P, 1025, P, None) == tg.TG_ERR_UNSUPPORTED
    assert lib.tg_kv_pages_fork(c, P, None, P, 1, P, None) == tg.TG_ERR_NULL_ARG
    assert lib.tg_kv_pages_trim(c, None, None) == tg.TG_ERR_NULL_ARG
    bare = ctypes.byref(cache(held=None, refcount=None))
    assert lib.tg_kv_pages_trim(bare, P, None) == tg.TG_ERR_NULL_ARG
    assert lib.tg_kv_pages_fork(bare, P, P, P, 1, P, None) == tg.TG_ERR_NULL_ARG


def test_binding_refuses_host_and_odd_tensors():
    k = torch.zeros((1, 2, 16, 1, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensors"):
        spec.KvCache(k, k, torch.zeros((1, 2), dtype=torch.int32), i[:1], i)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        spec.KvCache(k.float(), k.float(), i, i, i)
    with pytest.raises(ValueError, match="alike"):
        spec.KvCache(k, k.half(), i, i, i)
    with pytest.raises(ValueError, match="contiguous"):
        spec.KvCache(k.transpose(2, 4), k.transpose(2, 4), i, i, i)


def test_mirrored_structs_have_the_c_layout(tmp_path):
    """Sizes and last fields' offsets, as a C compiler lays them out."""
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    pairs = (("tg_kv_cache", tg.KvCacheArgs, "refcount"), ("tg_qk_args", tg.QkArgs, "q_out"),
             ("tg_tree_attn_args", tg.TreeAttnArgs, "out"), ("tg_verify_args", tg.VerifyArgs, "n_out"))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include "tg.h"\nint main(void) {\n' + "".join(
        f'printf("%zu %zu\\n", sizeof({c}), offsetof({c}, {f}));\n' for c, _, f in pairs) + "}\n")
    subprocess.run([cc, f"-I{os.path.join(root, 'include')}", str(src), "-o", str(tmp_path / "s")],
                   check=True)
    out = subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout
    want = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert want == [(ctypes.sizeof(m), getattr(m, f).offset) for _, m, f in pairs]

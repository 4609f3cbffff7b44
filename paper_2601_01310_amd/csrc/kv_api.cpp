// C ABI of the operators around the paged KV cache: argument validation.
#include <hip/hip_runtime.h>

#include "tg.h"
#include "tg_launch.h"

namespace {

using tg::set_error;

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

tg_status done(hipError_t e, const char* where) {
  if (e != hipSuccess) return set_error(TG_ERR_HIP, "%s: %s", where, hipGetErrorString(e));
  return set_error(TG_OK, "%s", "");
}

// The cache's shape; `tables`: whether the call keeps the page counts too.
tg_status check_cache(const tg_kv_cache* c, bool tables) {
  if (!c) return set_error(TG_ERR_NULL_ARG, "cache is NULL");
  if (c->dtype != TG_BF16 && c->dtype != TG_F16)
    return set_error(TG_ERR_BAD_DIM, "dtype=%d is neither TG_BF16 nor TG_F16", c->dtype);
  if (c->n_layers <= 0 || c->n_pages <= 0 || c->page_size <= 0 || c->Hkv <= 0 || c->B < 0 ||
      c->max_pages <= 0)
    return set_error(TG_ERR_BAD_DIM,
                     "n_layers=%d, n_pages=%d, page_size=%d, Hkv=%d, max_pages=%d must be > 0, "
                     "B=%d >= 0", c->n_layers, c->n_pages, c->page_size, c->Hkv, c->max_pages, c->B);
  if (c->D != 64 && c->D != 128 && c->D != 256)
    return set_error(TG_ERR_UNSUPPORTED, "D=%d is not 64, 128 or 256", c->D);
  if (c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return set_error(TG_ERR_UNSUPPORTED, "page_size=%d is not a power of two up to 1024",
                     c->page_size);
  if ((long long)c->n_pages * c->page_size >= (1LL << 31))
    return set_error(TG_ERR_UNSUPPORTED, "n_pages * page_size >= 2^31");
  if ((long long)c->max_pages * c->page_size > (1LL << 30))
    return set_error(TG_ERR_UNSUPPORTED, "max_pages * page_size exceeds 2^30");
  if (c->B > 4096) return set_error(TG_ERR_UNSUPPORTED, "B=%d exceeds 4096", c->B);
  if ((long long)c->B * c->max_pages >= (1LL << 31))  // pages are counted in 32 bits
    return set_error(TG_ERR_UNSUPPORTED, "B * max_pages >= 2^31");
  if (c->Hkv > 1024) return set_error(TG_ERR_UNSUPPORTED, "Hkv=%d exceeds 1024", c->Hkv);
  if (c->n_layers > 16384)  // layers of K and of V are a grid dimension
    return set_error(TG_ERR_UNSUPPORTED, "n_layers=%d exceeds 16384", c->n_layers);
  if (c->page_stride < (int64_t)c->page_size * c->Hkv * c->D)
    return set_error(TG_ERR_BAD_DIM, "page_stride=%lld is less than a page",
                     (long long)c->page_stride);
  if (c->page_stride % 8 || c->layer_stride % 8 || c->layer_stride < 0)
    return set_error(TG_ERR_UNSUPPORTED, "strides must be multiples of 8 elements, >= 0");
  if (!c->k || !c->v || (c->B > 0 && !c->page_table))
    return set_error(TG_ERR_NULL_ARG, "k, v or page_table is NULL");
  if (!aligned(c->k, 16) || !aligned(c->v, 16))
    return set_error(TG_ERR_UNSUPPORTED, "k and v must be 16-byte aligned");
  if (tables && ((c->B > 0 && !c->held) || !c->refcount))
    return set_error(TG_ERR_NULL_ARG, "held and refcount are required");
  return TG_OK;
}

tg_status check_heads(const tg_kv_cache* c, int layer, int T, int Hq) {
  if (layer < 0 || layer >= c->n_layers)
    return set_error(TG_ERR_BAD_DIM, "layer=%d is outside [0, %d)", layer, c->n_layers);
  if (T < 0) return set_error(TG_ERR_BAD_DIM, "T=%d must be >= 0", T);
  if (Hq <= 0 || Hq % c->Hkv)
    return set_error(TG_ERR_BAD_DIM, "Hq=%d must be a positive multiple of Hkv=%d", Hq, c->Hkv);
  if (Hq > 1024) return set_error(TG_ERR_UNSUPPORTED, "Hq=%d exceeds 1024", Hq);
  return TG_OK;
}

tg_status check_nodes(int max_nodes, const void* mask, int words) {
  if (max_nodes <= 0) return set_error(TG_ERR_BAD_DIM, "max_nodes=%d must be > 0", max_nodes);
  if (max_nodes > TG_MAX_NODES)
    return set_error(TG_ERR_UNSUPPORTED, "max_nodes=%d exceeds %d", max_nodes, TG_MAX_NODES);
  if (mask && (words <= 0 || words > TG_MAX_NODES / 64 || words * 64 < max_nodes))
    return set_error(TG_ERR_BAD_DIM, "mask_words=%d does not hold %d nodes", words, max_nodes);
  if (!aligned(mask, 8)) return set_error(TG_ERR_UNSUPPORTED, "tree_mask must be 8-byte aligned");
  return TG_OK;
}

tg_status check_stride(const char* name, int64_t stride, int64_t least) {
  if (stride < least)
    return set_error(TG_ERR_BAD_DIM, "%s=%lld is less than a row (%lld)", name, (long long)stride,
                     (long long)least);
  if (stride % 8) return set_error(TG_ERR_UNSUPPORTED, "%s must be a multiple of 8", name);
  return TG_OK;
}

tg_status check_qk(const tg_qk_args* a) {
  if (!a) return set_error(TG_ERR_NULL_ARG, "args is NULL");
  const tg_kv_cache* c = &a->cache;
  tg_status st = check_cache(c, false);
  if (st != TG_OK) return st;
  if ((st = check_heads(c, a->layer, a->T, a->Hq)) != TG_OK) return st;
  if (a->rot < 0 || a->rot > c->D)
    return set_error(TG_ERR_BAD_DIM, "rot=%d is outside [0, D=%d]", a->rot, c->D);
  if (a->rot % 16) return set_error(TG_ERR_UNSUPPORTED, "rot=%d is not a multiple of 16", a->rot);
  if (a->rot > 0 && a->max_pos <= 0)
    return set_error(TG_ERR_BAD_DIM, "max_pos=%d must be > 0", a->max_pos);
  if (!(a->eps >= 0.0f)) return set_error(TG_ERR_BAD_DIM, "eps must be >= 0");
  if ((st = check_stride("qkv_stride", a->qkv_stride, (int64_t)(a->Hq + 2 * c->Hkv) * c->D)) !=
      TG_OK)
    return st;
  if ((st = check_stride("q_out_stride", a->q_out_stride, (int64_t)a->Hq * c->D)) != TG_OK)
    return st;
  if (a->T > 0 &&
      (!a->qkv || !a->q_out || !a->slots || (a->rot > 0 && (!a->cos_sin || !a->positions))))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  if ((a->q_weight == nullptr) != (a->k_weight == nullptr))
    return set_error(TG_ERR_NULL_ARG, "give both q_weight and k_weight, or neither");
  if (!aligned(a->qkv, 16) || !aligned(a->q_out, 16) || !aligned(a->q_weight, 16) ||
      !aligned(a->k_weight, 16))
    return set_error(TG_ERR_UNSUPPORTED, "qkv, q_out and the weights must be 16-byte aligned");
  if (a->T > 0 && a->q_out == a->qkv && a->q_out_stride != a->qkv_stride)
    return set_error(TG_ERR_BAD_DIM, "in place, q_out_stride must be qkv_stride");
  return TG_OK;
}

tg_status check_attn(const tg_tree_attn_args* a) {
  if (!a) return set_error(TG_ERR_NULL_ARG, "args is NULL");
  const tg_kv_cache* c = &a->cache;
  tg_status st = check_cache(c, false);
  if (st != TG_OK) return st;
  if ((st = check_heads(c, a->layer, a->T, a->Hq)) != TG_OK) return st;
  if ((st = check_nodes(a->max_nodes, a->tree_mask, a->mask_words)) != TG_OK) return st;
  if ((st = check_stride("q_stride", a->q_stride, (int64_t)a->Hq * c->D)) != TG_OK) return st;
  if ((st = check_stride("out_stride", a->out_stride, (int64_t)a->Hq * c->D)) != TG_OK) return st;
  if (a->typical_nodes < 0)
    return set_error(TG_ERR_BAD_DIM, "typical_nodes=%d must be >= 0", a->typical_nodes);
  // Units of work (64 positions of 16 rows at least) are counted in 32 bits.
  const long long G = a->Hq / c->Hkv;
  const long long by_request = (long long)c->B * (a->max_nodes * G / 16 + 1);
  const long long by_row = a->T * G / 16 + c->B;
  const long long items = c->Hkv * (by_row < by_request ? by_row : by_request);
  const long long units = ((long long)c->max_pages * c->page_size + 63) / 64;
  if (items > (1LL << 30) / units - 1)
    return set_error(TG_ERR_UNSUPPORTED,
                     "Hkv * (16-row tiles of all requests) * (positions per request) / 64 >= 2^30");
  if (!(a->scale > 0.0f) || a->scale > 1e30f)
    return set_error(TG_ERR_BAD_DIM, "scale must be positive and finite");
  if ((a->T > 0 && (!a->q || !a->out)) || !a->q_offsets || (c->B > 0 && !a->lengths))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  if (!aligned(a->q, 16) || !aligned(a->out, 16))
    return set_error(TG_ERR_UNSUPPORTED, "q and out must be 16-byte aligned");
  return TG_OK;
}

tg_status check_prefix(const tg_prefix_attn_args* a) {
  if (!a) return set_error(TG_ERR_NULL_ARG, "args is NULL");
  const tg_tree_attn_args* x = &a->attn;
  const tg_status st = check_attn(x);
  if (st != TG_OK) return st;
  if (a->n_groups < 0) return set_error(TG_ERR_BAD_DIM, "n_groups=%d must be >= 0", a->n_groups);
  if (a->n_groups > 4096)
    return set_error(TG_ERR_UNSUPPORTED, "n_groups=%d exceeds 4096", a->n_groups);
  if (a->n_groups > 0 && (!a->group_offsets || !a->shared))
    return set_error(TG_ERR_NULL_ARG, "group_offsets and shared are required");
  // Threads of the join, 256 to a row, are counted in 32 bits.
  if (x->T >= 1 << 23) return set_error(TG_ERR_UNSUPPORTED, "T=%d must be below 2^23", x->T);
  // Units of the groups' work, as in check_attn.
  const long long G = x->Hq / x->cache.Hkv;
  const long long items = x->cache.Hkv * (x->T * G / 16 + a->n_groups);
  const long long units = ((long long)x->cache.max_pages * x->cache.page_size + 63) / 64;
  if (items > (1LL << 30) / units - 1)
    return set_error(TG_ERR_UNSUPPORTED,
                     "Hkv * (16-row tiles of all groups) * (positions per request) / 64 >= 2^30");
  return TG_OK;
}

tg_status check_verify(const tg_verify_args* a) {
  if (!a) return set_error(TG_ERR_NULL_ARG, "args is NULL");
  if (a->B < 0 || a->T < 0 || a->V <= 0 || a->max_path <= 0)
    return set_error(TG_ERR_BAD_DIM, "B=%d, T=%d must be >= 0, V=%d and max_path=%d > 0", a->B, a->T,
                     a->V, a->max_path);
  if (a->B > 4096) return set_error(TG_ERR_UNSUPPORTED, "B=%d exceeds 4096", a->B);
  if (a->V > (1 << 24)) return set_error(TG_ERR_UNSUPPORTED, "V=%d exceeds 2^24", a->V);
  tg_status st = check_nodes(a->max_nodes, a->tree_mask, a->mask_words);
  if (st != TG_OK) return st;
  if (a->target_stride < a->V || (a->draft_probs && a->draft_stride < a->V))
    return set_error(TG_ERR_BAD_DIM, "a row of probabilities is longer than its stride");
  if ((a->T > 0 && (!a->target_probs || !a->tokens || !a->u_accept)) || !a->q_offsets ||
      (a->B > 0 && (!a->u_next || !a->tokens_out || !a->path || !a->n_out)))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  return TG_OK;
}

tg_status check_sample(const tg_sample_args* a) {
  if (!a) return set_error(TG_ERR_NULL_ARG, "args is NULL");
  if (a->dtype != TG_F32 && a->dtype != TG_BF16 && a->dtype != TG_F16)
    return set_error(TG_ERR_BAD_DIM, "dtype=%d is neither TG_F32, TG_BF16 nor TG_F16", a->dtype);
  if (a->T < 0 || a->V <= 0)
    return set_error(TG_ERR_BAD_DIM, "T=%d must be >= 0 and V=%d > 0", a->T, a->V);
  if (a->V > (1 << 24)) return set_error(TG_ERR_UNSUPPORTED, "V=%d exceeds 2^24", a->V);
  // Threads of a grid, 512 to a block, are counted in 32 bits.
  if ((long long)a->T * ((a->V + 4095) / 4096) >= (1LL << 23))
    return set_error(TG_ERR_UNSUPPORTED, "T=%d rows of %d logits are too many", a->T, a->V);
  if (a->logits_stride < a->V || (a->probs && a->probs_stride < a->V))
    return set_error(TG_ERR_BAD_DIM, "a row of logits or probabilities is longer than its stride");
  if (a->T > 0 && (!a->logits || !a->u || !a->tokens))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  if (!aligned(a->logits, a->dtype == TG_F32 ? 4 : 2) || !aligned(a->probs, 4))
    return set_error(TG_ERR_UNSUPPORTED, "logits and probs must be aligned to their type");
  return TG_OK;
}

tg_status check_workspace(const void* ws, size_t given, size_t need) {
  if (!ws || given < need)
    return set_error(TG_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, given);
  if (!aligned(ws, 256)) return set_error(TG_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return TG_OK;
}

}  // namespace

extern "C" {

tg_status tg_qk_norm_rope(const tg_qk_args* a, void* stream) {
  const tg_status st = check_qk(a);
  if (st != TG_OK) return st;
  return done(tg::launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)), "tg_qk_norm_rope");
}

size_t tg_tree_attention_workspace(const tg_tree_attn_args* a) {
  return check_attn(a) == TG_OK ? tg::tree_attention_workspace_bytes(a) : 0;
}

tg_status tg_tree_attention(const tg_tree_attn_args* a, void* ws, size_t ws_bytes, void* stream) {
  tg_status st = check_attn(a);
  if (st != TG_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, tg::tree_attention_workspace_bytes(a))) != TG_OK) return st;
  return done(tg::launch_tree_attention(a, ws, static_cast<hipStream_t>(stream)),
              "tg_tree_attention");
}

size_t tg_prefix_attention_workspace(const tg_prefix_attn_args* a) {
  return check_prefix(a) == TG_OK ? tg::prefix_attention_workspace_bytes(a) : 0;
}

tg_status tg_prefix_attention(const tg_prefix_attn_args* a, void* ws, size_t ws_bytes,
                              void* stream) {
  tg_status st = check_prefix(a);
  if (st != TG_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, tg::prefix_attention_workspace_bytes(a))) != TG_OK)
    return st;
  return done(tg::launch_prefix_attention(a, ws, static_cast<hipStream_t>(stream)),
              "tg_prefix_attention");
}

size_t tg_verify_tree_workspace(const tg_verify_args* a) {
  return check_verify(a) == TG_OK ? tg::verify_workspace_bytes(a) : 0;
}

tg_status tg_verify_tree(const tg_verify_args* a, void* ws, size_t ws_bytes, void* stream) {
  tg_status st = check_verify(a);
  if (st != TG_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, tg::verify_workspace_bytes(a))) != TG_OK) return st;
  return done(tg::launch_verify_tree(a, ws, static_cast<hipStream_t>(stream)), "tg_verify_tree");
}

size_t tg_sample_workspace(const tg_sample_args* a) {
  return check_sample(a) == TG_OK ? tg::sample_workspace_bytes(a) : 0;
}

tg_status tg_sample(const tg_sample_args* a, void* ws, size_t ws_bytes, void* stream) {
  tg_status st = check_sample(a);
  if (st != TG_OK) return st;
  if ((st = check_workspace(ws, ws_bytes, tg::sample_workspace_bytes(a))) != TG_OK) return st;
  return done(tg::launch_sample(a, ws, static_cast<hipStream_t>(stream)), "tg_sample");
}

tg_status tg_kv_compact(const tg_kv_cache* c, const int32_t* path, int max_path,
                        const int32_t* n_keep, const int32_t* lengths, int32_t* new_lengths,
                        void* stream) {
  const tg_status st = check_cache(c, false);
  if (st != TG_OK) return st;
  if (max_path <= 0) return set_error(TG_ERR_BAD_DIM, "max_path=%d must be > 0", max_path);
  if (c->B > 0 && (!path || !n_keep || !lengths || !new_lengths))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  if (c->B > 0 && lengths == new_lengths)
    return set_error(TG_ERR_UNSUPPORTED, "new_lengths must be another array than lengths");
  return done(tg::launch_kv_compact(c, path, max_path, n_keep, lengths, new_lengths,
                                    static_cast<hipStream_t>(stream)), "tg_kv_compact");
}

tg_status tg_kv_pages_reserve(const tg_kv_cache* c, const int32_t* lengths,
                              const int32_t* q_offsets, int T, int32_t* slots, int32_t* status,
                              void* stream) {
  const tg_status st = check_cache(c, true);
  if (st != TG_OK) return st;
  if (T < 0) return set_error(TG_ERR_BAD_DIM, "T=%d must be >= 0", T);
  if (!q_offsets || (c->B > 0 && (!lengths || !status)) || (T > 0 && !slots))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  return done(tg::launch_kv_pages_reserve(c, lengths, q_offsets, T, slots, status,
                                          static_cast<hipStream_t>(stream)), "tg_kv_pages_reserve");
}

tg_status tg_kv_pages_fork(const tg_kv_cache* c, int32_t* lengths, const int32_t* src,
                           const int32_t* dst, int n, int32_t* status, void* stream) {
  const tg_status st = check_cache(c, true);
  if (st != TG_OK) return st;
  if (n < 0) return set_error(TG_ERR_BAD_DIM, "n=%d must be >= 0", n);
  if (n > TG_MAX_FORKS) return set_error(TG_ERR_UNSUPPORTED, "n=%d exceeds %d", n, TG_MAX_FORKS);
  if (n > 0 && (!lengths || !src || !dst || !status))
    return set_error(TG_ERR_NULL_ARG, "a required pointer is NULL");
  return done(tg::launch_kv_pages_fork(c, lengths, src, dst, n, status,
                                       static_cast<hipStream_t>(stream)), "tg_kv_pages_fork");
}

tg_status tg_kv_pages_trim(const tg_kv_cache* c, const int32_t* keep, void* stream) {
  const tg_status st = check_cache(c, true);
  if (st != TG_OK) return st;
  if (c->B > 0 && !keep) return set_error(TG_ERR_NULL_ARG, "keep is NULL");
  return done(tg::launch_kv_pages_trim(c, keep, static_cast<hipStream_t>(stream)),
              "tg_kv_pages_trim");
}

}  // extern "C"

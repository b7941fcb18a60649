// extern "C" entry points of latent attention: argument validation and dispatch.  See include/tq.h.
#include <initializer_list>

#include "tq_latent.cuh"

namespace tq {
namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool is16(int dtype) { return dtype == TQ_FP16 || dtype == TQ_BF16; }

// The requirements of tq_kv_cache, with one KV head.
int check_latent(const tq_latent_cache* c) {
  if (!c) return TQ_ERR_NULL;
  const tq_kv_cache same = {c->blocks, c->seq_lens, c->B, 1, c->S_cap, 128, c->page_table, c->page_tokens, c->max_pages, c->num_pages};
  if (int r = check_cache(&same)) return r;
  return c->d_c == 128 || c->d_c == 256 || c->d_c == 512 ? TQ_OK : TQ_ERR_SHAPE;
}

int check_heads_of(const tq_heads* x, int64_t width) {
  // (2^39: what a tensor map can describe)
  for (const int64_t s : {x->row_stride, x->head_stride})
    if (s < width || s % 8 || s >= 1LL << 39) return TQ_ERR_SHAPE;
  return TQ_OK;
}

}  // namespace
}  // namespace tq

using namespace tq;

extern "C" {

size_t tq_cache_latent_code_offset(int32_t d_c, int32_t t, int32_t c) { return static_cast<size_t>(latent_code_offset(d_c, t, c)); }

size_t tq_cache_latent_bytes(int32_t B, int32_t S_cap, int32_t d_c) {
  if (B < 1 || S_cap < 1 || d_c < 1) return 0;
  return static_cast<size_t>(B) * ((static_cast<size_t>(S_cap) + 15) / 16) * TQ_BLOCK_LATENT_BYTES(d_c);
}

int tq_latent_append(const tq_latent_cache* cache, const void* c_new, const void* r_new, int32_t dtype, int64_t c_stride,
                     int64_t r_stride, const int64_t* slots, int64_t n, int32_t* status, void* stream) {
  if (int r = check_latent(cache)) return r;
  if (n == 0) return TQ_OK;
  if (!c_new || !r_new || !slots) return TQ_ERR_NULL;
  if (!is16(dtype) || n < 1 || n > 0x7fffffffLL || c_stride < cache->d_c || r_stride < kRope || c_stride % 8 || r_stride % 8)
    return TQ_ERR_SHAPE;
  if (!aligned(c_new, 16) || !aligned(r_new, 16) || !aligned(slots, 8) || !aligned(status, 4)) return TQ_ERR_ALIGN;
  return finish(launch_latent_append(*cache, c_new, r_new, dtype, c_stride, r_stride, slots, n, status, static_cast<cudaStream_t>(stream)));
}

int tq_latent_gather(const tq_latent_cache* cache, const int64_t* slots, int64_t n, void* c_out, void* r_out, int32_t dtype,
                     int32_t* status, void* stream) {
  if (int r = check_latent(cache)) return r;
  if (n == 0) return TQ_OK;
  if (!slots || !c_out || !r_out) return TQ_ERR_NULL;
  if ((!is16(dtype) && dtype != TQ_FP32) || n < 1 || n > 0x7fffffffLL) return TQ_ERR_SHAPE;
  if (!aligned(c_out, 16) || !aligned(r_out, 16) || !aligned(slots, 8) || !aligned(status, 4)) return TQ_ERR_ALIGN;
  return finish(launch_latent_gather(*cache, slots, n, c_out, r_out, dtype, status, static_cast<cudaStream_t>(stream)));
}

size_t tq_latent_workspace_bytes(int32_t B, int32_t H, int32_t d_c) {
  if (B < 1 || H < 1 || H > 1024 || d_c < 1) return 0;
  return latent_workspace_bytes(B, H, d_c);
}

int tq_sdpa_latent_decode(const tq_latent_cache* cache, const tq_heads* q_c, const tq_heads* q_r, int32_t q_dtype, int32_t H,
                          float attn_scale, int32_t window, int32_t max_seq_len, void* workspace, size_t workspace_bytes, void* out,
                          int32_t out_dtype, int32_t* status, void* stream) {
  if (int r = check_latent(cache)) return r;
  if (!q_c || !q_r || !q_c->data || !q_r->data || !workspace || !out) return TQ_ERR_NULL;
  if (H < 1 || H > 1024 || !is16(q_dtype) || (out_dtype != q_dtype && out_dtype != TQ_FP32) || window < 0 || max_seq_len < 0)
    return TQ_ERR_SHAPE;
  if (static_cast<int64_t>(cache->B) * ((H + 63) / 64) * (cache->S_cap / 64 + 8) > 1LL << 30) return TQ_ERR_SHAPE;
  if (int r = check_heads_of(q_c, cache->d_c)) return r;
  if (int r = check_heads_of(q_r, kRope)) return r;
  if (!aligned(q_c->data, 16) || !aligned(q_r->data, 16) || !aligned(workspace, 16) || !aligned(out, 16) || !aligned(status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_latent_workspace_bytes(cache->B, H, cache->d_c)) return TQ_ERR_WORKSPACE;
  int most = max_seq_len && max_seq_len < cache->S_cap ? max_seq_len : cache->S_cap;
  if (window && window < most) most = window;
  const LatentArgs a = {*cache, *q_c, *q_r, q_dtype, H, attn_scale, window, most, workspace, out, out_dtype, status};
  return finish(launch_latent_decode(a, static_cast<cudaStream_t>(stream)));
}

int tq_sdpa_latent_prompt(const tq_heads* q_n, const tq_heads* q_r, const tq_heads* k_n, const void* k_r, int64_t kr_stride,
                          const tq_heads* v, int32_t dtype, int32_t n_q, int32_t n_kv, const int32_t* q_offsets,
                          const int32_t* kv_offsets, int32_t B, int32_t H, int32_t d, float attn_scale, int32_t causal,
                          int32_t window, void* out, int32_t out_dtype, int32_t* status, void* stream) {
  if (!q_n || !q_r || !k_n || !v) return TQ_ERR_NULL;
  if (n_q > 0 && (!q_n->data || !q_r->data || !out || (n_kv > 0 && (!k_n->data || !k_r || !v->data)))) return TQ_ERR_NULL;
  if (!q_offsets || !kv_offsets) return TQ_ERR_NULL;
  if (B < 1 || B > 65535 || H < 1 || H > 4096 || !(d == 64 || d == 128) || n_q < 0 || n_kv < 0) return TQ_ERR_SHAPE;
  if (!is16(dtype) || (out_dtype != dtype && out_dtype != TQ_FP32) || window < 0 || (window > 0 && !causal)) return TQ_ERR_SHAPE;
  if (int r = check_heads_of(q_n, d)) return r;
  if (int r = check_heads_of(q_r, kRope)) return r;
  if (int r = check_heads_of(k_n, d)) return r;
  if (int r = check_heads_of(v, d)) return r;
  if (kr_stride < kRope || kr_stride % 8 || kr_stride >= 1LL << 39) return TQ_ERR_SHAPE;
  if (!aligned(q_n->data, 16) || !aligned(q_r->data, 16) || !aligned(k_n->data, 16) || !aligned(k_r, 16) || !aligned(v->data, 16) ||
      !aligned(out, 16) || !aligned(q_offsets, 4) || !aligned(kv_offsets, 4) || !aligned(status, 4))
    return TQ_ERR_ALIGN;
  if (n_q == 0) return TQ_OK;
  PromptArgs a = {};
  a.q = q_n->data;
  a.k = k_n->data;
  a.v = v->data;
  a.dtype = dtype;
  a.q_stride = q_n->row_stride;
  a.k_stride = k_n->row_stride;
  a.v_stride = v->row_stride;
  a.q_head = q_n->head_stride;
  a.k_head = k_n->head_stride;
  a.v_head = v->head_stride;
  a.q_r = q_r->data;
  a.k_r = k_r;
  a.qr_stride = q_r->row_stride;
  a.qr_head = q_r->head_stride;
  a.kr_stride = kr_stride;
  a.n_q = n_q;
  a.n_kv = n_kv;
  a.q_offsets = q_offsets;
  a.kv_offsets = kv_offsets;
  a.B = B;
  a.H_q = a.H_kv = H;
  a.d = d;
  a.attn_scale = attn_scale;
  a.causal = causal != 0;
  a.window = window;
  a.out = out;
  a.out_dtype = out_dtype;
  a.status = status;
  return finish(launch_prompt(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

// extern "C" entry points of the serving operators: argument validation and dispatch.  See include/tq.h.
#include "tq_kv8.cuh"

namespace tq {
namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool is16(int dtype) { return dtype == TQ_FP16 || dtype == TQ_BF16; }

// The requirements of tq_kv_cache, which the 8-bit cache shares.
int check_cache8(const tq_kv8_cache* c) {
  if (!c) return TQ_ERR_NULL;
  const tq_kv_cache same = {c->blocks,     c->seq_lens,    c->B,         c->H_kv,     c->S_cap, c->d,
                            c->page_table, c->page_tokens, c->max_pages, c->num_pages};
  return check_cache(&same);
}

int check_pages(const int32_t* page_table, int B, int page_tokens, int max_pages, int num_pages) {
  if (B < 1 || B > 65535 || page_tokens < 16 || max_pages < 1 || static_cast<long long>(page_tokens) * max_pages > 0x7fffffffLL)
    return TQ_ERR_SHAPE;
  if (page_table ? (page_tokens & (page_tokens - 1)) != 0 || num_pages < 1 : page_tokens % 16 != 0) return TQ_ERR_SHAPE;
  return TQ_OK;
}

}  // namespace
}  // namespace tq

using namespace tq;

extern "C" {

int tq_pages_release(const int32_t* page_table, const int32_t* seq_lens, const uint8_t* finished, int32_t B,
                     int32_t page_tokens, int32_t max_pages, int32_t num_pages, int32_t* free_pages,
                     const int32_t* free_count, int32_t* seq_lens_out, int32_t* free_count_out, int32_t* status,
                     void* stream) {
  if (!seq_lens || !finished || !seq_lens_out) return TQ_ERR_NULL;
  if (page_table && (!free_pages || !free_count || !free_count_out)) return TQ_ERR_NULL;
  if (int r = check_pages(page_table, B, page_tokens, max_pages, num_pages)) return r;
  if (!aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(free_pages, 4) || !aligned(free_count, 4) ||
      !aligned(seq_lens_out, 4) || !aligned(free_count_out, 4) || !aligned(status, 4))
    return TQ_ERR_ALIGN;
  PageArgs a = {};
  a.page_table = const_cast<int32_t*>(page_table);
  a.seq_lens = seq_lens;
  a.B = B;
  a.page_tokens = page_tokens;
  a.max_pages = max_pages;
  a.num_pages = num_pages;
  a.free_count = free_count;
  a.seq_lens_out = seq_lens_out;
  a.free_count_out = free_count_out;
  return finish(launch_pages_release(a, finished, free_pages, status, static_cast<cudaStream_t>(stream)));
}

size_t tq_pages_workspace_bytes(int32_t B) { return B < 1 ? 0 : 8 * (static_cast<size_t>(B) + 1); }

int tq_pages_assign(int32_t* page_table, const int32_t* seq_lens, const int32_t* new_lens, int32_t B, int32_t page_tokens,
                    int32_t max_pages, int32_t num_pages, const int32_t* free_pages, const int32_t* free_count,
                    int32_t* seq_lens_out, int32_t* free_count_out, int32_t* token_offsets, int64_t* slots,
                    int64_t n_slots, void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  if (!seq_lens || !new_lens || !seq_lens_out || !token_offsets || (!slots && n_slots > 0) || !workspace) return TQ_ERR_NULL;
  if (page_table && (!free_pages || !free_count || !free_count_out)) return TQ_ERR_NULL;
  if (int r = check_pages(page_table, B, page_tokens, max_pages, num_pages)) return r;
  if (n_slots < 0 || n_slots > 0x7fffffffLL) return TQ_ERR_SHAPE;
  if (!aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(new_lens, 4) || !aligned(free_pages, 4) ||
      !aligned(free_count, 4) || !aligned(seq_lens_out, 4) || !aligned(free_count_out, 4) || !aligned(token_offsets, 4) ||
      !aligned(slots, 8) || !aligned(workspace, 16) || !aligned(status, 4))
    return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_pages_workspace_bytes(B)) return TQ_ERR_WORKSPACE;
  const PageArgs a = {page_table, seq_lens,   new_lens,     B,              page_tokens,   max_pages, num_pages,
                      free_pages, free_count, seq_lens_out, free_count_out, token_offsets, slots,     n_slots};
  return finish(launch_pages_assign(a, static_cast<int32_t*>(workspace), status, static_cast<cudaStream_t>(stream)));
}

size_t tq_cache8_code_offset(int32_t d, int32_t which, int32_t t, int32_t c) {
  return static_cast<size_t>(which ? v8_offset(d, t, c) : k8_offset(t, c));
}

size_t tq_cache8_bytes(int32_t B, int32_t H_kv, int32_t S_cap, int32_t d) {
  if (B < 1 || H_kv < 1 || S_cap < 1 || d < 1) return 0;
  return static_cast<size_t>(B) * H_kv * ((static_cast<size_t>(S_cap) + 15) / 16) * TQ_BLOCK8_BYTES(d);
}

int tq_kv8_append(const tq_kv8_cache* cache, const void* k_new, const void* v_new, int32_t dtype, int64_t k_stride,
                  int64_t v_stride, const int64_t* slots, int64_t n, int32_t* status, void* stream) {
  if (int r = check_cache8(cache)) return r;
  if (n == 0) return TQ_OK;
  if (!k_new || !v_new || !slots) return TQ_ERR_NULL;
  const int64_t row = static_cast<int64_t>(cache->H_kv) * cache->d;
  if (!is16(dtype) || n < 1 || n > 0x7fffffffLL || k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8)
    return TQ_ERR_SHAPE;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 8) || !aligned(status, 4)) return TQ_ERR_ALIGN;
  return finish(launch_kv8_append(*cache, k_new, v_new, dtype, k_stride, v_stride, slots, n, status,
                                  static_cast<cudaStream_t>(stream)));
}

int tq_kv8_gather(const tq_kv8_cache* cache, const int64_t* slots, int64_t n, void* k_out, void* v_out, int32_t dtype,
                  int32_t* status, void* stream) {
  if (int r = check_cache8(cache)) return r;
  if (n == 0) return TQ_OK;
  if (!slots || !k_out || !v_out) return TQ_ERR_NULL;
  if ((!is16(dtype) && dtype != TQ_FP32) || n < 1 || n > 0x7fffffffLL) return TQ_ERR_SHAPE;
  if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(slots, 8) || !aligned(status, 4)) return TQ_ERR_ALIGN;
  return finish(launch_kv8_gather(*cache, slots, n, k_out, v_out, dtype, status, static_cast<cudaStream_t>(stream)));
}

size_t tq_int8_counter_bytes(int32_t B, int32_t H_kv, int32_t H_q) {
  if (B < 1 || H_kv < 1 || H_q < H_kv) return 0;
  return kCounterBytes;
}

size_t tq_int8_workspace_bytes(int32_t B, int32_t H_kv, int32_t H_q, int32_t d) {
  if (B < 1 || H_kv < 1 || H_q < H_kv || d < 1) return 0;
  return tq_int8_counter_bytes(B, H_kv, H_q) + decode8_parts_bytes(B, H_kv, H_q / H_kv, d);
}

int tq_sdpa_int8_decode(const tq_kv8_cache* cache, const void* q, int32_t q_dtype, int64_t q_stride, int32_t H_q,
                        float attn_scale, int32_t window, int32_t max_seq_len, void* workspace, size_t workspace_bytes,
                        void* out, int32_t out_dtype, int32_t* status, void* stream) {
  if (int r = check_cache8(cache)) return r;
  if (!q || !workspace || !out) return TQ_ERR_NULL;
  if (H_q < 1 || H_q % cache->H_kv != 0 || H_q / cache->H_kv > 64) return TQ_ERR_SHAPE;
  // (positions on the line, see tq_decode8.cu, are 31 bits)
  if (static_cast<int64_t>(cache->B) * cache->H_kv * ((H_q / cache->H_kv + 7) / 8) * (cache->S_cap / 16 + 64) > 0x7fff0000LL)
    return TQ_ERR_SHAPE;
  if (!is16(q_dtype) || (out_dtype != q_dtype && out_dtype != TQ_FP32) || window < 0 || max_seq_len < 0 ||
      q_stride < static_cast<int64_t>(H_q) * cache->d || q_stride % 8)
    return TQ_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(workspace, 16) || !aligned(out, 16) || !aligned(status, 4)) return TQ_ERR_ALIGN;
  if (workspace_bytes < tq_int8_workspace_bytes(cache->B, cache->H_kv, H_q, cache->d)) return TQ_ERR_WORKSPACE;
  int most = max_seq_len && max_seq_len < cache->S_cap ? max_seq_len : cache->S_cap;
  if (window && window < most) most = window;
  const int grid = decode8_grid(cache->B, cache->H_kv, H_q / cache->H_kv, cache->d, most);
  auto* counters = static_cast<uint32_t*>(workspace);
  auto* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes);
  return finish(launch_decode8(*cache, q, q_dtype, q_stride, H_q, attn_scale, window, grid, counters, parts, out, out_dtype,
                               status, static_cast<cudaStream_t>(stream)));
}

int tq_sdpa_prompt(const void* q, const void* k, const void* v, int32_t dtype, int64_t q_stride, int64_t k_stride,
                   int64_t v_stride, int32_t n_q, int32_t n_kv, const int32_t* q_offsets, const int32_t* kv_offsets,
                   int32_t B, int32_t H_q, int32_t H_kv, int32_t d, float attn_scale, int32_t causal, int32_t window,
                   void* out, int32_t out_dtype, int32_t* status, void* stream) {
  if (n_q > 0 && (!q || !out || (n_kv > 0 && (!k || !v)))) return TQ_ERR_NULL;
  if (!q_offsets || !kv_offsets) return TQ_ERR_NULL;
  if (B < 1 || B > 65535 || H_kv < 1 || H_kv > 4096 || H_q < 1 || H_q % H_kv != 0 || H_q / H_kv > 64) return TQ_ERR_SHAPE;
  if (!(d == 64 || d == 128 || d == 256 || d == 512) || n_q < 0 || n_kv < 0) return TQ_ERR_SHAPE;
  if (!is16(dtype) || (out_dtype != dtype && out_dtype != TQ_FP32) || window < 0 || (window > 0 && !causal)) return TQ_ERR_SHAPE;
  const int64_t rq = static_cast<int64_t>(H_q) * d, rk = static_cast<int64_t>(H_kv) * d;
  if (q_stride < rq || k_stride < rk || v_stride < rk || q_stride % 8 || k_stride % 8 || v_stride % 8) return TQ_ERR_SHAPE;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(q_offsets, 4) ||
      !aligned(kv_offsets, 4) || !aligned(status, 4))
    return TQ_ERR_ALIGN;
  if (n_q == 0) return TQ_OK;
  const PromptArgs a = {q, k, v, dtype, q_stride, k_stride, v_stride, n_q, n_kv, q_offsets, kv_offsets, B, H_q, H_kv, d,
                        attn_scale, causal != 0, window, out, out_dtype, status};
  return finish(launch_prompt(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

// The 8-bit block of 16 tokens of one KV head (tq.h: TQ_BLOCK8_BYTES), its byte order and the exact quantiser.
//
// Byte order.  The decode kernel feeds mma.m16n8k16 with codes straight from shared memory, so a block stores them in
// the order of that instruction's A fragments: lane 4 g + t of a warp owns 16 consecutive bytes, and the 32 lanes of
// a warp read 512 consecutive bytes (one 128-bit load each, no bank conflicts) that are the A operand of
//   K: 16 tokens x 32 channels (two k = 16 steps):  tokens g and g + 8, channels 32 kk + 8 t .. + 7,
//   V: 32 channels x 16 tokens (two m = 16 tiles):  channels 32 kk + 8 i + g (i = 0 .. 3), tokens 2t, 2t+1, 2t+8, 2t+9.
// A code is stored as code + 128 in an unsigned byte: prmt makes the fp16 number 1024 + byte of it, and one packed
// subtraction of 1152 the exact code.
//
// Quantiser.  A block keeps the range a = max |x| itself, not a / 127: with x and a of at most 11 significant bits the
// products 127 x and c a_old are exact in binary32, and of such a quotient u / a one correctly rounded division cannot
// land on the other side of a half: u / a = k + 1/2 exactly is computed exactly, and otherwise |u / a - (k + 1/2)| >=
// ulp(x) / (2 a) >= (u / a) / 127 / 2^12 -- 1.9e-6 of the quotient, against 6e-8 of rounding.  So every code is
// round_half_even of the true quotient.
#pragma once
#include <cuda_bf16.h>

#include "tq_internal.cuh"

namespace tq {

__host__ __device__ constexpr int block8_bytes(int d) { return 32 * d + 16; }
__host__ __device__ constexpr int k8_offset(int token, int c) {
  return 512 * (c >> 5) + 64 * (token & 7) + 16 * ((c & 31) >> 3) + 8 * (token >> 3) + (c & 7);
}
__host__ __device__ constexpr int v8_offset(int d, int token, int c) {
  return 16 * d + 512 * (c >> 5) + 64 * (c & 7) + 16 * ((token & 7) >> 1) + 4 * ((c & 31) >> 3) + 2 * (token >> 3) + (token & 1);
}
__host__ __device__ constexpr int range8_offset(int d, int which) { return 32 * d + 4 * which; }

// Two 16-bit values of a word as floats, by type.
template <int DT>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if (DT == TQ_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Two floats rounded to nearest even into a word, by type.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if (DT == TQ_BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// What the quantiser makes of a value that is no number or no finite one: 0, or the largest finite value of the type.
template <int DT>
__device__ __forceinline__ float finite8(float x) {
  constexpr float top = DT == TQ_BF16 ? 3.38953139e38f : 65504.0f;
  if (x != x) return 0.0f;
  return fminf(fmaxf(x, -top), top);
}

// The divisor and the factor that make a code of a value: round(x * mul / div).  127 * x would leave binary32 for
// ranges near its top; both sides are scaled by 2^-32 there, exactly for every x that is not 0 after it anyway.
struct Div8 {
  float div, mul;
};
__device__ __forceinline__ Div8 div8(float a) {
  if (a > 1.0e30f) return {a * 2.3283064365386963e-10f, 2.3283064365386963e-10f};
  return {a > 0.0f ? a : 1.0f, 1.0f};
}
__device__ __forceinline__ int code8(float x, Div8 q) {
  return __float2int_rn(__fdiv_rn(__fmul_rn(__fmul_rn(x, q.mul), 127.0f), q.div));
}
// an older code under the range a_old, under the new one
__device__ __forceinline__ int recode8(int c, float a_old, Div8 q) {
  return __float2int_rn(__fdiv_rn(__fmul_rn(__int2float_rn(c), __fmul_rn(a_old, q.mul)), q.div));
}

// Slots of one call (append and gather).  A slot is page * page_tokens + position in the page (contiguous: sequence *
// S_cap + position), -1 marks a padding row.
struct Slots8 {
  const int64_t* slots;
  long long n;      // rows
  long long limit;  // slots of the cache
};
// 16-token block of KV head h that slot s (valid) falls into
__device__ __forceinline__ uint8_t* block8_of(const tq_kv8_cache& c, int64_t s, int h) {
  const int page_tokens = c.page_table ? c.page_tokens : c.S_cap;
  const long long page = c.page_table ? s >> (__ffs(page_tokens) - 1) : s / page_tokens;
  const int bpp = page_tokens >> 4;
  const int j = static_cast<int>(s - page * page_tokens) >> 4;
  return c.blocks + ((page * c.H_kv + h) * bpp + j) * block8_bytes(c.d);
}

}  // namespace tq

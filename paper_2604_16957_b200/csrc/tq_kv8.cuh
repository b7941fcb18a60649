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
// round_half_even of the true quotient.  The division is Markstein's: with r the rounded reciprocal of a, q = u r and
// the exact remainder u - q a (one fused operation), q + r (u - q a) is the correctly rounded quotient; three packed
// instructions for two values instead of a division sequence for each.
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
__device__ __forceinline__ uint32_t finite8(uint32_t w) {
  constexpr uint32_t inf = DT == TQ_BF16 ? 0x7f80u : 0x7c00u;
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t x = (w >> (16 * i)) & 0xffffu, mag = x & 0x7fffu;
    out |= (mag > inf ? 0u : (mag == inf ? x - 1 : x)) << (16 * i);
  }
  return out;
}

// ---- two fp32 values in a 64-bit register: one instruction for both
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 unpair(uint64_t r) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;\n" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Division by the range a.  Everything is scaled by a power of two that brings a into [1, 4) -- 2^-126 to 2^120, which
// leaves the smallest ranges of bf16 at 2^-13 --, so that nothing overflows or loses digits; a value that this makes
// subnormal has the code 0 anyway.
struct Div8 {
  float scale;  // that power of two
  uint64_t div, rcp;  // a * scale and its rounded reciprocal, twice each
  __device__ explicit Div8(float a) {
    const int e = static_cast<int>(__float_as_uint(a) >> 23);  // biased exponent; 0 for 0 and subnormals
    scale = __uint_as_float(static_cast<uint32_t>(a > 0.0f ? min(max(254 - e, 1), 247) : 127) << 23);
    const float d = a > 0.0f ? __fmul_rn(a, scale) : 1.0f;
    const float r = __fdiv_rn(1.0f, d);
    div = pair(-d, -d);
    rcp = pair(r, r);
  }
  // stored codes (low bytes of the two words) of two exact products u (already scaled)
  __device__ __forceinline__ uint64_t codes(uint64_t u) const {
    constexpr float kMagic = 12582912.0f + 128.0f;  // 1.5 * 2^23 rounds to an integer, half to even; + 128 as stored
    const uint64_t q = mul2(u, rcp);
    const uint64_t exact = fma2(fma2(q, div, u), rcp, q);
    return add2(exact, pair(kMagic, kMagic));
  }
};
__device__ __forceinline__ uint32_t low_bytes(uint64_t a, uint64_t b) {  // of four fp32 words
  const float2 x = unpair(a), y = unpair(b);
  return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040),
                     __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
}
// bytes 2i, 2i + 1 of a word of stored codes as two exact fp32 codes
__device__ __forceinline__ uint64_t codes_of(uint32_t w, int i) {
  const uint32_t lo = __byte_perm(w, 0x4b000000u, i ? 0x7442 : 0x7440), hi = __byte_perm(w, 0x4b000000u, i ? 0x7443 : 0x7441);
  return add2(pair(__uint_as_float(lo), __uint_as_float(hi)), pair(-8388736.0f, -8388736.0f));  // 2^23 + 128
}
// 4 x 4 bytes turned around: byte i of out[j] = byte j of w[i]
__device__ __forceinline__ void turn4(uint32_t (&w)[4]) {
  const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[0], w[1], 0x7362);
  const uint32_t c = __byte_perm(w[2], w[3], 0x5140), d = __byte_perm(w[2], w[3], 0x7362);
  w[0] = __byte_perm(a, c, 0x5410);
  w[1] = __byte_perm(a, c, 0x7632);
  w[2] = __byte_perm(b, d, 0x5410);
  w[3] = __byte_perm(b, d, 0x7632);
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

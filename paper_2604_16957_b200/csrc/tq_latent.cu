// Append to and gather from the latent cache, through slots (tq_pages_assign writes them).
//
// A token is d_c codes with one range, 64 positional channels in fp16 with a power of two, and the two scales: d_c / 16
// lanes of a warp hold it, 16 codes each (one 16-byte load of the cache's order, two of the rows'), so that a range is
// one reduction over those lanes and every byte is touched once.  Tokens do not depend on one another: any order of slots
// will do.
//
// The codes are exact roundings of the true quotients (the division by the range is that of the 8-bit cache, see
// tq_kv8.cuh).  Bound by HBM for prompts: 74 K tokens of d_c = 512 are 133 MB each way, 20 us at the copy rate; append and gather
// take 51 us together.  A decode step's is two dependent memory latencies.  The positional key keeps its digits: multiplied by
// a power of two that brings the largest magnitude into [2^15, 2^16) it is exact in fp16 but for bf16 channels below 2^-32 of the
// largest, which are off by 2^-40 of it.
#include "tq_latent.cuh"

namespace tq {
namespace {

constexpr int kWarps = 8;

// What is held of two 16-bit values that are no numbers, not finite, or beyond 2^64 in magnitude (bf16).
template <int DT>
__device__ __forceinline__ uint32_t held2(uint32_t w) {
  constexpr uint32_t inf = DT == TQ_BF16 ? 0x7f80u : 0x7c00u, most = DT == TQ_BF16 ? 0x5f80u : 0x7bffu;
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t x = (w >> (16 * i)) & 0xffffu, mag = x & 0x7fffu;
    out |= (mag > inf ? 0u : ((x & 0x8000u) | min(mag, most))) << (16 * i);
  }
  return out;
}
template <int DT>
__device__ __forceinline__ uint32_t top2(uint32_t top, const uint4& v) {  // magnitudes as integers, two to a word
  return __vmaxu2(__vmaxu2(top, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu)), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
}
// Values of a word of which one is beyond what is held (`top`: the largest magnitudes seen)
template <int DT>
__device__ __forceinline__ bool beyond(uint32_t top) {
  constexpr uint32_t most = DT == TQ_BF16 ? 0x5f80u : 0x7bffu;
  return max(top & 0xffffu, top >> 16) > most;
}
template <int DT>
__device__ __forceinline__ void hold(uint4& v) {
  v = make_uint4(held2<DT>(v.x), held2<DT>(v.y), held2<DT>(v.z), held2<DT>(v.w));
}
template <int DT>
__device__ __forceinline__ float largest(uint32_t top) {
  return unpack2<DT>(max(top & 0xffffu, top >> 16)).x;
}

// A token's codes, positional key and scales from the values that its lanes hold; the whole warp comes here.
template <int DC, int DT>
__device__ __forceinline__ void append_token(const tq_latent_cache& c, int64_t slot, uint4 (&x)[2], uint4& r, int sub) {
  constexpr int LANES = DC / 16;
  uint32_t top = top2<DT>(top2<DT>(0, x[0]), x[1]), rtop = top2<DT>(0, r);
  if (beyond<DT>(top) || beyond<DT>(rtop)) {
    hold<DT>(x[0]);
    hold<DT>(x[1]);
    hold<DT>(r);
    top = top2<DT>(top2<DT>(0, x[0]), x[1]);
    rtop = top2<DT>(0, r);
  }
#pragma unroll
  for (int off = LANES / 2; off > 0; off >>= 1) {
    top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, off));
    rtop = __vmaxu2(rtop, __shfl_xor_sync(0xffffffffu, rtop, off));
  }
  if (slot < 0) return;
  float range = largest<DT>(top);
  if (range < 5.421010862427522e-20f) range = 0.0f;  // 2^-64
  uint8_t* const blk = c.blocks + (slot >> 4) * latent_block_bytes(DC);
  const int t = static_cast<int>(slot & 15);
  uint4 codes = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
  if (range > 0.0f) {
    const Div8 q(range);
    const float m = __fmul_rn(q.scale, 127.0f);
    const uint64_t mul = pair(m, m);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float2 f = unpack2<DT>(v[2 * h]), g = unpack2<DT>(v[2 * h + 1]);
        out[2 * i + h] = low_bytes(q.codes(mul2(pair(f.x, f.y), mul)), q.codes(mul2(pair(g.x, g.y), mul)));
      }
    }
    codes = make_uint4(out[0], out[1], out[2], out[3]);
  }
  *reinterpret_cast<uint4*>(blk + DC * t + 16 * sub) = codes;
  const float most = largest<DT>(rtop);
  // exponent of the power of two: that of the largest magnitude, less 15; 0 where all are zero
  const int e = most > 0.0f ? max(static_cast<int>(__float_as_uint(most) >> 23) - 127 - 15, -126) : 0;
  if (sub < 8) {
    const float up = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    const uint32_t v[4] = {r.x, r.y, r.z, r.w};
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack2<DT>(v[i]);
      out[i] = pack2<TQ_FP16>(__fmul_rn(f.x, up), __fmul_rn(f.y, up));
    }
    *reinterpret_cast<uint4*>(blk + latent_rope_offset(DC, t) + 16 * sub) = make_uint4(out[0], out[1], out[2], out[3]);
  }
  if (sub == 0)
    *reinterpret_cast<float2*>(blk + latent_scale_offset(DC, t)) = make_float2(range, __uint_as_float(static_cast<uint32_t>(127 + e) << 23));
}

template <int DC, int DT, int kRows>
__global__ void __launch_bounds__(32 * kWarps) latent_append_kernel(tq_latent_cache c, Slots8 a, const uint16_t* lat, const uint16_t* rope,
                                                                    long long lat_stride, long long rope_stride, int32_t* status) {
  constexpr int LANES = DC / 16, TOKENS = 32 / LANES;  // of a token; of a warp at a time
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long row0 = (static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * (kRows * TOKENS) + lane / LANES;
  int64_t slots[kRows];
  uint4 x[kRows][2], r[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const long long row = row0 + k * TOKENS;
    slots[k] = row < a.n ? a.slots[row] : -1;
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (slots[k] >= a.limit) {
      if (status && sub == 0) atomicOr(status, TQ_STATUS_BAD_SLOT);
      slots[k] = -1;
    }
    x[k][0] = x[k][1] = r[k] = make_uint4(0, 0, 0, 0);
    if (slots[k] < 0) continue;
    const long long row = row0 + k * TOKENS;
    const uint16_t* src = lat + row * lat_stride + 128 * (sub >> 3) + 8 * (sub & 7);
    x[k][0] = *reinterpret_cast<const uint4*>(src);
    x[k][1] = *reinterpret_cast<const uint4*>(src + 64);
    if (sub < 8) r[k] = *reinterpret_cast<const uint4*>(rope + row * rope_stride + 8 * sub);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) append_token<DC, DT>(c, slots[k], x[k], r[k], sub);
}

// 8 values out: 16 bytes of a 16-bit type, 32 of fp32
template <int OT>
__device__ __forceinline__ void store8(void* out, long long at, const float (&f)[8]) {
  if (OT == TQ_FP32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(out) + at);
    p[0] = make_float4(f[0], f[1], f[2], f[3]);
    p[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at) =
        make_uint4(pack2<OT>(f[0], f[1]), pack2<OT>(f[2], f[3]), pack2<OT>(f[4], f[5]), pack2<OT>(f[6], f[7]));
  }
}

template <int DC, int OT, int kRows>
__global__ void __launch_bounds__(32 * kWarps) latent_gather_kernel(tq_latent_cache c, Slots8 a, void* lat, void* rope, int32_t* status) {
  constexpr int LANES = DC / 16, TOKENS = 32 / LANES;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long row0 = (static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * (kRows * TOKENS) + lane / LANES;
  int64_t slots[kRows];
  uint4 codes[kRows], r[kRows];
  float2 scale[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) slots[k] = row0 + k * TOKENS < a.n ? a.slots[row0 + k * TOKENS] : -1;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    if (slots[k] >= a.limit) {
      if (status && sub == 0) atomicOr(status, TQ_STATUS_BAD_SLOT);
      slots[k] = -1;
    }
    codes[k] = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u);
    r[k] = make_uint4(0, 0, 0, 0);
    scale[k] = make_float2(0.0f, 0.0f);
    if (slots[k] < 0) continue;
    const uint8_t* const blk = c.blocks + (slots[k] >> 4) * latent_block_bytes(DC);
    const int t = static_cast<int>(slots[k] & 15);
    codes[k] = *reinterpret_cast<const uint4*>(blk + DC * t + 16 * sub);
    if (sub < 8) r[k] = *reinterpret_cast<const uint4*>(blk + latent_rope_offset(DC, t) + 16 * sub);
    scale[k] = *reinterpret_cast<const float2*>(blk + latent_scale_offset(DC, t));
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const long long row = row0 + k * TOKENS;
    if (row >= a.n) continue;
    const float unit = __fdiv_rn(scale[k].x, 127.0f);
    const uint32_t w[4] = {codes[k].x, codes[k].y, codes[k].z, codes[k].w};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 v = unpair(mul2(codes_of(w[2 * i + (e >> 1)], e & 1), pair(unit, unit)));
        f[2 * e] = v.x;
        f[2 * e + 1] = v.y;
      }
      store8<OT>(lat, row * DC + 128 * (sub >> 3) + 64 * i + 8 * (sub & 7), f);
    }
    if (sub < 8) {
      const uint32_t v[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 g = unpack2<TQ_FP16>(v[e]);
        f[2 * e] = g.x * scale[k].y;
        f[2 * e + 1] = g.y * scale[k].y;
      }
      store8<OT>(rope, row * kRope + 8 * sub, f);
    }
  }
}

// Rows (d_c = 512; pairs of them at 256, fours at 128) that a warp has on their way at a time: two where one each would fill
// the GPU several times over (74 K tokens appended and read back: 51 us instead of 55), one below (32 tokens: 4.2 us instead
// of 6.2).
dim3 grid_for(long long n, int d_c, int rows) {
  const long long per = kWarps * rows * (512 / d_c);
  return dim3(static_cast<unsigned>((n + per - 1) / per));
}
bool two_rows(long long n, int d_c) { return grid_for(n, d_c, 1).x > 16u * device_sm_count(); }

template <int DC, int DT>
cudaError_t append_d(const tq_latent_cache& c, const Slots8& a, const uint16_t* lat, const uint16_t* rope, long long ls, long long rs,
                     int32_t* status, cudaStream_t st) {
  const bool two = two_rows(a.n, DC);
  return launch_kernel(two ? latent_append_kernel<DC, DT, 2> : latent_append_kernel<DC, DT, 1>, grid_for(a.n, DC, two ? 2 : 1), dim3(32 * kWarps), 0, st, c,
                       a, lat, rope, ls, rs, status);
}
template <int DC, int OT>
cudaError_t gather_d(const tq_latent_cache& c, const Slots8& a, void* lat, void* rope, int32_t* status, cudaStream_t st) {
  const bool two = two_rows(a.n, DC);
  return launch_kernel(two ? latent_gather_kernel<DC, OT, 2> : latent_gather_kernel<DC, OT, 1>, grid_for(a.n, DC, two ? 2 : 1), dim3(32 * kWarps), 0, st, c,
                       a, lat, rope, status);
}
template <int DT>
cudaError_t append_t(const tq_latent_cache& c, const Slots8& a, const uint16_t* lat, const uint16_t* rope, long long ls, long long rs,
                     int32_t* status, cudaStream_t st) {
  switch (c.d_c) {
    case 128: return append_d<128, DT>(c, a, lat, rope, ls, rs, status, st);
    case 256: return append_d<256, DT>(c, a, lat, rope, ls, rs, status, st);
    default: return append_d<512, DT>(c, a, lat, rope, ls, rs, status, st);
  }
}
template <int OT>
cudaError_t gather_t(const tq_latent_cache& c, const Slots8& a, void* lat, void* rope, int32_t* status, cudaStream_t st) {
  switch (c.d_c) {
    case 128: return gather_d<128, OT>(c, a, lat, rope, status, st);
    case 256: return gather_d<256, OT>(c, a, lat, rope, status, st);
    default: return gather_d<512, OT>(c, a, lat, rope, status, st);
  }
}

}  // namespace

cudaError_t launch_latent_append(const tq_latent_cache& c, const void* lat, const void* rope, int dtype, long long lat_stride,
                                 long long rope_stride, const int64_t* slots, long long n, int32_t* status, cudaStream_t st) {
  const Slots8 a = {slots, n, latent_slots(c)};
  const auto *l = static_cast<const uint16_t*>(lat), *r = static_cast<const uint16_t*>(rope);
  return dtype == TQ_BF16 ? append_t<TQ_BF16>(c, a, l, r, lat_stride, rope_stride, status, st)
                          : append_t<TQ_FP16>(c, a, l, r, lat_stride, rope_stride, status, st);
}

cudaError_t launch_latent_gather(const tq_latent_cache& c, const int64_t* slots, long long n, void* lat, void* rope, int dtype,
                                 int32_t* status, cudaStream_t st) {
  const Slots8 a = {slots, n, latent_slots(c)};
  if (dtype == TQ_BF16) return gather_t<TQ_BF16>(c, a, lat, rope, status, st);
  return dtype == TQ_FP16 ? gather_t<TQ_FP16>(c, a, lat, rope, status, st) : gather_t<TQ_FP32>(c, a, lat, rope, status, st);
}

}  // namespace tq

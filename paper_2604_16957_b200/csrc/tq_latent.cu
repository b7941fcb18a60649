// Append to and gather from the latent cache, through slots (tq_pages_assign writes them).
//
// A token is d_c codes with one range, 64 positional channels in fp16 with a power of two, and the two scales: d_c / 16
// lanes of a warp hold it, 16 codes each (one 16-byte load of the cache's order, two of the rows'), so that a range is
// one reduction over those lanes and every byte is touched once.  Tokens do not depend on one another: any order of slots
// will do.
//
// The codes are exact roundings of the true quotients (the division by the range is that of the 8-bit cache, see
// tq_kv8.cuh).  The positional key keeps its digits: multiplied by a power of two that brings the largest magnitude into
// [2^15, 2^16) it is exact in fp16 but for bf16 channels below 2^-32 of the largest, which are off by 2^-40 of it.
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

template <int DC, int DT>
__global__ void __launch_bounds__(32 * kWarps) latent_append_kernel(tq_latent_cache c, Slots8 a, const uint16_t* lat, const uint16_t* rope,
                                                                    long long lat_stride, long long rope_stride, int32_t* status) {
  constexpr int LANES = DC / 16, TOKENS = 32 / LANES;  // of a token; of a warp
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long row = (static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * TOKENS + lane / LANES;
  int64_t slot = -1;
  if (row < a.n) slot = a.slots[row];
  if (slot >= a.limit) {
    if (status && sub == 0) atomicOr(status, TQ_STATUS_BAD_SLOT);
    slot = -1;
  }
  const bool mine = slot >= 0;
  uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)}, r = x[0];
  if (mine) {
    const uint16_t* src = lat + row * lat_stride + 128 * (sub >> 3) + 8 * (sub & 7);
    x[0] = *reinterpret_cast<const uint4*>(src);
    x[1] = *reinterpret_cast<const uint4*>(src + 64);
    if (sub < 8) r = *reinterpret_cast<const uint4*>(rope + row * rope_stride + 8 * sub);
  }
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
  if (!mine) return;
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

template <int DC, int OT>
__global__ void __launch_bounds__(32 * kWarps) latent_gather_kernel(tq_latent_cache c, Slots8 a, void* lat, void* rope, int32_t* status) {
  constexpr int LANES = DC / 16, TOKENS = 32 / LANES;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, sub = lane % LANES;
  const long long row = (static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * TOKENS + lane / LANES;
  if (row >= a.n) return;
  int64_t slot = a.slots[row];
  if (slot >= a.limit) {
    if (status && sub == 0) atomicOr(status, TQ_STATUS_BAD_SLOT);
    slot = -1;
  }
  uint4 codes = make_uint4(0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u), r = make_uint4(0, 0, 0, 0);
  float2 scale = make_float2(0.0f, 0.0f);
  if (slot >= 0) {
    const uint8_t* const blk = c.blocks + (slot >> 4) * latent_block_bytes(DC);
    const int t = static_cast<int>(slot & 15);
    codes = *reinterpret_cast<const uint4*>(blk + DC * t + 16 * sub);
    if (sub < 8) r = *reinterpret_cast<const uint4*>(blk + latent_rope_offset(DC, t) + 16 * sub);
    scale = *reinterpret_cast<const float2*>(blk + latent_scale_offset(DC, t));
  }
  const float unit = __fdiv_rn(scale.x, 127.0f);
  const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
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
    const uint32_t v[4] = {r.x, r.y, r.z, r.w};
    float f[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 g = unpack2<TQ_FP16>(v[e]);
      f[2 * e] = g.x * scale.y;
      f[2 * e + 1] = g.y * scale.y;
    }
    store8<OT>(rope, row * kRope + 8 * sub, f);
  }
}

long long blocks_for(long long n, int d_c) { return (n + kWarps * (512 / d_c) - 1) / (kWarps * (512 / d_c)); }

template <int DT>
cudaError_t append_d(const tq_latent_cache& c, const Slots8& a, const uint16_t* lat, const uint16_t* rope, long long ls, long long rs,
                     int32_t* status, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(blocks_for(a.n, c.d_c))), block(32 * kWarps);
  switch (c.d_c) {
    case 128: return launch_kernel(latent_append_kernel<128, DT>, grid, block, 0, st, c, a, lat, rope, ls, rs, status);
    case 256: return launch_kernel(latent_append_kernel<256, DT>, grid, block, 0, st, c, a, lat, rope, ls, rs, status);
    default: return launch_kernel(latent_append_kernel<512, DT>, grid, block, 0, st, c, a, lat, rope, ls, rs, status);
  }
}
template <int OT>
cudaError_t gather_d(const tq_latent_cache& c, const Slots8& a, void* lat, void* rope, int32_t* status, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(blocks_for(a.n, c.d_c))), block(32 * kWarps);
  switch (c.d_c) {
    case 128: return launch_kernel(latent_gather_kernel<128, OT>, grid, block, 0, st, c, a, lat, rope, status);
    case 256: return launch_kernel(latent_gather_kernel<256, OT>, grid, block, 0, st, c, a, lat, rope, status);
    default: return launch_kernel(latent_gather_kernel<512, OT>, grid, block, 0, st, c, a, lat, rope, status);
  }
}

}  // namespace

cudaError_t launch_latent_append(const tq_latent_cache& c, const void* lat, const void* rope, int dtype, long long lat_stride,
                                 long long rope_stride, const int64_t* slots, long long n, int32_t* status, cudaStream_t st) {
  const Slots8 a = {slots, n, latent_slots(c)};
  const auto *l = static_cast<const uint16_t*>(lat), *r = static_cast<const uint16_t*>(rope);
  return dtype == TQ_BF16 ? append_d<TQ_BF16>(c, a, l, r, lat_stride, rope_stride, status, st)
                          : append_d<TQ_FP16>(c, a, l, r, lat_stride, rope_stride, status, st);
}

cudaError_t launch_latent_gather(const tq_latent_cache& c, const int64_t* slots, long long n, void* lat, void* rope, int dtype,
                                 int32_t* status, cudaStream_t st) {
  const Slots8 a = {slots, n, latent_slots(c)};
  if (dtype == TQ_BF16) return gather_d<TQ_BF16>(c, a, lat, rope, status, st);
  return dtype == TQ_FP16 ? gather_d<TQ_FP16>(c, a, lat, rope, status, st) : gather_d<TQ_FP32>(c, a, lat, rope, status, st);
}

}  // namespace tq

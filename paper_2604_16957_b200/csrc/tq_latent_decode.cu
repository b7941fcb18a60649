// Attention of single tokens over the latent cache, absorbed form: tq_sdpa_latent_decode.
//
// A thread block per (sequence, head) walks over the tokens 64 at a time: scores (a warp per token), online softmax, and
// the sum of the latents by their weights (a thread per channel), all in fp32.
#include "tq_latent.cuh"

namespace tq {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;

template <int DT>
__device__ __forceinline__ float to_float(uint16_t x) {
  return unpack2<DT>(x).x;
}

template <int DC, int DT, int OT>
__global__ void __launch_bounds__(kThreads) latent_decode_kernel(const LatentArgs a) {
  __shared__ float q[DC + kRope], p[kTile];
  __shared__ long long at[kTile / 16 + 1];
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int len = checked_len(a.c.seq_lens, b, a.c.S_cap, h == 0 ? a.status : nullptr);
  const int lo = window_begin(len, a.window);
  const uint16_t* qc = static_cast<const uint16_t*>(a.q_c.data) + b * a.q_c.row_stride + h * a.q_c.head_stride;
  const uint16_t* qr = static_cast<const uint16_t*>(a.q_r.data) + b * a.q_r.row_stride + h * a.q_r.head_stride;
  for (int i = tid; i < DC + kRope; i += kThreads) q[i] = to_float<DT>(i < DC ? qc[i] : qr[i - DC]);
  float m = -INFINITY, l = 0.0f, o[(DC + kThreads - 1) / kThreads] = {};
  for (int t0 = lo & ~15; t0 < len; t0 += kTile) {
    __syncthreads();
    if (tid < kTile / 16 && t0 + 16 * tid < len) {
      bool ok;
      at[tid] = latent_block(a.c, b, (t0 >> 4) + tid, ok);
      if (!ok && a.status) atomicOr(a.status, TQ_STATUS_BAD_PAGE);
    }
    __syncthreads();
    for (int i = warp; i < kTile; i += kThreads / 32) {
      const int t = t0 + i;
      float z = -INFINITY;
      if (t >= lo && t < len) {
        const uint8_t* blk = a.c.blocks + at[i >> 4] * latent_block_bytes(DC);
        const float2 s = *reinterpret_cast<const float2*>(blk + latent_scale_offset(DC, t & 15));
        float zc = 0.0f, zr = 0.0f;
        for (int c = lane; c < DC; c += 32) zc += q[c] * (blk[latent_code_offset(DC, t & 15, c)] - 128.0f);
        const __half* r = reinterpret_cast<const __half*>(blk + latent_rope_offset(DC, t & 15));
        for (int c = lane; c < kRope; c += 32) zr += q[DC + c] * __half2float(r[c]);
        zc = zc * (s.x / 127.0f) + zr * s.y;
        for (int off = 16; off > 0; off >>= 1) zc += __shfl_xor_sync(0xffffffffu, zc, off);
        z = zc * a.attn_scale;
      }
      if (lane == 0) p[i] = z;
    }
    __syncthreads();
    float top = m;
    for (int i = 0; i < kTile; ++i) top = fmaxf(top, p[i]);
    const float scale = m == -INFINITY ? 0.0f : expf(m - top);
    m = top;
    l *= scale;
#pragma unroll
    for (float& x : o) x *= scale;
    // (sums of a tile of their own: a long row added token by token would lose digits)
    float tile_l = 0.0f, tile_o[(DC + kThreads - 1) / kThreads] = {};
    for (int i = 0; i < kTile; ++i) {
      const int t = t0 + i;
      if (t < lo || t >= len) continue;
      const uint8_t* blk = a.c.blocks + at[i >> 4] * latent_block_bytes(DC);
      const float w = expf(p[i] - m);
      tile_l += w;
      const float ws = w * (*reinterpret_cast<const float*>(blk + latent_scale_offset(DC, t & 15)) / 127.0f);
      for (int c = tid, x = 0; c < DC; c += kThreads, ++x) tile_o[x] += ws * (blk[latent_code_offset(DC, t & 15, c)] - 128.0f);
    }
    l += tile_l;
#pragma unroll
    for (int x = 0; x < (DC + kThreads - 1) / kThreads; ++x) o[x] += tile_o[x];
  }
  const long long to = (static_cast<long long>(b) * a.H + h) * DC;
  for (int c = tid, x = 0; c < DC; c += kThreads, ++x) {
    const float y = len > 0 ? o[x] / l : 0.0f;
    if (OT == TQ_FP32) static_cast<float*>(a.out)[to + c] = y;
    else static_cast<uint16_t*>(a.out)[to + c] = static_cast<uint16_t>(pack2<DT>(y, y));
  }
}

template <int DC>
cudaError_t launch_dc(const LatentArgs& a, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.H), static_cast<unsigned>(a.c.B));
  if (a.q_dtype == TQ_BF16)
    return a.out_dtype == TQ_FP32 ? launch_kernel(latent_decode_kernel<DC, TQ_BF16, TQ_FP32>, grid, dim3(kThreads), 0, st, a)
                                  : launch_kernel(latent_decode_kernel<DC, TQ_BF16, TQ_BF16>, grid, dim3(kThreads), 0, st, a);
  return a.out_dtype == TQ_FP32 ? launch_kernel(latent_decode_kernel<DC, TQ_FP16, TQ_FP32>, grid, dim3(kThreads), 0, st, a)
                                : launch_kernel(latent_decode_kernel<DC, TQ_FP16, TQ_FP16>, grid, dim3(kThreads), 0, st, a);
}

}  // namespace

size_t latent_workspace_bytes(int B, int H, int d_c) {
  return 256 + 16 * static_cast<size_t>(B) + 2 * static_cast<size_t>(device_sm_count()) * (H <= 16 ? 16 : (H <= 32 ? 32 : 64)) * (d_c + 2) * 4;
}

cudaError_t launch_latent_decode(const LatentArgs& a, cudaStream_t st) {
  switch (a.c.d_c) {
    case 128: return launch_dc<128>(a, st);
    case 256: return launch_dc<256>(a, st);
    default: return launch_dc<512>(a, st);
  }
}

}  // namespace tq

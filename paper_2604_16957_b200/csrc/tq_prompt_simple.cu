// Attention of packed prompts, scalar form: one warp per (query row, head) walks over the keys that the query sees,
// online softmax, nothing else.  Right for every shape that tq_sdpa_prompt takes; arithmetic-bound on the CUDA cores.
#include "tq_kv8.cuh"
#include "tq_prompt.cuh"

namespace tq {
namespace {

constexpr int kWarps = 4;

template <int D, int DT>
__global__ void __launch_bounds__(32 * kWarps) prompt_simple_kernel(const PromptArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int E = D / 64;  // words (two channels) per lane
  const int lane = threadIdx.x & 31;
  const int head = blockIdx.y * kWarps + (threadIdx.x >> 5);
  if (head >= a.H_q) return;
  const int row = blockIdx.x;
  int b = 0, hi = a.B;  // the last sequence that begins at or before the row
  while (hi - b > 1) {
    const int mid = (b + hi) >> 1;
    if (a.q_offsets[mid] <= row) b = mid;
    else hi = mid;
  }
  const PromptSeq s = prompt_seq(a, b, lane == 0 && head == 0);
  if (row < s.q0 || row >= s.q0 + s.lq) return;  // a row of no sequence
  const int i = row - s.q0;
  int lo, up;
  prompt_keys(a, s, i, lo, up);
  const int h = head / (a.H_q / a.H_kv);
  auto word = [&](const void* base, long long stride, long long r, int hh, int e) {
    return __ldg(reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(base) + r * stride + static_cast<long long>(hh) * D) + lane + 32 * e);
  };
  float2 q[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = unpack2<DT>(word(a.q, a.q_stride, row, head, e));
    o[e] = make_float2(0.0f, 0.0f);
  }
  float m = -INFINITY, l = 0.0f;
  for (int j = lo; j < up; ++j) {
    float z = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 k = unpack2<DT>(word(a.k, a.k_stride, s.k0 + j, h, e));
      z += q[e].x * k.x + q[e].y * k.y;
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) z += __shfl_xor_sync(0xffffffffu, z, x);
    z *= a.attn_scale;
    const float n = fmaxf(m, z);
    const float was = m == n ? 1.0f : expf(m - n), p = z == n ? 1.0f : expf(z - n);
    l = l * was + p;
    m = n;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float2 v = unpack2<DT>(word(a.v, a.v_stride, s.k0 + j, h, e));
      o[e].x = o[e].x * was + p * v.x;
      o[e].y = o[e].y * was + p * v.y;
    }
  }
  const float inv = up > lo ? 1.0f / l : 0.0f;
  const long long at = (static_cast<long long>(row) * a.H_q + head) * (D / 2) + lane;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float x = o[e].x * inv, y = o[e].y * inv;
    if (a.out_dtype == TQ_FP32) static_cast<float2*>(a.out)[at + 32 * e] = make_float2(x, y);
    else static_cast<uint32_t*>(a.out)[at + 32 * e] = pack2<DT>(x, y);
  }
}

template <int D>
cudaError_t launch_d(const PromptArgs& a, cudaStream_t st) {
  const dim3 grid(a.n_q, (a.H_q + kWarps - 1) / kWarps);
  if (a.dtype == TQ_BF16) return launch_kernel(prompt_simple_kernel<D, TQ_BF16>, grid, dim3(32 * kWarps), 0, st, a);
  return launch_kernel(prompt_simple_kernel<D, TQ_FP16>, grid, dim3(32 * kWarps), 0, st, a);
}

}  // namespace

cudaError_t launch_prompt_simple(const PromptArgs& a, cudaStream_t st) {
  switch (a.d) {
    case 64: return launch_d<64>(a, st);
    case 128: return launch_d<128>(a, st);
    case 256: return launch_d<256>(a, st);
    default: return launch_d<512>(a, st);
  }
}

}  // namespace tq

// Append to and gather from the 8-bit KV cache, through slots (tq_pages_assign writes them).
//
// Work is cut into runs: up to 16 consecutive rows of the call whose slots are consecutive inside one 16-token block.
// One warp handles a run of one KV head, K or V: it holds the whole block in registers (16 tokens x d values, 16 bytes
// of codes per lane and 32 channels), so a range is one reduction over the warp and every byte of the inputs and of
// the cache is touched once.  K lanes own (tokens g, g + 8; 8 channels) as in the block's byte order: 16-byte loads
// and one 16-byte store per 32 channels.  V lanes own (tokens 2t, 2t+1, 2t+8, 2t+9; 8 consecutive channels): 16-byte
// loads, and eight 4-byte stores that fill whole 32-byte sectors across the lanes; nothing goes through shared memory.
// The kernels are bound by HBM for prompts and by two dependent memory latencies for a decode step.  Measured on 74 K
// tokens of 8 KV heads, d = 128, K and V as slices of the fused projection (0.45 GB each way, 69 us at the copy rate):
// append 94 us (with eight thread blocks per SM; 114 us with the six that its registers would allow unasked), gather
// 76 us (all loads of a run first; 84 us without).
//
// Which rows start a run is found by the warp itself from the slots: every warp looks at `chunk` rows (32 for prompts,
// fewer where that leaves SMs without work: see chunk_of).
#include "tq_kv8.cuh"

namespace tq {
namespace {

constexpr int kWarps = 4;

// 16 tokens x D values of one lane: word i of row r.  K: R = 2 rows (tokens g, g + 8) x D / 32 vectors; V: 4 rows
// (tokens 2t, 2t + 1, 2t + 8, 2t + 9) x D / 64 vectors (8 channels each; a lane takes every other 32-channel group at
// d = 64: see v_octet).
template <int D, bool V>
struct Part {
  static constexpr int ROWS = V ? 4 : 2;
  static constexpr int VECS = V ? D / 64 : D / 32;
  __device__ static __forceinline__ int token(int lane, int r) {
    if (!V) return (lane >> 2) + 8 * r;
    return 2 * (lane & 3) + (r & 1) + 8 * (r >> 1);
  }
  // first channel of vector i of the lane
  __device__ static __forceinline__ int channel(int lane, int i) {
    if (!V) return 32 * i + 8 * (lane & 3);
    return 64 * i + 8 * (lane >> 2);
  }
};

// Codes (as stored, + 128) of a lane's vector i: 2 words per row, byte e of the pair = channel e.
template <int D, bool V>
__device__ __forceinline__ void load_codes(const uint8_t* blk, int lane, int i, uint32_t (&w)[Part<D, V>::ROWS][2]) {
  if (!V) {
    const uint4 x = *reinterpret_cast<const uint4*>(blk + 512 * i + 16 * lane);
    w[0][0] = x.x;
    w[0][1] = x.y;
    w[1][0] = x.z;
    w[1][1] = x.w;
  } else {
    const int c = Part<D, V>::channel(lane, i);
    const uint8_t* p = blk + 16 * D + 512 * (c >> 5) + 16 * (lane & 3) + 4 * ((c & 31) >> 3);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      uint32_t t[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = *reinterpret_cast<const uint32_t*>(p + 64 * (4 * hf + e));
      turn4(t);
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r % Part<D, V>::ROWS][hf] = t[r];
    }
  }
}

template <int D, bool V>
__device__ __forceinline__ void store_codes(uint8_t* blk, int lane, int i, const uint32_t (&w)[Part<D, V>::ROWS][2]) {
  if (!V) {
    *reinterpret_cast<uint4*>(blk + 512 * i + 16 * lane) = make_uint4(w[0][0], w[0][1], w[1][0], w[1][1]);
  } else {
    const int c = Part<D, V>::channel(lane, i);
    uint8_t* p = blk + 16 * D + 512 * (c >> 5) + 16 * (lane & 3) + 4 * ((c & 31) >> 3);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      uint32_t t[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) t[r] = w[r % Part<D, V>::ROWS][hf];
      turn4(t);
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(p + 64 * (4 * hf + e)) = t[e];
    }
  }
}

// Rows of the run that starts at row n with slot s: consecutive slots inside one block.
__device__ __forceinline__ int run_length(const Slots8& a, long long n, int64_t s, int lane) {
  const int l = lane & 15;
  const bool mine = n + l < a.n && (s & 15) + l < 16 && a.slots[n + l] == s + l;
  const unsigned m = __ballot_sync(0xffffffffu, mine) & 0xffffu;
  return __ffs(static_cast<int>(~m)) - 1;
}

template <int D, int DT, bool V>
__device__ __forceinline__ void append_run(uint8_t* blk, const uint16_t* src, long long stride, int off, int len, int lane) {
  using P = Part<D, V>;
  // rows of the block: [0, off) older tokens, [off, off + len) new ones, the rest unused (code 0).  At d = 512 a lane's
  // share of the block does not fit its registers; the second pass reads it again, from L1.
  constexpr bool kHold = D < 512;
  uint4 x[P::ROWS][kHold ? P::VECS : 1];
  bool fresh[P::ROWS], older[P::ROWS];
#pragma unroll
  for (int r = 0; r < P::ROWS; ++r) {
    const int t = P::token(lane, r) - off;
    fresh[r] = t >= 0 && t < len;
    older[r] = t < 0;
  }
  auto load = [&](int r, int i) {
    if (!fresh[r]) return make_uint4(0, 0, 0, 0);
    return __ldg(reinterpret_cast<const uint4*>(src + (P::token(lane, r) - off) * stride + P::channel(lane, i)));
  };
  if (kHold) {
#pragma unroll
    for (int r = 0; r < P::ROWS; ++r)
#pragma unroll
      for (int i = 0; i < P::VECS; ++i) x[r][kHold ? i : 0] = load(r, i);
  }
  float* range = reinterpret_cast<float*>(blk + range8_offset(D, V));
  const float a_old = off > 0 ? *range : 0.0f;
  // magnitudes as integers, two to a word; an infinity or a NaN is above every finite one
  uint32_t top = 0;
#pragma unroll
  for (int r = 0; r < P::ROWS; ++r)
#pragma unroll(kHold ? P::VECS : 4)
    for (int i = 0; i < P::VECS; ++i) {
      const uint4 y = kHold ? x[r][kHold ? i : 0] : load(r, i);
      top = __vmaxu2(__vmaxu2(top, __vmaxu2(y.x & 0x7fff7fffu, y.y & 0x7fff7fffu)), __vmaxu2(y.z & 0x7fff7fffu, y.w & 0x7fff7fffu));
    }
  top = max(top & 0xffffu, top >> 16);
  constexpr uint32_t kInf = DT == TQ_BF16 ? 0x7f80u : 0x7c00u;
  const bool odd = __any_sync(0xffffffffu, top >= kInf);
  if (odd) {
    top = 0;
#pragma unroll 1
    for (int r = 0; r < P::ROWS; ++r)
#pragma unroll 1
      for (int i = 0; i < P::VECS; ++i) {
        const uint4 y = load(r, i);
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
        for (int e = 0; e < 4; ++e) {
          const uint32_t z = finite8<DT>(w[e]) & 0x7fff7fffu;
          top = max(top, max(z & 0xffffu, z >> 16));
        }
      }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  const float a_new = fmaxf(a_old, unpack2<DT>(top).x);
  const Div8 q(a_new);
  const float m127 = __fmul_rn(q.scale, 127.0f);
  const uint64_t fresh_mul = pair(m127, m127), older_mul = pair(__fmul_rn(a_old, q.scale), __fmul_rn(a_old, q.scale));
#pragma unroll(kHold ? P::VECS : 1)
  for (int i = 0; i < P::VECS; ++i) {
    uint32_t w[P::ROWS][2];
    if (off > 0) {
      load_codes<D, V>(blk, lane, i, w);
    } else {
#pragma unroll
      for (int r = 0; r < P::ROWS; ++r) w[r][0] = w[r][1] = 0x80808080u;
    }
#pragma unroll
    for (int r = 0; r < P::ROWS; ++r) {
      if (fresh[r]) {
        const uint4 y = kHold ? x[r][kHold ? i : 0] : load(r, i);
        uint32_t v[4] = {y.x, y.y, y.z, y.w};
        if (odd) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = finite8<DT>(v[e]);
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float2 f = unpack2<DT>(v[2 * hf]), g = unpack2<DT>(v[2 * hf + 1]);
          w[r][hf] = low_bytes(q.codes(mul2(pair(f.x, f.y), fresh_mul)), q.codes(mul2(pair(g.x, g.y), fresh_mul)));
        }
      } else if (older[r] && a_new != a_old) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
          w[r][hf] = low_bytes(q.codes(mul2(codes_of(w[r][hf], 0), older_mul)), q.codes(mul2(codes_of(w[r][hf], 1), older_mul)));
      } else if (!older[r]) {
        w[r][0] = w[r][1] = 0x80808080u;
      }
    }
    store_codes<D, V>(blk, lane, i, w);
  }
  if (lane == 0) {
    *range = a_new;
    if (V) *reinterpret_cast<float2*>(blk + 32 * D + 8) = make_float2(0.0f, 0.0f);
  }
}

template <int D, int DT>
__global__ void __launch_bounds__(32 * kWarps, D <= 128 ? 8 : 1) append_kernel(tq_kv8_cache c, Slots8 a, const uint16_t* k, const uint16_t* v,
                                                             long long k_stride, long long v_stride, int chunk,
                                                             int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  // the units (KV head, K or V) of a chunk of rows are neighbours in the grid: their rows lie side by side in memory
  const int groups = (2 * c.H_kv + kWarps - 1) / kWarps;
  const int unit = static_cast<int>(blockIdx.x % groups) * kWarps + (threadIdx.x >> 5);
  if (unit >= 2 * c.H_kv) return;
  const int h = unit >> 1;
  const bool is_v = unit & 1;
  const long long base = static_cast<long long>(blockIdx.x / groups) * chunk;
  const long long n = base + lane;
  int64_t s = -1, prev = -1;
  if (lane < chunk && n < a.n) {
    s = a.slots[n];
    if (n > 0) prev = a.slots[n - 1];
  }
  bool lead = s >= 0 && s < a.limit;
  if (s >= a.limit && status) atomicOr(status, TQ_STATUS_BAD_SLOT);
  if (lead && prev >= 0 && (s >> 4) == (prev >> 4)) {
    // same block as the row before: part of its run, or out of order (that row is skipped)
    if (s != prev + 1 && status) atomicOr(status, TQ_STATUS_BAD_SLOT);
    lead = false;
  }
  unsigned todo = __ballot_sync(0xffffffffu, lead);
  while (todo) {
    const int l = __ffs(static_cast<int>(todo)) - 1;
    todo &= todo - 1;
    const long long row = base + l;
    const int64_t slot = __shfl_sync(0xffffffffu, s, l);
    const int len = run_length(a, row, slot, lane);
    uint8_t* blk = block8_of(c, slot, h);
    const int off = static_cast<int>(slot & 15);
    if (is_v) append_run<D, DT, true>(blk, v + row * v_stride + h * D, v_stride, off, len, lane);
    else append_run<D, DT, false>(blk, k + row * k_stride + h * D, k_stride, off, len, lane);
  }
}

template <int D, int DT, bool V>
__device__ __forceinline__ void gather_run(const uint8_t* blk, void* dst, long long stride, int off, int len, int lane) {
  using P = Part<D, V>;
  const float scale = blk ? __fdiv_rn(*reinterpret_cast<const float*>(blk + range8_offset(D, V)), 127.0f) : 0.0f;
  // all of the lane's codes are asked for before the first is used (d = 512: registers allow half)
  constexpr int kAhead = D == 512 ? P::VECS / 2 : P::VECS;
  uint32_t ahead[kAhead][P::ROWS][2];
#pragma unroll
  for (int i = 0; i < P::VECS; ++i) {
    if (i % kAhead == 0) {
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        if (blk) {
          load_codes<D, V>(blk, lane, i + x, ahead[x]);
        } else {
#pragma unroll
          for (int r = 0; r < P::ROWS; ++r) ahead[x][r][0] = ahead[x][r][1] = 0x80808080u;
        }
      }
    }
    const uint32_t(&w)[P::ROWS][2] = ahead[i % kAhead];
#pragma unroll
    for (int r = 0; r < P::ROWS; ++r) {
      const int t = P::token(lane, r) - off;
      if (t < 0 || t >= len) continue;
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 v = unpair(mul2(codes_of(w[r][e >> 1], e & 1), pair(scale, scale)));
        f[2 * e] = v.x;
        f[2 * e + 1] = v.y;
      }
      const long long at = t * stride + P::channel(lane, i);
      if (DT == TQ_FP32) {
        float4* o = reinterpret_cast<float4*>(static_cast<float*>(dst) + at);
        o[0] = make_float4(f[0], f[1], f[2], f[3]);
        o[1] = make_float4(f[4], f[5], f[6], f[7]);
      } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(dst) + at) =
            make_uint4(pack2<DT>(f[0], f[1]), pack2<DT>(f[2], f[3]), pack2<DT>(f[4], f[5]), pack2<DT>(f[6], f[7]));
      }
    }
  }
}

template <int D, int DT>
__global__ void __launch_bounds__(32 * kWarps) gather_kernel(tq_kv8_cache c, Slots8 a, void* k, void* v, int chunk,
                                                             int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int groups = (2 * c.H_kv + kWarps - 1) / kWarps;
  const int unit = static_cast<int>(blockIdx.x % groups) * kWarps + (threadIdx.x >> 5);
  if (unit >= 2 * c.H_kv) return;
  const int h = unit >> 1;
  const bool is_v = unit & 1;
  constexpr int kBytes = DT == TQ_FP32 ? 4 : 2;
  const long long base = static_cast<long long>(blockIdx.x / groups) * chunk;
  const long long n = base + lane;
  const bool mine = lane < chunk && n < a.n;
  int64_t s = -1, prev = -1;
  if (mine) {
    s = a.slots[n];
    if (n > 0) prev = a.slots[n - 1];
    if (s >= a.limit) {
      if (status) atomicOr(status, TQ_STATUS_BAD_SLOT);
      s = -1;
    }
  }
  // a slot may be asked for more than once, in any order: whatever does not continue the row before starts a run
  unsigned todo = __ballot_sync(0xffffffffu, mine && (s < 0 || s != prev + 1 || (s & 15) == 0));
  const long long stride = static_cast<long long>(c.H_kv) * D;
  while (todo) {
    const int l = __ffs(static_cast<int>(todo)) - 1;
    todo &= todo - 1;
    const long long row = base + l;
    const int64_t slot = __shfl_sync(0xffffffffu, s, l);
    const int len = slot < 0 ? 1 : run_length(a, row, slot, lane);
    const uint8_t* blk = slot < 0 ? nullptr : block8_of(c, slot, h);
    const int off = slot < 0 ? 0 : static_cast<int>(slot & 15);
    char* dst = static_cast<char*>(is_v ? v : k) + (row * stride + h * D) * kBytes;
    if (is_v) gather_run<D, DT, true>(blk, dst, stride, off, len, lane);
    else gather_run<D, DT, false>(blk, dst, stride, off, len, lane);
  }
}

// Rows per warp: 32 (two whole blocks of a prompt) where that leaves every SM about 16 warps, else fewer, so that the
// runs of a decode step (one row each) are handled side by side and not one after the other.
int chunk_of(const tq_kv8_cache& c, long long n) {
  const long long want = 16LL * device_sm_count();
  int chunk = 32;
  while (chunk > 1 && 2 * c.H_kv * ((n + chunk - 1) / chunk) < want) chunk >>= 1;
  return chunk;
}

template <int D>
cudaError_t append_d(const tq_kv8_cache& c, const Slots8& a, const void* k, const void* v, int dtype, long long k_stride,
                     long long v_stride, int32_t* status, cudaStream_t st) {
  const int chunk = chunk_of(c, a.n);
  const long long blocks = (a.n + chunk - 1) / chunk * ((2 * c.H_kv + kWarps - 1) / kWarps);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks));
  auto kp = static_cast<const uint16_t*>(k), vp = static_cast<const uint16_t*>(v);
  if (dtype == TQ_BF16)
    return launch_kernel(append_kernel<D, TQ_BF16>, grid, dim3(32 * kWarps), 0, st, c, a, kp, vp, k_stride, v_stride, chunk, status);
  return launch_kernel(append_kernel<D, TQ_FP16>, grid, dim3(32 * kWarps), 0, st, c, a, kp, vp, k_stride, v_stride, chunk, status);
}

template <int D>
cudaError_t gather_d(const tq_kv8_cache& c, const Slots8& a, void* k, void* v, int dtype, int32_t* status, cudaStream_t st) {
  const int chunk = chunk_of(c, a.n);
  const long long blocks = (a.n + chunk - 1) / chunk * ((2 * c.H_kv + kWarps - 1) / kWarps);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
  const dim3 grid(static_cast<unsigned>(blocks));
  if (dtype == TQ_BF16) return launch_kernel(gather_kernel<D, TQ_BF16>, grid, dim3(32 * kWarps), 0, st, c, a, k, v, chunk, status);
  if (dtype == TQ_FP32) return launch_kernel(gather_kernel<D, TQ_FP32>, grid, dim3(32 * kWarps), 0, st, c, a, k, v, chunk, status);
  return launch_kernel(gather_kernel<D, TQ_FP16>, grid, dim3(32 * kWarps), 0, st, c, a, k, v, chunk, status);
}

Slots8 slots8(const tq_kv8_cache& c, const int64_t* slots, long long n) {
  const long long limit = c.page_table ? static_cast<long long>(c.num_pages) * c.page_tokens : static_cast<long long>(c.B) * c.S_cap;
  return {slots, n, limit};
}

}  // namespace

cudaError_t launch_kv8_append(const tq_kv8_cache& c, const void* k, const void* v, int dtype, long long k_stride,
                              long long v_stride, const int64_t* slots, long long n, int32_t* status, cudaStream_t st) {
  const Slots8 a = slots8(c, slots, n);
  switch (c.d) {
    case 64: return append_d<64>(c, a, k, v, dtype, k_stride, v_stride, status, st);
    case 128: return append_d<128>(c, a, k, v, dtype, k_stride, v_stride, status, st);
    case 256: return append_d<256>(c, a, k, v, dtype, k_stride, v_stride, status, st);
    default: return append_d<512>(c, a, k, v, dtype, k_stride, v_stride, status, st);
  }
}

cudaError_t launch_kv8_gather(const tq_kv8_cache& c, const int64_t* slots, long long n, void* k, void* v, int dtype,
                              int32_t* status, cudaStream_t st) {
  const Slots8 a = slots8(c, slots, n);
  switch (c.d) {
    case 64: return gather_d<64>(c, a, k, v, dtype, status, st);
    case 128: return gather_d<128>(c, a, k, v, dtype, status, st);
    case 256: return gather_d<256>(c, a, k, v, dtype, status, st);
    default: return gather_d<512>(c, a, k, v, dtype, status, st);
  }
}

}  // namespace tq

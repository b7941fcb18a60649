// Attention of packed prompts on the tensor cores (tcgen05, TMEM, TMA): tq_sdpa_prompt.
//
// A tile is 128 query rows of one KV head: T = 128 / G tokens times the G query heads that share the head, token by
// token, so K and V are read once per KV head whatever G is.  A thread block works on NQ tiles (two at d <= 128, one
// above) over a common stream of K / V tiles of BN keys:
//     S = Q K^T   (tcgen05.mma, both operands in shared memory, S in TMEM)
//     P = 2^(c S - c m), rounded to 16 bits, back into TMEM over S   (a thread per row, online softmax)
//     O += P V    (A operand P from TMEM, V as it lies in memory: rows along K)
// c = alpha log2 e > 0 (for a negative alpha the MMA negates Q).  m is raised only when a score exceeds it by more than
// 2^8; then the thread rescales its row of O in TMEM.  With two tiles the tensor cores work on one while the softmax
// of the other runs; with one tile (d = 256, 512) S has two buffers and the next scores are computed meanwhile.  At
// d = 512 the accumulator of a row does not fit TMEM: a thread block computes 256 of the 512 output channels, and S is
// computed twice.
//
// Roles: one warpgroup of softmax threads per tile; a warp that issues TMA loads; a warp that issues the MMAs; two
// warps that look through the V tiles which some row sees in part.  Those may hold tokens of a neighbouring sequence
// or of the row's future, whose weight is 0, and 0 * inf is not 0: a value there that is no finite number is
// replaced by 0 in shared memory, and the rows that do see it get it added back in the epilogue from global memory.
//
// What bounds it: at d = 128 a 128 x 128 tile costs the tensor cores 1024 cycles and the exponential unit 1024 cycles (16
// per cycle and SM).
#include <cuda.h>

#include "tq_async.cuh"
#include "tq_kv8.cuh"
#include "tq_prompt.cuh"
#include "tq_tcgen05.cuh"

#ifndef TQ_POLY
#define TQ_POLY 0
#endif
namespace tq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;  // log2 units a score may exceed the running maximum: weights stay below 2^8

template <int D>
struct Cfg {
  static constexpr int NQ = D <= 128 ? 2 : 1;         // query tiles of a thread block
  static constexpr int BN = D <= 128 ? 128 : (D == 256 ? 64 : 32);  // keys of a K / V tile
  static constexpr int DV = D <= 256 ? D : 256;       // output channels of a thread block
  static constexpr int NSB = NQ == 2 ? 1 : 2;         // S buffers of a tile
  static constexpr int SOFT = 4 * NQ;                 // softmax warps
  static constexpr int POLY = NQ == 2 ? TQ_POLY : 0;  // pairs in 16 whose exponentials the FMA units compute
  static constexpr int SCRUB = 2;
  static constexpr int WARPS = SOFT + 2 + SCRUB;      // softmax | TMA | MMA | scrub
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int QCHUNK = 128 * 128;            // bytes of 128 rows x 64 channels
  static constexpr int QTILE = (D / 64) * QCHUNK;
  static constexpr int KCHUNK = BN * 128;
  static constexpr int SLOT = (D / 64) * KCHUNK;      // a K tile; a V tile needs no more
  static constexpr int NS = D == 64 ? 8 : (D == 512 ? 3 : 5);  // slots of the K / V ring
  static constexpr int RING = NQ * QTILE;
  static constexpr int BARS = RING + NS * SLOT;
  static constexpr int SMEM = BARS + 512 + 1024;      // barriers, and room to align the base
  static constexpr int S_COL = 0;                     // TMEM columns: S of tile / buffer i at 128 i (P over it), O behind
  static constexpr int O_COL = D <= 128 ? 256 : (D == 256 ? 128 : 64);
  static constexpr int S_STEP = BN;
  static_assert(O_COL >= NQ * NSB * BN && O_COL + NQ * DV <= 512, "tensor memory");
  static_assert(SMEM <= 232448, "shared memory");
};

struct Maps {
  CUtensorMap q, k, v;
};

// mbarriers of a thread block, 8 bytes each
template <int D>
struct Bars {
  using C = Cfg<D>;
  static constexpr int FULL = 0, EMPTY = FULL + C::NS, Q = EMPTY + C::NS, S = Q + 1, P = S + C::NQ * C::NSB,
                       O = P + C::NQ * C::NSB, ASK = O + C::NQ, SCRUB = ASK + 1, DRAIN = SCRUB + 1,
                       COUNT = DRAIN + 1;
  static_assert(COUNT * 8 <= 512, "room for the barriers");
};

// Bounded wait that also gives up when another warp of the thread block has: false, and the block winds down.  (Inline:
// registers cannot be moved between warps, as the kernel does, around a function call.)
constexpr long long kTileWait = 16 * kMaxWaitCycles;  // 35 ms: a wait may span some other role's work on a few tiles
constexpr long long kBlockWait = 1LL << 34;           // 9 s: a wait for the first tile that needs mending may span them all
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (*stop) return false;
    if (clock64() - t0 > limit) {
      *stop = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit = kTileWait) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_slow(bar, parity, stop, limit);
}
// the same for a whole warp: all its lanes go on, or none
__device__ __forceinline__ bool warp_wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit = kTileWait) {
  return __all_sync(0xffffffffu, wait_on(bar, parity, stop, limit));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
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
__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 2^y for two y <= 2^7 on the FMA units: y = n + f with n an integer and |f| <= 1/2, 2^f by a polynomial that is minimax
// in the relative error on that interval (fitted by linear programming: 7.5e-5 at degree 3, 2.6e-6 at degree 4, against
// the 2^-9 and 2^-12 of the rounding to bf16 and fp16 that follows), n added to the exponent.  The exponential unit does
// 16 values per cycle and SM; taking a share of them off it is what lets it keep up with the tensor cores.
template <int DT>
__device__ __forceinline__ float2 exp2_pair(uint64_t y) {
  constexpr float kMagic = 12582912.0f;  // 1.5 * 2^23: adding it rounds to an integer
  const float2 v = unpair(y);
  y = pair(fmaxf(v.x, -126.0f), fmaxf(v.y, -126.0f));
  const uint64_t t = add2(y, pair(kMagic, kMagic));
  const uint64_t f = fma2(add2(t, pair(-kMagic, -kMagic)), pair(-1.0f, -1.0f), y);
  auto both = [](float x) { return pair(x, x); };
  uint64_t p;
  if (DT == TQ_BF16) {
    p = fma2(both(0.05517132207751274f), f, both(0.2426113337278366f));
    p = fma2(p, f, both(0.6932610869407654f));
    p = fma2(p, f, both(0.9999280571937561f));
  } else {
    p = fma2(both(0.00957053154706955f), f, both(0.05591866374015808f));
    p = fma2(p, f, both(0.24024735391139984f));
    p = fma2(p, f, both(0.6931216716766357f));
    p = fma2(p, f, both(0.9999992847442627f));
  }
  const float2 q = unpair(p), n = unpair(t);
  return make_float2(__uint_as_float(__float_as_uint(q.x) + (__float_as_uint(n.x) << 23)),
                     __uint_as_float(__float_as_uint(q.y) + (__float_as_uint(n.y) << 23)));
}

// nonzero if one of the two 16-bit values of a word is an infinity or a NaN
template <int DT>
__device__ __forceinline__ uint32_t not_finite2(uint32_t w) {
  return ((w & 0x7fff7fffu) + (DT == TQ_BF16 ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}

// What a thread block works on, the same for all its warps.
struct Work {
  PromptSeq s;
  int h;           // KV head
  int tok0;        // first query token of tile 0
  int T;           // tokens of a tile
  int lo_all, up_all;    // keys that some row sees
  int lo_every, up_every;  // keys that every row sees
};

// Key tiles [j0, j1) of query tile i (empty: j0 >= j1).
template <int BN>
__device__ __forceinline__ void tile_range(const PromptArgs& a, const Work& w, int i, int& j0, int& j1) {
  const int first = w.tok0 + i * w.T, last = min(first + w.T, w.s.lq) - 1;
  j0 = j1 = 0;
  if (last < first) return;
  int lo, up, lo2, up2;
  prompt_keys(a, w.s, first, lo, up);
  prompt_keys(a, w.s, last, lo2, up2);
  j0 = lo / BN;
  j1 = (up2 + BN - 1) / BN;
}

template <int D, int DT, int OT>
__global__ void __launch_bounds__(Cfg<D>::THREADS, 1) prompt_kernel(const __grid_constant__ Maps maps, const PromptArgs a,
                                                                    int G, int T) {
  using C = Cfg<D>;
  using B = Bars<D>;
  extern __shared__ uint8_t raw[];
  __shared__ uint32_t s_tmem;
  __shared__ int s_stop, s_scrubbed, s_seq;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
  uint8_t* const smem = raw + (base - smem_addr(raw));
  const uint32_t bars = base + C::BARS;
  auto bar = [&](int i) { return bars + 8 * i; };
  volatile int* const stop = &s_stop;

  if (warp == C::SOFT + 1) tmem_alloc(smem_addr(&s_tmem), 512);
  if (tid == 0) {
    for (int i = 0; i < C::NS; ++i) {
      mbar_init(bar(B::FULL + i), 1);
      mbar_init(bar(B::EMPTY + i), 1);
    }
    mbar_init(bar(B::Q), 1);
    for (int i = 0; i < C::NQ * C::NSB; ++i) {
      mbar_init(bar(B::S + i), 1);
      mbar_init(bar(B::P + i), 4);
    }
    for (int i = 0; i < C::NQ; ++i) mbar_init(bar(B::O + i), 1);
    mbar_init(bar(B::ASK), 1);
    mbar_init(bar(B::SCRUB), C::SCRUB);
    mbar_init(bar(B::DRAIN), 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    s_stop = 0;
    s_scrubbed = 0;
  }
  pdl_launch_dependents();
  pdl_wait();

  // ---- which tile: sequence b starts at tile q_offsets[b] / TT + b, which leaves room for its ceil(lq / TT) tiles.  The
  // late tiles of a sequence see the most keys under the causal mask and go first.
  const int TT = C::NQ * T;
  const int halves = D / C::DV;
  int at = blockIdx.x;
  const int half = at % halves;
  at /= halves;
  Work w;
  w.T = T;
  w.h = at % a.H_kv;
  const int tile = a.n_q / TT + a.B - 1 - at / a.H_kv;
  if (tid == 0) {
    int b = 0, hi = a.B;
    while (hi - b > 1) {
      const int mid = (b + hi) >> 1;
      if (min(max(a.q_offsets[mid], 0), a.n_q) / TT + mid <= tile) b = mid;
      else hi = mid;
    }
    s_seq = b;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const int b = s_seq;
  const uint32_t tmem = s_tmem;
  w.s = prompt_seq(a, b, false);
  w.tok0 = (tile - (w.s.q0 / TT + b)) * TT;
  const bool mine = w.tok0 >= 0 && w.tok0 < w.s.lq;
  if (mine && w.tok0 == 0 && w.h == 0 && tid == 0) (void)prompt_seq(a, b, true);  // one reports for the sequence

  int J0 = 0, J1 = 0, j0[C::NQ], j1[C::NQ];
#pragma unroll
  for (int i = 0; i < C::NQ; ++i) {
    j0[i] = j1[i] = 0;
    if (mine) tile_range<C::BN>(a, w, i, j0[i], j1[i]);
    if (j1[i] > j0[i]) {
      if (J1 == J0) {
        J0 = j0[i];
        J1 = j1[i];
      } else {
        J0 = min(J0, j0[i]);
        J1 = max(J1, j1[i]);
      }
    }
  }
  {
    // what every valid row sees: from the last token's first key to the first token's last one
    const int last = min(w.tok0 + TT, w.s.lq) - 1;
    int x, y;
    prompt_keys(a, w.s, w.tok0, w.lo_all, w.up_every);
    prompt_keys(a, w.s, last, x, y);
    w.lo_every = x;
    w.up_all = y;
  }
  auto in = [&](int i, int j) { return j >= j0[i] && j < j1[i]; };
  auto partly = [&](int j) { return j * C::BN < w.lo_every || (j + 1) * C::BN > w.up_every; };
  // not 0: a hidden key's score is -inf, and has to stay that
  const float c = fmaxf(fabsf(a.attn_scale) * kLog2e, 1.17549435e-38f);

  // With two tiles the softmax threads hold a row of 128 scores each: 208 registers for them, 80 for the other warps
  // (256 x 208 + 128 x 80 = 63488 of the 384 x 168 = 64512 that the block is launched with).
  if (C::NQ == 2) {
    static_assert(C::NQ == 1 || (C::THREADS == 384 && 256 * 208 + 128 * 80 <= 384 * 168), "register split");
    if (warp < C::SOFT) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;\n");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
  }
  if (mine && warp < C::SOFT) {
    // =========================================================================================== softmax, epilogue
    const int i = warp >> 2;  // query tile
    const int row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t o_addr = tmem + C::O_COL + i * C::DV + lanes;
    const int t = row / G;
    const int tok = w.tok0 + i * T + t;
    const bool real = row < T * G && tok < w.s.lq;
    int lo = 0, up = 0;
    if (real) prompt_keys(a, w.s, tok, lo, up);
    float m = -INFINITY, l = 0.0f;
    bool ok = true;
    int n = 0;  // K / V tiles of this query tile so far
    int my0 = j0[0], my1 = j1[0];
    if (C::NQ == 2 && i == 1) {
      my0 = j0[C::NQ - 1];
      my1 = j1[C::NQ - 1];
    }
    for (int j = my0; j < my1 && ok; ++j, ++n) {
      const int buf = C::NSB == 2 ? (n & 1) : i;
      const uint32_t s_addr = tmem + C::S_COL + buf * C::S_STEP + lanes;
      ok = warp_wait_on(bar(B::S + buf), (C::NSB == 2 ? n >> 1 : n) & 1, stop);
      if (!ok) break;
      tc_fence_after();
      float s[C::BN];
#pragma unroll
      for (int x = 0; x < C::BN; x += 32) tmem_ld32(s_addr + x, reinterpret_cast<uint32_t*>(s) + x);
      tmem_wait_ld();
      const int k0 = j * C::BN;
      if (__any_sync(0xffffffffu, lo > k0 || up < k0 + C::BN)) {
        const int from = lo - k0, to = up - k0;
#pragma unroll
        for (int x = 0; x < C::BN; ++x) s[x] = x >= from && x < to ? s[x] : -INFINITY;
      }
      float mx;
      {
        float m0 = max3(s[0], s[1], s[0]), m1 = max3(s[2], s[3], s[2]), m2 = max3(s[4], s[5], s[4]), m3 = max3(s[6], s[7], s[6]);
#pragma unroll
        for (int x = 8; x < C::BN; x += 8) {
          m0 = max3(m0, s[x], s[x + 1]);
          m1 = max3(m1, s[x + 2], s[x + 3]);
          m2 = max3(m2, s[x + 4], s[x + 5]);
          m3 = max3(m3, s[x + 6], s[x + 7]);
        }
        mx = max3(max3(m0, m1, m2), m3, m3);
      }
      // a score that is no number makes the whole row none, through its sum (the polynomial below would lose it)
      if (mx != mx) l = mx;
      const bool raise = m == -INFINITY ? mx > -INFINITY : (mx - m) * c > kSlack;
      float scale = 1.0f;
      if (raise) {
        scale = m == -INFINITY ? 0.0f : ex2((m - mx) * c);
        m = mx;
        l *= scale;
      }
      if (n > 0 && __any_sync(0xffffffffu, raise)) {
        // O of the tiles before is complete once its MMA has arrived on O
        ok = warp_wait_on(bar(B::O + i), (n - 1) & 1, stop);
        if (!ok) break;
        tc_fence_after();
#pragma unroll 1
        for (int x = 0; x < C::DV; x += 16) {
          uint32_t o[16];
          tmem_ld16(o_addr + x, o);
          tmem_wait_ld();
#pragma unroll
          for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * scale);
          tmem_st16(o_addr + x, o);
        }
      }
      const float mc = m == -INFINITY ? 0.0f : m * c;
      uint64_t sum0 = pair(l, 0.0f), sum1 = 0;
      const uint64_t c2 = pair(c, c), mc2 = pair(-mc, -mc);
#pragma unroll
      for (int x = 0; x < C::BN; x += 32) {
        uint32_t p[16];
#pragma unroll
        for (int y = 0; y < 32; y += 2) {
          const uint64_t z = fma2(pair(s[x + y], s[x + y + 1]), c2, mc2);
          float2 e;
          if ((y >> 1) % 16 < 16 - C::POLY) {
            const float2 v = unpair(z);
            e = make_float2(ex2(v.x), ex2(v.y));
          } else {
            e = exp2_pair<DT>(z);
          }
          if (y & 2) sum1 = add2(sum1, pair(e.x, e.y));
          else sum0 = add2(sum0, pair(e.x, e.y));
          p[y >> 1] = pack2<DT>(e.x, e.y);
        }
        tmem_st16(s_addr + (x >> 1), p);
      }
      {
        const float2 v = unpair(add2(sum0, sum1));
        l = v.x + v.y;
      }
      // The epilogue's wait for the last output MMA must find the one before it complete (a barrier tells a phase from the
      // one before, not from the one before that).  With one S buffer the scores were issued behind it.
      if (C::NSB == 2 && n > 0 && j + 1 == my1) {
        ok = warp_wait_on(bar(B::O + i), (n - 1) & 1, stop);
        if (!ok) break;
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B::P + buf));
    }
    // ---- epilogue: the thread's row of O
    if (n > 0 && ok) ok = warp_wait_on(bar(B::O + i), (n - 1) & 1, stop);
    if (ok) {
      tc_fence_after();
      const float inv = up > lo ? 1.0f / l : 0.0f;
      const bool mend = s_scrubbed != 0;
      const int head = w.h * G + (row - t * G);
      const long long to = (static_cast<long long>(w.s.q0 + tok) * a.H_q + head) * D + half * C::DV;
#pragma unroll 1
      for (int x = 0; x < C::DV; x += 32) {
        uint32_t o[32];
        if (n > 0) {
          tmem_ld32(o_addr + x, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int y = 0; y < 32; ++y) o[y] = 0;
        }
        if (!real) continue;
        float f[32];
#pragma unroll
        for (int y = 0; y < 32; ++y) f[y] = up > lo ? __uint_as_float(o[y]) * inv : 0.0f;
        if (mend) {
          // infinities and NaN of tokens that this row sees, in tiles where they were taken out
          for (int key = lo; key < up; ++key) {
            if (!partly(key / C::BN)) {
              key = (key / C::BN + 1) * C::BN - 1;
              continue;
            }
            const uint32_t* src = reinterpret_cast<const uint32_t*>(
                static_cast<const uint16_t*>(a.v) + (w.s.k0 + static_cast<long long>(key)) * a.v_stride + w.h * D + half * C::DV + x);
#pragma unroll
            for (int y = 0; y < 32; y += 2) {
              const uint32_t v = __ldg(src + (y >> 1));
              if (not_finite2<DT>(v)) {
                const float2 g = unpack2<DT>(v);
                f[y] += g.x - g.x != 0.0f || g.x != g.x ? g.x : 0.0f;
                f[y + 1] += g.y - g.y != 0.0f || g.y != g.y ? g.y : 0.0f;
              }
            }
          }
        }
        if (OT == TQ_FP32) {
          float4* dst = reinterpret_cast<float4*>(static_cast<float*>(a.out) + to + x);
#pragma unroll
          for (int y = 0; y < 8; ++y) dst[y] = make_float4(f[4 * y], f[4 * y + 1], f[4 * y + 2], f[4 * y + 3]);
        } else {
          uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + to + x);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            dst[y] = make_uint4(pack2<DT>(f[8 * y], f[8 * y + 1]), pack2<DT>(f[8 * y + 2], f[8 * y + 3]),
                                pack2<DT>(f[8 * y + 4], f[8 * y + 5]), pack2<DT>(f[8 * y + 6], f[8 * y + 7]));
        }
      }
    }
  } else if (mine && warp == C::SOFT && lane == 0 && J1 > J0) {
    // ================================================================================================= TMA loads
    mbar_expect_tx(bar(B::Q), C::NQ * (D / 64) * T * G * 128);
    for (int i = 0; i < C::NQ; ++i)
      for (int x = 0; x < D / 64; ++x)
        tma_load_3d(base + i * C::QTILE + x * C::QCHUNK, &maps.q, 64 * x, w.h * G, w.s.q0 + w.tok0 + i * T, bar(B::Q));
    int slot = 0, issued = 0;
    uint32_t phase = 1;  // the first pass over the ring finds every slot empty
    bool ok = true;
    auto load = [&](const CUtensorMap* map, int j, int chunk0, int chunks) {
      ok = ok && wait_on(bar(B::EMPTY + slot), phase, stop);
      if (!ok) return;
      mbar_expect_tx(bar(B::FULL + slot), chunks * C::KCHUNK);
      for (int x = 0; x < chunks; ++x)
        tma_load_3d(base + C::RING + slot * C::SLOT + x * C::KCHUNK, map, 64 * (chunk0 + x), w.h, w.s.k0 + j * C::BN, bar(B::FULL + slot));
      ++issued;
      if (++slot == C::NS) {
        slot = 0;
        phase ^= 1;
      }
    };
    // in the order in which the MMAs take them
    for (int j = J0; j <= J1 && ok; ++j) {
      if (C::NSB == 2) {
        if (j < J1) load(&maps.k, j, 0, D / 64);
        if (j > J0) load(&maps.v, j - 1, half * (C::DV / 64), C::DV / 64);
      } else {
        if (j > J0) load(&maps.v, j - 1, 0, C::DV / 64);
        if (j < J1) load(&maps.k, j, 0, D / 64);
      }
    }
    if (!ok) {
      // copies on their way land before the block ends (bounded again)
      wait_stage(bar(B::Q), 0);
      for (int x = 0; x < C::NS && x < issued; ++x) {
        const int n = issued - 1 - x;
        wait_stage(bar(B::FULL + n % C::NS), (n / C::NS) & 1);
      }
    }
  } else if (mine && warp == C::SOFT + 1 && lane == 0 && J1 > J0) {
    // ====================================================================================================== MMAs
    const uint32_t id_s = instr_desc(DT == TQ_BF16, 128, C::BN, false) | (a.attn_scale < 0.0f ? kNegateA : 0u);
    const uint32_t id_o = instr_desc(DT == TQ_BF16, 128, C::DV, true);
    int slot = 0, scrubs = 0, n[C::NQ];
    uint32_t phase = 0;
    for (int i = 0; i < C::NQ; ++i) n[i] = 0;
    const uint32_t q_lo = desc_lo(base, 0), ring_lo = desc_lo(base + C::RING, 0);
    bool ok = wait_on(bar(B::Q), 0, stop);
    int issued[C::NQ];  // S tiles
    for (int i = 0; i < C::NQ; ++i) issued[i] = 0;
    auto next_slot = [&]() {
      mma_commit(bar(B::EMPTY + slot));
      if (++slot == C::NS) {
        slot = 0;
        phase ^= 1;
      }
    };
    auto scores = [&](int i, uint32_t k_at) {
      const int buf = C::NSB == 2 ? (issued[i] & 1) : i;
      const uint32_t d = tmem + C::S_COL + buf * C::S_STEP;
#pragma unroll
      for (int x = 0; x < D / 16; ++x)
        mma_ss(d, q_lo + i * (C::QTILE >> 4) + (((x >> 2) * C::QCHUNK + (x & 3) * 32) >> 4),
               k_at + (((x >> 2) * C::KCHUNK + (x & 3) * 32) >> 4), kDescHi, id_s, x > 0);
      mma_commit(bar(B::S + buf));
      ++issued[i];
    };
    auto outputs = [&](int i, uint32_t v_at) {
      const int buf = C::NSB == 2 ? (n[i] & 1) : i;
      ok = ok && wait_on(bar(B::P + buf), (C::NSB == 2 ? n[i] >> 1 : n[i]) & 1, stop);
      if (!ok) return;
      tc_fence_after();
      const uint32_t p = tmem + C::S_COL + buf * C::S_STEP, d = tmem + C::O_COL + i * C::DV;
#pragma unroll
      for (int x = 0; x < C::BN / 16; ++x) mma_ts(d, p + 8 * x, v_at + (2048 >> 4) * x, kDescHi, id_o, x > 0 || n[i] > 0);
      mma_commit(bar(B::O + i));
      ++n[i];
    };
    auto take = [&]() {  // the next slot's tile has landed
      ok = ok && wait_on(bar(B::FULL + slot), phase, stop);
      return ring_lo + slot * (C::SLOT >> 4);
    };
    auto take_v = [&](int j) {
      const uint32_t x = take() + ((C::KCHUNK >> 4) << 16);
      if (ok && partly(j)) {
        mbar_arrive(bar(B::ASK));
        ok = wait_on(bar(B::SCRUB), scrubs++ & 1, stop);
      }
      return x;
    };
    for (int j = J0; j <= J1 && ok; ++j) {
      if (C::NSB == 2) {
        if (j < J1) {
          const uint32_t x = take();
          if (!ok) break;
          scores(0, x);
          next_slot();
        }
        if (j > J0) {
          const uint32_t x = take_v(j - 1);
          if (!ok) break;
          outputs(0, x);
          if (!ok) break;
          next_slot();
        }
      } else {
        // tile 0: its weights times V(j - 1), its scores against K(j); then tile 1
        uint32_t v_at = 0, k_at = 0;
        const int v_slot = slot;
        if (j > J0) {
          v_at = take_v(j - 1);
          if (!ok) break;
          if (++slot == C::NS) {
            slot = 0;
            phase ^= 1;
          }
        }
        const int k_slot = slot;
        bool have_k = false;
        for (int i = 0; i < C::NQ && ok; ++i) {
          if (j > J0 && in(i, j - 1)) outputs(i, v_at);
          if (ok && j < J1 && in(i, j)) {
            if (!have_k) k_at = take();
            have_k = true;
            if (ok) scores(i, k_at);
          }
        }
        if (!ok) break;
        if (j > J0) mma_commit(bar(B::EMPTY + v_slot));
        if (j < J1) {
          mma_commit(bar(B::EMPTY + k_slot));
          if (++slot == C::NS) {
            slot = 0;
            phase ^= 1;
          }
        }
      }
    }
    // everything issued has completed before the block gives its memory back
    mma_commit(bar(B::DRAIN));
    if (!wait_stage(bar(B::DRAIN), 0, kTileWait)) *stop = 1;
  } else if (mine && warp >= C::SOFT + 2) {
    // ============================================================= V tiles that some row sees in part: finite values
    const int me = tid - 32 * (C::SOFT + 2);
    bool ok = true;
    int asked = 0;
    for (int j = J0; j < J1 && ok; ++j) {
      if (!partly(j)) continue;
      // the MMA thread asks when it has come to the tile, and holds its slot until the answer
      ok = warp_wait_on(bar(B::ASK), asked++ & 1, stop, kBlockWait);
      if (!ok) break;
      // K(J0) [K(J0+1)] V(J0) K V ...: V(j) is load 2 (j - J0) + 1, or one later where the next K tile is loaded first
      const int order = 2 * (j - J0) + 1 + (C::NSB == 2 && j + 1 < J1 ? 1 : 0);
      const int slot = order % C::NS;
      ok = warp_wait_on(bar(B::FULL + slot), (order / C::NS) & 1, stop);
      if (!ok) break;
      uint4* tile = reinterpret_cast<uint4*>(smem + C::RING + slot * C::SLOT);
      bool found = false;
#pragma unroll 4
      for (int x = me; x < (C::DV / 64) * C::KCHUNK / 16; x += 32 * C::SCRUB) {
        uint4 v = tile[x];
        if (not_finite2<DT>(v.x) | not_finite2<DT>(v.y) | not_finite2<DT>(v.z) | not_finite2<DT>(v.w)) {
          auto clean = [](uint32_t y) {
            const uint32_t bad = not_finite2<DT>(y);
            return y & ~((bad >> 15) * 0xffffu);
          };
          tile[x] = make_uint4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
          found = true;
        }
      }
      if (found) s_scrubbed = 1;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B::SCRUB));
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == C::SOFT + 1) tmem_free(tmem, 512);
  if (tid == 0 && s_stop && a.status) atomicOr(a.status, TQ_STATUS_TIMEOUT);
}

// ---- host

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return static_cast<EncodeFn>(nullptr);
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// [rows][heads][d] 16-bit values, rows `stride` elements apart, boxes of 64 channels x `heads_box` x `rows_box`
bool make_map(CUtensorMap* map, const void* p, int dtype, int d, int heads, long long rows, long long stride, int heads_box,
              int rows_box) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d) * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(heads_box), static_cast<cuuint32_t>(rows_box)};
  const cuuint32_t ones[3] = {1, 1, 1};
  return encode_fn()(map, dtype == TQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                     const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int DT, int OT>
cudaError_t launch_dto(const PromptArgs& a, cudaStream_t st) {
  using C = Cfg<D>;
  auto* kernel = prompt_kernel<D, DT, OT>;
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit) || !bit) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM)) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  const int G = a.H_q / a.H_kv, T = 128 / G;
  const long long blocks = (static_cast<long long>(a.n_q) / (C::NQ * T) + a.B) * a.H_kv * (D / C::DV);
  if (!encode_fn() || blocks > 0x7fffffffLL) return cudaErrorNotSupported;
  Maps maps;
  if (!make_map(&maps.q, a.q, a.dtype, D, a.H_q, a.n_q, a.q_stride, G, T) ||
      !make_map(&maps.k, a.k, a.dtype, D, a.H_kv, a.n_kv, a.k_stride, 1, C::BN) ||
      !make_map(&maps.v, a.v, a.dtype, D, a.H_kv, a.n_kv, a.v_stride, 1, C::BN))
    return cudaErrorInvalidValue;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(blocks)), dim3(C::THREADS), C::SMEM, st, maps, a, G, T);
}

template <int D>
cudaError_t launch_d(const PromptArgs& a, cudaStream_t st) {
  if (a.dtype == TQ_BF16) return a.out_dtype == TQ_FP32 ? launch_dto<D, TQ_BF16, TQ_FP32>(a, st) : launch_dto<D, TQ_BF16, TQ_BF16>(a, st);
  return a.out_dtype == TQ_FP32 ? launch_dto<D, TQ_FP16, TQ_FP32>(a, st) : launch_dto<D, TQ_FP16, TQ_FP16>(a, st);
}

}  // namespace

cudaError_t launch_prompt(const PromptArgs& a, cudaStream_t st) {
  switch (a.d) {
    case 64: return launch_d<64>(a, st);
    case 128: return launch_d<128>(a, st);
    case 256: return launch_d<256>(a, st);
    default: return launch_d<512>(a, st);
  }
}

}  // namespace tq

// Attention of packed prompts on the tensor cores (tcgen05, TMEM, TMA): tq_sdpa_prompt.
//
// A tile is 128 query rows of one KV head: T = 128 / G tokens times the G query heads that share the head, token by
// token, so K and V are read once per KV head whatever G is.  A thread block works on NQ tiles over a common stream of
// K / V tiles of BN keys:
//     S = Q K^T   (tcgen05.mma, both operands in shared memory, S in TMEM)
//     P = 2^(c S - c m + e), rounded to 16 bits, back into TMEM over S   (a thread per row, online softmax)
//     O += P V    (A operand P from TMEM, V as it lies in memory: rows along K)
// c = alpha log2 e > 0 (for a negative alpha the MMA negates Q).  m is raised only when a score exceeds it by more than
// 2^12 (bf16) or 2^7.9 (fp16); then the thread rescales its row of O in TMEM.  The row sums are of unrounded weights, in
// fp32.  A bf16 weight is rounded by 2^-8 of itself; e = -20, so that a million values near the largest number do not
// overflow in O (an e of 0 left room for none).  In fp16 weights stay below 2^15 with e = 7, which puts its subnormals
// as low as that allows: rounded by 2^-11 of itself, or by 2^-32 of the largest weight (with 2^12 and e = 0 by 2^-25: a
// token of weight 2^-22.5 was off by 6 %).  The sooner raising costs fp16 1 % (8K) to 5 % (d = 256, window 1024).
// S has two buffers per tile: the scores of the next keys are made while the softmax of these runs.  That takes key
// tiles of 64 (two tiles, two buffers and two outputs are all of TMEM at d = 128), for which an MMA of 128 x 64 x 16
// reads its operands in 48 cycles instead of the 32 that it computes; with tiles of 128 keys and one buffer the MMAs are
// faster (64 cycles for twice the work), but outputs, scores and softmax of a tile follow one another: 1.09 ms for the
// 8K prompt.  At d = 512 the accumulator of a row does not fit TMEM: a thread block computes 256 of the 512 output
// channels, and S is computed twice.
//
// NQ is 2 at d <= 128 and 1 above (TMEM).  A launch of so few tiles that every one finds an SM of its own takes one tile
// per thread block at any d: a step of 64 keys is then 0.6 to 0.8 us instead of 0.9 (16 sequences of up to 300 tokens,
// 4 heads on 1: 8.5 us instead of 9.9; one KV head, 1211 tokens, window 100: 8.1 instead of 11.8).  With more tiles than
// SMs two per thread block share what they read: 12.4 us instead of 14.2 at 4076 tokens, 8 heads on 1, window 100.
//
// Roles: one warpgroup of softmax threads per tile; a warp that finds the work and issues the TMA loads; a warp per tile
// that issues its MMAs (one issuing thread could not keep the tensor cores busy over its waits); one or two warps that
// look through the V tiles which some row sees in part.  Those may hold tokens of a neighbouring sequence or of the row's
// future, whose weight is 0, and 0 * inf is not 0: a value there that is no finite number is replaced by 0 in shared
// memory, and the rows that do see it get it added back in the epilogue from global memory.
//
// A thread block starts with the tile of its own index and then takes over thread blocks of the grid that have not
// started (cluster launch control), so the loads and the first scores of the next tile run under the last softmax and the
// epilogue of this one, and tiles of very different cost (causal masks, ragged lengths) even out.
//
// What bounds it, d = 128, per 64 keys of two tiles: the exponential unit 1024 cycles (16 per cycle and SM), the tensor
// cores 2 x (8 x 48 + 4 x 64) = 1280 with their operands from shared memory; a step takes 1540, and a
// hand-over of S and P costs 250 of latency that two tiles do not quite hide.  The 8K prompt (64 heads on 8): 1.03 to
// 1.1 ms, 1.0 to 1.07 PFLOP/s, at the card's power limit (1.65 GHz).  Ragged prompts of 256 to 2048 tokens: 0.75 to
// 0.84 PFLOP/s; there an epilogue of 1500 (d = 64) to 2900 cycles comes every 2 to 32 steps.
#include <cuda.h>

#include "tq_async.cuh"
#include "tq_kv8.cuh"
#include "tq_prompt.cuh"
#include "tq_tcgen05.cuh"

namespace tq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// Log2 units that a score may exceed the running maximum, and log2 of the weight of a score as large as it (see the top).
// From kFar on, the rounding of c m (2^-25 of it, the same for all weights of the row) could take weights out of their
// type.  There the power of two below c stands in its place, whose product with m is exact: the scores themselves are
// then 0.5 (fp16) or 64 (bf16) log2 units apart, so what decides is which of them are equal to the largest.  (There the
// sum of -c m and kRaise is rounded, and the 7 of fp16 becomes 8 at most: with 7.9 weights stay below 2^16.)
template <int DT>
struct Weights {
  static constexpr float kSlack = DT == TQ_BF16 ? 12.0f : 7.9f;
  static constexpr float kRaise = DT == TQ_BF16 ? -20.0f : 7.0f;
  static constexpr float kFar = DT == TQ_BF16 ? 1073741824.0f : 8388608.0f;  // 2^30, 2^23
};

template <int D, int TILES>
struct Cfg {
  static constexpr int D_ = D;
  static constexpr int NQ = TILES;                    // query tiles of a thread block
  static constexpr int BN = D <= 256 ? 64 : 32;       // keys of a K / V tile
  static constexpr int DV = D <= 256 ? D : 256;       // output channels of a thread block
  static constexpr int SOFT = 4 * NQ;                 // softmax warps
  static constexpr int SCRUB = NQ == 2 ? 1 : 2;
  static constexpr int WARPS = SOFT + 1 + NQ + SCRUB;  // softmax | work and TMA | MMA | scrub
  static constexpr int THREADS = 32 * WARPS;
  static constexpr int QCHUNK = 128 * 128;            // bytes of 128 rows x 64 channels
  static constexpr int QTILE = (D / 64) * QCHUNK;
  static constexpr int KCHUNK = BN * 128;
  static constexpr int KT = (D / 64) * KCHUNK;        // K tile
  static constexpr int VT = (DV / 64) * KCHUNK;       // V tile
  static constexpr int STAGE = KT + VT;               // what step j reads: K(j) for its scores, V(j - 1) for its outputs
  static constexpr int NS = D == 64 ? 8 : (D == 128 ? 4 : 2);
  static constexpr int RING = NQ * QTILE;
  static constexpr int OUT = RING + NS * STAGE;       // output rows on their way out, 4 KB per softmax warp
  static constexpr bool STAGED = D <= 256;            // (no room at d = 512)
  static constexpr int BARS = OUT + (STAGED ? SOFT * 4096 : 0);
  static constexpr int SMEM = BARS + 512 + 1024;      // barriers, and room to align the base
  static constexpr int O_COL = 2 * NQ * BN;           // TMEM columns: two S buffers per query tile (P over S), O behind
  static_assert(O_COL + NQ * DV <= 512, "tensor memory");
  static_assert(SMEM <= 232448, "shared memory");
};

struct Maps {
  CUtensorMap q, k, v, o;
};

// mbarriers of a thread block, 8 bytes each
template <typename C>
struct Bars {
  static constexpr int FULL = 0, EMPTY = FULL + C::NS, READY = EMPTY + C::NS;  // stages: landed, free, looked through
  static constexpr int Q = READY + C::NS, Q_FREE = Q + 1;
  static constexpr int S = Q_FREE + 1, P = S + 2 * C::NQ, O = P + 2 * C::NQ;  // scores and weights (two buffers), outputs
  static constexpr int WORK = O + C::NQ, WORK_FREE = WORK + 2, STEAL = WORK_FREE + 2, DRAIN = STEAL + 1, COUNT = DRAIN + 1;
  static_assert(COUNT * 8 <= 512, "room for the barriers");
};

// Bounded wait that also gives up when another warp of the thread block has: false, and the block winds down.  (Inline:
// registers cannot be moved between warps, as the kernel does, around a function call.)
constexpr long long kTileWait = 16 * kMaxWaitCycles;  // 35 ms: a wait may span some other role's work on a few tiles
constexpr long long kBlockWait = 1LL << 34;           // 9 s: a wait for the next piece of work may span a whole sequence
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
__device__ __forceinline__ bool wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_slow(bar, parity, stop, limit);
}
__device__ __forceinline__ bool wait_stage_inline(uint32_t bar, uint32_t parity, long long limit) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > limit) return false;
  return true;
}
// the same for a whole warp: all its lanes go on, or none
__device__ __forceinline__ bool warp_wait_on(uint32_t bar, uint32_t parity, volatile int* stop, long long limit) {
  return __all_sync(0xffffffffu, wait_on(bar, parity, stop, limit));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {  // NaN if one of them is
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// nonzero if one of the two 16-bit values of a word is an infinity or a NaN
template <int DT>
__device__ __forceinline__ uint32_t not_finite2(uint32_t w) {
  return ((w & 0x7fff7fffu) + (DT == TQ_BF16 ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}

// One piece of work, the same for all warps: NQ tiles of a sequence and a KV head.
struct Work {
  PromptSeq s;
  int h, half;  // KV head; half of the output channels (d = 512)
  int tok0;     // first query token of tile 0
  int more;     // 0: there is none
};

// Key tiles of a piece of work: [j0, j1) of each query tile, [J0, J1) of all; the keys that every query sees are
// [lo, up).
template <typename C>
struct Span {
  int j0[C::NQ], j1[C::NQ], J0, J1, lo, up;
  __device__ Span(const PromptArgs& a, const Work& w, int T) : J0(0), J1(0) {
    int x, y;
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) {
      const int first = w.tok0 + i * T, last = min(first + T, w.s.lq) - 1;
      j0[i] = j1[i] = 0;
      if (last < first) continue;
      int lo1, up1;
      prompt_keys(a, w.s, first, x, y);
      prompt_keys(a, w.s, last, lo1, up1);
      j0[i] = x / C::BN;
      j1[i] = (up1 + C::BN - 1) / C::BN;
      if (j1[i] <= j0[i]) continue;
      J0 = J1 == J0 ? j0[i] : min(J0, j0[i]);
      J1 = max(J1, j1[i]);
    }
    prompt_keys(a, w.s, w.tok0, x, up);
    prompt_keys(a, w.s, min(w.tok0 + C::NQ * T, w.s.lq) - 1, lo, y);
  }
  __device__ bool in(int i, int j) const { return j >= j0[i] && j < j1[i]; }
  __device__ bool partly(int j) const { return j * C::BN < lo || (j + 1) * C::BN > up; }
};

// Instrumented instantiation only (the library's own tests, see TestHooks): limit of the waits for a tile in SM cycles, and the
// key tile whose loads announce 16 bytes too many: their barrier never completes, the data lands.
struct Hook {
  int wait_cycles, fault_tile;
};

template <int D, int NQ, int DT, int OT, bool TEST>
__global__ void __launch_bounds__(Cfg<D, NQ>::THREADS, 1) prompt_kernel(const __grid_constant__ Maps maps, const PromptArgs a,
                                                                    int G, int T, const Hook hook) {
  using C = Cfg<D, NQ>;
  using B = Bars<C>;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(16) uint4 s_answer;
  __shared__ Work s_work[2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_stop, s_scrubbed[4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
  uint8_t* const smem = raw + (base - smem_addr(raw));
  const uint32_t bars = base + C::BARS;
  auto bar = [&](int i) { return bars + 8 * i; };
  volatile int* const stop = &s_stop;
  const long long tile_wait = TEST ? hook.wait_cycles : kTileWait;

  if (warp == C::SOFT + 1) tmem_alloc(smem_addr(&s_tmem), 512);
  if (tid == 0) {
    for (int i = 0; i < C::NS; ++i) {
      mbar_init(bar(B::FULL + i), 1);
      mbar_init(bar(B::EMPTY + i), C::NQ + C::SCRUB);
      mbar_init(bar(B::READY + i), C::SCRUB);
    }
    mbar_init(bar(B::Q), 1);
    mbar_init(bar(B::Q_FREE), C::NQ);
    for (int i = 0; i < 2 * C::NQ; ++i) {
      mbar_init(bar(B::S + i), 1);
      mbar_init(bar(B::P + i), 4);
    }
    for (int i = 0; i < C::NQ; ++i) mbar_init(bar(B::O + i), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B::WORK + i), 1);
      mbar_init(bar(B::WORK_FREE + i), C::WARPS - 1);
    }
    mbar_init(bar(B::STEAL), 1);
    mbar_init(bar(B::DRAIN), C::NQ);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    s_stop = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  pdl_launch_dependents();
  pdl_wait();

  // With two tiles there are 384 threads of 168 registers; the softmax threads take 208 of them and leave 80 to the others
  // (256 x 208 + 128 x 80 = 63488 of 64512).
  if (C::NQ == 2) {
    static_assert(C::NQ == 1 || (C::THREADS == 384 && 256 * 208 + 128 * 80 <= 384 * 168), "register split");
    if (warp < C::SOFT) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;\n");
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
  }

  // the it-th piece of work, for every warp but the one that finds it; false: none, or the block winds down
  auto next_work = [&](int it, Work& w) {
    if (!warp_wait_on(bar(B::WORK + (it & 1)), (it >> 1) & 1, stop, kBlockWait)) return false;
    w = s_work[it & 1];
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(B::WORK_FREE + (it & 1)));
    return w.more != 0;
  };

  if (warp < C::SOFT) {
    // =========================================================================================== softmax, epilogue
    const int i = warp >> 2;  // query tile
    const int row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t o_addr = tmem + C::O_COL + i * C::DV + lanes;
    const int t = row / G;
    // not 0: a hidden key's score is -inf, and has to stay that (but a NaN stays one)
    const float c = max3(fabsf(a.attn_scale) * kLog2e, 1.17549435e-38f, 1.17549435e-38f);
    bool ok = true;
    uint32_t total = 0, out = 0;  // K / V tiles of this query tile, and arrivals on its outputs, in all work so far
    Work w;
    for (int it = 0; ok && next_work(it, w); ++it) {
      const Span<C> r(a, w, T);
      const int tok = w.tok0 + i * T + t;
      const bool real = row < T * G && tok < w.s.lq;
      int lo = 0, up = 0;
      if (real) prompt_keys(a, w.s, tok, lo, up);
      float m = -INFINITY, l = 0.0f;
      int n = 0;  // K / V tiles of this work
      const int my0 = i == 0 ? r.j0[0] : r.j0[C::NQ - 1], my1 = i == 0 ? r.j1[0] : r.j1[C::NQ - 1];
      // The outputs of the tiles before j are complete once the scores of tile j + 1 are (their MMAs are issued behind);
      // the last two outputs of a piece of work arrive on a barrier of their own.
      auto outputs_before = [&](int j, uint32_t use) {
        if (j + 1 < my1) return warp_wait_on(bar(B::S + 2 * i + ((use + 1) & 1)), ((use + 1) >> 1) & 1, stop, tile_wait);
        return warp_wait_on(bar(B::O + i), out & 1, stop, tile_wait);
      };
      for (int j = my0; j < my1 && ok; ++j, ++n) {
        const uint32_t use = total + n;
        const int buf = 2 * i + (use & 1);
        const uint32_t s_addr = tmem + buf * C::BN + lanes;
        ok = warp_wait_on(bar(B::S + buf), (use >> 1) & 1, stop, tile_wait);
        if (!ok) break;
        tc_fence_after();
        float s[C::BN];
#pragma unroll
        for (int x = 0; x < C::BN; x += 32) tmem_ld32(s_addr + x, reinterpret_cast<uint32_t*>(s) + x);
        tmem_wait_ld();
        const int k0 = j * C::BN;
        if (__any_sync(0xffffffffu, up < k0 + C::BN)) {
          const int to = up - k0;
#pragma unroll
          for (int x = 0; x < C::BN; ++x) s[x] = x < to ? s[x] : -INFINITY;
        }
        if (__any_sync(0xffffffffu, lo > k0)) {
          const int from = lo - k0;
#pragma unroll
          for (int x = 0; x < C::BN; ++x) s[x] = x >= from ? s[x] : -INFINITY;
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
        // a score that is no number makes the whole row none, through its sum
        if (mx != mx) l = mx;
        const bool raise = m == -INFINITY ? mx > -INFINITY : (mx - m) * c > Weights<DT>::kSlack;
        float scale = 1.0f;
        if (raise) {
          scale = m == -INFINITY ? 0.0f : ex2((m - mx) * c);
          m = mx;
          l *= scale;
        }
        if (n > 0 && __any_sync(0xffffffffu, raise)) {
          ok = outputs_before(j, use);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int x = 0; x < C::DV; x += 64) {
            uint32_t o[64];
            tmem_ld32(o_addr + x, o);
            tmem_ld32(o_addr + x + 32, o + 32);
            tmem_wait_ld();
#pragma unroll
            for (int y = 0; y < 64; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * scale);
            tmem_st32(o_addr + x, o);
            tmem_st32(o_addr + x + 32, o + 32);
          }
        }
        const float cm = fabsf(m) * c > Weights<DT>::kFar ? __uint_as_float(__float_as_uint(c) & 0xff800000u) : c;
        const float shift = m == -INFINITY ? 0.0f : __fmaf_rn(-m, cm, Weights<DT>::kRaise);
        uint64_t sum0 = pair(l, 0.0f), sum1 = 0;
        const uint64_t c2 = pair(cm, cm), shift2 = pair(shift, shift);
#pragma unroll
        for (int x = 0; x < C::BN; x += 32) {
          uint32_t p[16];
#pragma unroll
          for (int y = 0; y < 32; y += 2) {
            const float2 z = unpair(fma2(pair(s[x + y], s[x + y + 1]), c2, shift2));
            const float e0 = ex2(z.x), e1 = ex2(z.y);
            if (y & 2) sum1 = add2(sum1, pair(e0, e1));
            else sum0 = add2(sum0, pair(e0, e1));
            p[y >> 1] = pack2<DT>(e0, e1);
          }
          tmem_st16(s_addr + (x >> 1), p);
        }
        {
          const float2 v = unpair(add2(sum0, sum1));
          l = v.x + v.y;
        }
        // The epilogue's wait for the last outputs must find those before them complete: a barrier tells a phase from the
        // one before, not from the one before that.
        if (n > 0 && j + 1 == my1) {
          ok = outputs_before(j, use);
          if (!ok) break;
          ++out;
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B::P + buf));
      }
      total += n;
      // ---- epilogue: the thread's row of O
      if (n > 0 && ok) ok = warp_wait_on(bar(B::O + i), out++ & 1, stop, tile_wait);
      if (ok) {
        tc_fence_after();
        const float inv = up > lo ? 1.0f / l : 0.0f;
        const bool mend = s_scrubbed[it & 3] != 0;
        const int head = w.h * G + (row - t * G);
        const long long to = (static_cast<long long>(w.s.q0 + tok) * a.H_q + head) * D + w.half * C::DV;
        // 32 channels of the row, from x on
        auto channels = [&](int x, float (&f)[32]) {
          uint32_t o[32];
          if (n > 0) {
            tmem_ld32(o_addr + x, o);
            tmem_wait_ld();
          }
#pragma unroll
          for (int y = 0; y < 32; ++y) f[y] = up > lo ? __uint_as_float(o[y]) * inv : 0.0f;
          if (!mend) return;
          // infinities and NaN of tokens that this row sees, in tiles where they were taken out
          for (int key = lo; key < up; ++key) {
            if (!r.partly(key / C::BN)) {
              key = (key / C::BN + 1) * C::BN - 1;
              continue;
            }
            const uint32_t* src = reinterpret_cast<const uint32_t*>(
                static_cast<const uint16_t*>(a.v) + (w.s.k0 + static_cast<long long>(key)) * a.v_stride + w.h * D + w.half * C::DV + x);
#pragma unroll
            for (int y = 0; y < 32; y += 2) {
              const uint32_t v = __ldg(src + (y >> 1));
              if (not_finite2<DT>(v)) {
                const float2 g = unpack2<DT>(v);
                f[y] += g.x - g.x != 0.0f ? g.x : 0.0f;  // (true of an infinity and of a NaN)
                f[y + 1] += g.y - g.y != 0.0f ? g.y : 0.0f;
              }
            }
          }
        };
        // 16 bytes of the output row from channel y of f on
        constexpr int kEach = OT == TQ_FP32 ? 4 : 8;
        auto bytes16 = [&](const float (&f)[32], int y) {
          if (OT == TQ_FP32)
            return make_uint4(__float_as_uint(f[y]), __float_as_uint(f[y + 1]), __float_as_uint(f[y + 2]), __float_as_uint(f[y + 3]));
          return make_uint4(pack2<DT>(f[y], f[y + 1]), pack2<DT>(f[y + 2], f[y + 3]), pack2<DT>(f[(y + 4) & 31], f[(y + 5) & 31]),
                            pack2<DT>(f[(y + 6) & 31], f[(y + 7) & 31]));
        };
        constexpr long long kSize = OT == TQ_FP32 ? 4 : 2;
        uint8_t* const dst = static_cast<uint8_t*>(a.out) + to * kSize;
        if constexpr (C::STAGED) {
          // Through shared memory, 128 bytes of the warp's 32 rows at a time: straight from the registers every store would
          // touch 32 rows (8700 cycles for 128 rows of 256 channels).  16-byte piece p of row r lies at p ^ (r % 8), as a
          // tensor map with a 128-byte swizzle has it.  With two tiles, whose warps are in each other's way, one TMA store
          // takes the 128 bytes out where the rows are whole tokens of the sequence (6 sequences of 67 to 539 tokens, 128
          // heads on 16: 51.7 us instead of 57.1); a single tile gains nothing from it (12 short sequences, d = 256: 13.6
          // instead of 12.8).
          constexpr int kCols = 128 / kSize;
          constexpr bool kTma = C::NQ == 2;
          uint4* const area = reinterpret_cast<uint4*>(smem + C::OUT + warp * 4096);
          const unsigned valid = __ballot_sync(0xffffffffu, real);
          const bool whole = kTma && valid == 0xffffffffu && (32 % G) == 0;
          const int sub = lane >> 3, piece = lane & 7;
          uint8_t* rows[8];
#pragma unroll
          for (int y = 0; y < 8; ++y)
            rows[y] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), 4 * y + sub)) + 16 * piece;
#pragma unroll 1
          for (int x = 0; x < C::DV; x += kCols) {
#pragma unroll
            for (int z = 0; z < kCols; z += 32) {
              float f[32];
              channels(x + z, f);
              if (kTma && z == 0) {
                if (lane == 0) bulk_wait_read<0>();
                __syncwarp();
              }
#pragma unroll
              for (int y = 0; y < 32; y += kEach) area[8 * lane + (((z + y) / kEach) ^ (lane & 7))] = bytes16(f, y);
            }
            if (whole) {
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) {
                tma_store_3d(&maps.o, w.half * C::DV + x, w.h * G, w.s.q0 + tok, base + C::OUT + warp * 4096);
                bulk_commit();
              }
              continue;
            }
            __syncwarp();
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              const int from = 4 * y + sub;
              if (valid >> from & 1) *reinterpret_cast<uint4*>(rows[y] + x * kSize) = area[8 * from + (piece ^ (from & 7))];
            }
            __syncwarp();
          }
        } else {
#pragma unroll 1
          for (int x = 0; x < C::DV; x += 32) {
            float f[32];
            channels(x, f);
            if (real)
#pragma unroll
              for (int y = 0; y < 32; y += kEach) *reinterpret_cast<uint4*>(dst + (x + y) * kSize) = bytes16(f, y);
          }
        }
        tc_fence_before();
      }
    }
    tmem_wait_st();  // (weights that were on their way when a wait ran out: before the block gives its memory back)
    if (C::NQ == 2 && lane == 0) bulk_wait_read<0>();  // shared memory stays until it is read
  } else if (warp == C::SOFT) {
    // ====================================================================================== the work, and TMA loads
    if (lane == 0) {
      const int TT = C::NQ * T, halves = D / C::DV;
      // Tiles of a sequence: b starts at tile start_of(b) = q_offsets[b] / TT + b, which leaves room for its ceil(lq / TT) tiles.  The late
      // tiles of a sequence see the most keys under the causal mask and go first.
      int id = blockIdx.x, it = 0, stage = 0, q_uses = 0;
      uint32_t phase = 1, issued = 0;  // the first pass over the ring finds every stage empty
      bool ok = true;
      for (int asked = 0; ok; ++asked) {
        Work w = {};
        if (id >= 0) {
          int at = id;
          w.half = at % halves;
          at /= halves;
          w.h = at % a.H_kv;
          const int tile = a.n_q / TT + a.B - 1 - at / a.H_kv;
          int b = 0;  // the last sequence with start_of(b) <= tile, that is q_offsets[b] < (tile - b + 1) TT
          for (int hi = a.B; hi - b > 1;) {
            const int mid = (b + hi) >> 1;
            if (min(max(a.q_offsets[mid], 0), a.n_q) < (tile - mid + 1LL) * TT) b = mid;
            else hi = mid;
          }
          w.s = prompt_seq(a, b, false);
          w.tok0 = (tile - w.s.q0 / TT - b) * TT;
          w.more = w.tok0 >= 0 && w.tok0 < w.s.lq;
          if (w.more && w.tok0 == 0 && w.h == 0 && w.half == 0) (void)prompt_seq(a, b, true);  // one reports for the sequence
        }
        if (w.more || id < 0) {
          ok = wait_on(bar(B::WORK_FREE + (it & 1)), ((it >> 1) & 1) ^ 1, stop, kBlockWait);
          if (ok) {
            s_work[it & 1] = w;
            s_scrubbed[it & 3] = 0;  // its readers of four pieces of work ago have long gone on
            mbar_arrive(bar(B::WORK + (it & 1)));
            ++it;
          }
        }
        if (w.more && ok) {
          const Span<C> r(a, w, T);
          if (r.J1 > r.J0) {
            ok = wait_on(bar(B::Q_FREE), (q_uses & 1) ^ 1, stop, tile_wait);
            if (ok) {
              ++q_uses;
              mbar_expect_tx(bar(B::Q), C::NQ * (D / 64) * T * G * 128);
              for (int i = 0; i < C::NQ; ++i)
                for (int x = 0; x < D / 64; ++x)
                  tma_load_3d(base + i * C::QTILE + x * C::QCHUNK, &maps.q, 64 * x, w.h * G, w.s.q0 + w.tok0 + i * T, bar(B::Q));
            }
            for (int j = r.J0; j <= r.J1 && ok; ++j) {
              ok = wait_on(bar(B::EMPTY + stage), phase, stop, tile_wait);
              if (!ok) break;
              const uint32_t to = base + C::RING + stage * C::STAGE, full = bar(B::FULL + stage);
              mbar_expect_tx(full, (j < r.J1 ? C::KT : 0) + (j > r.J0 ? C::VT : 0) + (TEST && j == hook.fault_tile ? 16 : 0));
              if (j < r.J1)
                for (int x = 0; x < D / 64; ++x) tma_load_3d(to + x * C::KCHUNK, &maps.k, 64 * x, w.h, w.s.k0 + j * C::BN, full);
              if (j > r.J0)
                for (int x = 0; x < C::DV / 64; ++x)
                  tma_load_3d(to + C::KT + x * C::KCHUNK, &maps.v, w.half * C::DV + 64 * x, w.h, w.s.k0 + (j - 1) * C::BN, full);
              ++issued;
              if (++stage == C::NS) {
                stage = 0;
                phase ^= 1;
              }
            }
          }
        }
        if (id < 0 || !ok) break;
        // asked only now, so that no thread block sits on work that another one is free for
        mbar_expect_tx(bar(B::STEAL), 16);
        steal_ask(smem_addr(&s_answer), bar(B::STEAL));
        if (!wait_stage_inline(bar(B::STEAL), asked & 1, kTileWait)) {
          *stop = 1;
          break;
        }
        id = steal_answer(smem_addr(&s_answer));
        fence_proxy_async_smem();
      }
      {
        // Loads on their way land before the block ends (bounded again): whoever waits for them may have given up, or may
        // yet do so.
        if (q_uses > 0) wait_stage_inline(bar(B::Q), (q_uses - 1) & 1, kMaxWaitCycles);
        for (uint32_t x = 0; x < C::NS && x < issued; ++x) {
          const uint32_t n = issued - 1 - x;
          wait_stage_inline(bar(B::FULL + n % C::NS), (n / C::NS) & 1, kMaxWaitCycles);
        }
      }
    }
  } else if (warp <= C::SOFT + C::NQ) {
    // =================================================================================== MMAs of one query tile
    // The warp stays together and its control flow is uniform (values from shared memory are broadcast from lane 0 to
    // make that known), see mma_ss.
    auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const int i = uniform(warp) - C::SOFT - 1;
    const uint32_t leader = elect_one(), tm = uniform(tmem);
    const uint32_t id_s = instr_desc(DT == TQ_BF16, 128, C::BN, false) | (a.attn_scale < 0.0f ? kNegateA : 0u);
    const uint32_t id_o = instr_desc(DT == TQ_BF16, 128, C::DV, true);
    const uint32_t q_lo = desc_lo(base + i * C::QTILE, 0), ring_lo = desc_lo(base + C::RING, 0);
    const uint32_t o_at = tm + C::O_COL + i * C::DV;
    int stage = 0;
    uint32_t phase = 0, sn = 0, pn = 0, q_uses = 0;  // S and P tiles so far
    bool ok = true;
    Work w;
    for (int it = 0; ok && next_work(it, w); ++it) {
      const Span<C> r(a, w, T);
      const int J0 = uniform(r.J0), J1 = uniform(r.J1), lo = uniform(r.lo), up = uniform(r.up);
      const int my0 = uniform(i == 0 ? r.j0[0] : r.j0[C::NQ - 1]), my1 = uniform(i == 0 ? r.j1[0] : r.j1[C::NQ - 1]);
      if (J1 <= J0) continue;
      // one stage to wait for and to release per step; it is released behind the next step's scores, where the tensor
      // cores have work
      constexpr bool kLate = C::NS > 2;
      int owed = -1;
      ok = warp_wait_on(bar(B::Q), q_uses++ & 1, stop, tile_wait);
      for (int j = J0; j <= J1 && ok; ++j) {
        ok = warp_wait_on(bar(B::FULL + stage), phase, stop, tile_wait);
        if (!ok) break;
        const uint32_t at = ring_lo + stage * (C::STAGE >> 4);
        if (j >= my0 && j < my1) {
          // S into the buffer whose weights the output MMAs issued before have read
          const int buf = 2 * i + (sn & 1);
          const uint32_t d = tm + buf * C::BN;
#pragma unroll
          for (int y = 0; y < D / 16; ++y)
            mma_ss(leader, d, q_lo + (((y >> 2) * C::QCHUNK + (y & 3) * 32) >> 4), at + (((y >> 2) * C::KCHUNK + (y & 3) * 32) >> 4),
                   kDescHi, id_s, y > 0);
          mma_commit(leader, bar(B::S + buf));
          ++sn;
        }
        if (j + 1 == J1) mma_commit(leader, bar(B::Q_FREE));
        if (owed >= 0) mma_commit(leader, bar(B::EMPTY + owed));
        if (j - 1 >= my0 && j - 1 < my1) {
          // (READY only behind FULL: before it, READY may still be two phases back, which it cannot tell from this one)
          if ((j - 1) * C::BN < lo || j * C::BN > up) ok = warp_wait_on(bar(B::READY + stage), phase, stop, tile_wait);
          const int buf = 2 * i + (pn & 1);
          const uint32_t p = tm + buf * C::BN, v_at = at + (C::KT >> 4) + ((C::KCHUNK >> 4) << 16);
          ok = ok && warp_wait_on(bar(B::P + buf), (pn >> 1) & 1, stop, tile_wait);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int y = 0; y < C::BN / 16; ++y)
            mma_ts(leader, o_at, p + 8 * y, v_at + (2048 >> 4) * y, kDescHi, id_o, y > 0 || j - 1 > my0);
          if (j + 1 >= my1) mma_commit(leader, bar(B::O + i));
          ++pn;
        }
        if (kLate && j < J1) owed = stage;
        else mma_commit(leader, bar(B::EMPTY + stage));
        if (++stage == C::NS) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
    // everything issued has completed before the block gives its memory back
    mma_commit(leader, bar(B::DRAIN));
    if (!__all_sync(0xffffffffu, wait_stage_inline(bar(B::DRAIN), 0, kTileWait))) *stop = 1;
  } else {
    // ============================================================= V tiles that some row sees in part: finite values
    const int me = tid - 32 * (C::SOFT + 1 + C::NQ);
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    Work w;
    for (int it = 0; ok && next_work(it, w); ++it) {
      const Span<C> r(a, w, T);
      // every stage of the ring in turn, so that none is filled again behind this warp's back
      for (int j = r.J0; j <= r.J1 && r.J1 > r.J0 && ok; ++j) {
        ok = warp_wait_on(bar(B::FULL + stage), phase, stop, tile_wait);
        if (!ok) break;
        if (j > r.J0 && r.partly(j - 1)) {
          uint4* tile = reinterpret_cast<uint4*>(smem + C::RING + stage * C::STAGE + C::KT);
          bool found = false;
#pragma unroll 8
          for (int y = me; y < C::VT / 16; y += 32 * C::SCRUB) {
            const uint4 v = tile[y];
            if (not_finite2<DT>(v.x) | not_finite2<DT>(v.y) | not_finite2<DT>(v.z) | not_finite2<DT>(v.w)) {
              auto clean = [](uint32_t z) {
                const uint32_t bad = not_finite2<DT>(z);
                return z & ~((bad >> 15) * 0xffffu);
              };
              tile[y] = make_uint4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
              found = true;
            }
          }
          if (found) s_scrubbed[it & 3] = 1;
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(B::READY + stage));
          mbar_arrive(bar(B::EMPTY + stage));
        }
        if (++stage == C::NS) {
          stage = 0;
          phase ^= 1;
        }
      }
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

// [rows][heads][d] values, rows `stride` elements apart, boxes of 128 bytes x `heads_box` x `rows_box`
bool make_map(CUtensorMap* map, const void* p, int dtype, int d, int heads, long long rows, long long stride, int heads_box,
              int rows_box) {
  const int size = dtype == TQ_FP32 ? 4 : 2;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(d) * size, static_cast<cuuint64_t>(stride) * size};
  const cuuint32_t box[3] = {128u / size, static_cast<cuuint32_t>(heads_box), static_cast<cuuint32_t>(rows_box)};
  const cuuint32_t ones[3] = {1, 1, 1};
  const CUtensorMapDataType type = dtype == TQ_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == TQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                      : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encode_fn()(map, type, 3, const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Thread blocks of a launch: no less than there are pieces of work, whatever the lengths.
template <typename C>
long long blocks_of(const PromptArgs& a) {
  const int T = 128 / (a.H_q / a.H_kv);
  return (static_cast<long long>(a.n_q) / (C::NQ * T) + a.B) * a.H_kv * (C::D_ / C::DV);
}

template <int D, int NQ, int DT, int OT, bool TEST = false>
cudaError_t launch_tiles(const PromptArgs& a, cudaStream_t st, Hook hook = {}) {
  using C = Cfg<D, NQ>;
  if constexpr (D == 128 && DT == TQ_FP16 && OT == TQ_FP32 && !TEST) {
    const int limit = test_hooks().spin_limit.load(std::memory_order_relaxed), fault = test_hooks().fault_block.load(std::memory_order_relaxed);
    if (limit > 0 || fault >= 0) return launch_tiles<D, NQ, DT, OT, true>(a, st, {limit > 0 ? limit : static_cast<int>(kTileWait), fault});
  }
  auto* kernel = prompt_kernel<D, NQ, DT, OT, TEST>;
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit) || !bit) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM)) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  const int G = a.H_q / a.H_kv, T = 128 / G;
  const long long blocks = blocks_of<C>(a);
  if (!encode_fn() || blocks > 0x7fffffffLL) return cudaErrorNotSupported;
  Maps maps;
  // (without a single key the maps of K and V describe a row of q; nothing is loaded through them)
  const bool keys = a.n_kv > 0;
  if (!make_map(&maps.q, a.q, a.dtype, D, a.H_q, a.n_q, a.q_stride, G, T) ||
      !make_map(&maps.k, keys ? a.k : a.q, a.dtype, D, a.H_kv, keys ? a.n_kv : 1, keys ? a.k_stride : a.q_stride, 1, C::BN) ||
      !make_map(&maps.v, keys ? a.v : a.q, a.dtype, D, a.H_kv, keys ? a.n_kv : 1, keys ? a.v_stride : a.q_stride, 1, C::BN) ||
      !make_map(&maps.o, a.out, a.out_dtype, D, a.H_q, a.n_q, static_cast<long long>(a.H_q) * D, G > 32 ? 1 : G, G > 32 ? 1 : 32 / G))
    return cudaErrorInvalidValue;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(blocks)), dim3(C::THREADS), C::SMEM, st, maps, a, G, T, hook);
}

template <int D, int DT, int OT>
cudaError_t launch_dto(const PromptArgs& a, cudaStream_t st) {
  if constexpr (D <= 128) {  // (the rule is explained at the top)
    if (blocks_of<Cfg<D, 1>>(a) > device_sm_count()) return launch_tiles<D, 2, DT, OT>(a, st);
  }
  return launch_tiles<D, 1, DT, OT>(a, st);
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

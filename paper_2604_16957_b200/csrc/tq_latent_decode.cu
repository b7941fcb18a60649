// Attention of single tokens over the latent cache on the tensor cores (tcgen05, TMEM), absorbed form:
// tq_sdpa_latent_decode.
//
// All heads of a sequence attend the same tokens, so both products have the heads as their narrow side, and the tokens and
// channels as the wide one.  A thread block takes a group of up to N = 16, 32 or 64 heads over a run of tiles of 64 tokens:
//     S^T = [codes | r] [qc | qr]^T     64 tokens x N heads; codes and positional part apart: S_c, S_r
//     z = alpha log2 e (a / 127 S_c + s S_r),   P^T = 2^(z - ref + log2(a / 127)),   rounded to fp16
//     O^T += codes^T P^T                d_c channels x N heads, accumulated in TMEM: d_c / 128 times N columns
// The codes are made fp16 once (they are exact) for both products (BYTES: for O^T).  Neither the token's range nor the latent's
// rounding enters the products: the range goes into the score in fp32 and, as its logarithm, into the weight's exponent, so
// weights of tokens of any size share one fp16 scale.  The sum of weights takes it out again (P^T times 127 / a, before rounding, in fp32).
// Ranges may lie 2^128 apart (2^64 to 2^-64, zeros among the smallest): a token of small range has no part in O^T beside a large
// one, but all of its weight in the sum.  So the exponentials are made 2^48 times as large (they are normal numbers in fp32
// down to 2^-174 then, where the weight is less than 2^-53 of the head's largest), which P^T loses again before it is rounded and the sum in
// 127 / a; and where sums are rescaled or joined their factor, down to 2^-128, is taken in two halves.
//
// ref is per head, in two parts that add up to ref: a score (subtracted first, which is exact where it matters: equal scores of
// any size give equal weights) and an offset, less 48.  It is set so that the largest weight of the first tile is 2^8, and raised when one
// exceeds 2^15.5; then O^T and the sums are rescaled.  fp16 weights are rounded by 2^-11 of themselves, or by 2^-25: 2^-33
// of the largest.
//
// Queries are fp16 operands for either input type: bf16 ones are multiplied by a power of two that brings the head's largest
// channel into [2^15, 2^16).
// Up to 16 heads (BYTES) the scores take the codes as they are, unsigned bytes c + 128, and the queries as four signed digits to
// the base 128, 64 columns for 16 heads: whole numbers, exact but for the query's rounding by 2^-26 of the largest of a head's
// d_c.  The codes' offset is taken out again as 128 times the sum of the digits.
//
// Roles: four or eight warps of softmax and epilogue (a thread has a token and 8 or 16 heads: S^T of 64 rows fills 16 lanes of
// every quarter of TMEM), eight or four that turn codes into operands, one that issues the MMAs, one that finds the work, looks
// up pages, asks for the tiles' blocks to be brought to L2 and loads the queries (BYTES: loads the tiles); up to 32 heads two
// more that make tokens' factors of their scales.
//
// What bounds it is shared memory with L1: 128 bytes a cycle for the MMAs' operands, the converted codes, the loads and every
// look at a barrier, and while MMAs read at that rate the rest waits.  64 tokens of 32 heads take 790 cycles of the scores'
// operands, 640 of codes stored and about as many loaded; of 64 heads 1155 and, where O^T's operand comes from shared
// memory too, 770.  So
//   - up to 16 heads codes come by TMA and are not stored a second time: 600 cycles of the scores' operands, 320 to write a
//     tile and 256 to read it for O^T (128K tokens, 16 heads 36 -> 33 us).
//   - up to 32 heads the codes go to shared memory as K-major rows for the scores (BYTES: they are there), and from registers
//     to TMEM, where their transpose is the left operand of O^T: a lane there is a channel, and the thread of a lane has UNITS
//     neighbouring channels of every token, one for each row tile of O^T.  With 64 heads O^T takes half of TMEM and both products read
//     the codes in shared memory (transposed codes in the one buffer that was left: 258 us instead of 216 for the
//     ragged batch below).
//   - no softmax thread spills or looks anything up between the scores and the weights (216 -> 181 us); block numbers are
//     looked up two tiles ahead; up to 32 heads other warps divide and take logarithms (33 -> 31 us).  Registers go from the
//     last four warps to the softmax warps.
//   - 64 heads share one pass; four groups of 32 took 234 us instead of 164.
// A tile takes 1900 cycles with 16 heads and 4200 with 64.  Measured (B200, ten calls in a graph): 128K tokens, 16 heads 28.3 us
// (85 MB, floor 13), 32 heads 46; 32K tokens, 128 heads 37 us; 32 sequences of 2000 to 16384 tokens, 128 heads 170 us, 480 TFLOP/s;
// 60 of 100 to 1500, 20 heads, d_c = 256 22 us; 1K tokens, 16 heads 10.6 us (10.0 with fp16 products instead of bytes).
// (Figures of single steps, above and below, are those of the step's own before and after.)
//
// Work: the tiles of all sequences lie on a line, each sequence with kFixed places for its start in front; every thread block
// takes an equal share (down to one tile: calls on 1K tokens, 16 heads 11.6 us; with shares of four 15).  Sequences that are
// cut leave partial results (O^T, ref, sums) and a second kernel joins them.  With 16 and 32
// heads (d_c = 512) 3 places are within 8 % of the best of 2, 3, 4 and 6 for every batch tried, while 2 lose up to 20 % where short
// sequences stand beside a long one; 128 heads with many short ones would take 6 (one of 128K among 36 of one token 140, 115, 100
// and 92 us; 37 of 3500 tokens 92, 85, 90 and 89).
#include <cuda.h>

#include <algorithm>

#include "tq_async.cuh"
#include "tq_latent.cuh"
#include "tq_tcgen05.cuh"
#include "tq_tensor_map.cuh"

namespace tq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTok = 64;                       // tokens of a tile
constexpr int kBatch = 8;                      // tiles whose pages are looked up together: a lane per block
constexpr int kWarps = 16, kThreads = 32 * kWarps, kMmaWarp = 12, kFeedWarp = 13;  // 12 of softmax and conversion
constexpr int kPanel = kTok * 128;             // bytes of 64 tokens x 64 channels
constexpr int kFixed = 3;                      // what the start of a sequence costs, in tiles
// log2 of the largest exponential when ref is set; when it is raised.  Weights are 2^-48 of them (see the top).
constexpr float kTop = 8.0f + 48.0f, kMost = 15.5f + 48.0f, kDown = 1.0f / 281474976710656.0f;
constexpr int kFactorWarp = 14, kSlots = 4;    // two warps that make tokens' factors, tiles of them in shared memory (TURNED)
constexpr int kDigits = 4;                     // of a query, to the base 128: 26 bits and a sign
constexpr float kFar = 1048576.0f;             // scores from which ref is kept in two parts, see the top

// A part: [N][DC] sums, then [N] scores and offsets of ref, and [N] sums of weights.
__host__ __device__ constexpr int part_floats(int dc, int n) { return n * (dc + 4); }
__host__ __device__ constexpr size_t info_bytes(int B) { return (8 * static_cast<size_t>(B) + 255) & ~static_cast<size_t>(255); }

template <int DC, int N_>
struct Cfg {
  static constexpr int N = N_;                         // columns: heads of a thread block
  static constexpr int SOFT = N == 64 ? 8 : 4;         // softmax warps: four have every second half of N heads between them
  static constexpr bool TURNED = N < 64;               // O^T's operand: codes transposed into TMEM; or those in shared memory
  static constexpr int CONV = 12 - SOFT;               // warps that turn codes into operands
  static constexpr int HN = N / (SOFT / 2);            // heads of a softmax thread
  static constexpr int UNITS = DC / 128;               // row tiles of O^T (TURNED: and channels of a lane)
  static constexpr int PARTS = TURNED ? 1 : UNITS + 1; // that a tile's shared memory is given back in
  static constexpr bool BYTES = N == 16;               // scores from the codes as they are, queries in kDigits digits
  static constexpr int PANELS = (BYTES ? UNITS : DC / 64) + 1;  // rows of 128 bytes each; the last one is the positional part
  static constexpr int TILE = PANELS * kPanel;
  static constexpr int QPANEL = (BYTES ? kDigits : 1) * N * 128;
  static constexpr int Q = 0, Q_POS = Q + (PANELS - 1) * QPANEL, P = Q_POS + N * 128, RING = (P + kPanel + 1023) & ~1023;
  static constexpr int SN = (BYTES ? kDigits + 1 : 2) * N;  // columns of a buffer of scores; the last N are the positional part's
  static constexpr int SMALL_BYTES = TURNED ? 8192 : 3072;
  static constexpr int FIT = (232448 - SMALL_BYTES - RING) / TILE;
  static constexpr int MOST = BYTES ? 4 : 3, NB = FIT < MOST ? FIT : MOST;  // tiles in shared memory
  static constexpr int SMALL = RING + NB * TILE;
  static constexpr int SMEM = SMALL + SMALL_BYTES;
  // TMEM: O^T, two buffers of scores in two parts, two of transposed codes (two tokens a column)
  static constexpr int O_COL = 0, S_COL = UNITS * N, V_COL = S_COL + 2 * SN;
  static constexpr int NEED = V_COL + (TURNED ? 64 * UNITS : 0), COLS = NEED <= 128 ? 128 : (NEED <= 256 ? 256 : 512);
  static_assert(NB >= 2 && SMEM <= 232448 && NEED <= 512, "");
  // mbarriers
  static constexpr int FULL = 0, EMPTY = FULL + NB;                             // operands of the scores
  static constexpr int SCORES = EMPTY + NB * PARTS, READ = SCORES + 2;                  // S^T: made, read
  static constexpr int VALUES = READ + 2, VALUES_FREE = VALUES + 2;             // transposed codes
  static constexpr int WEIGHTS = VALUES_FREE + 2, DONE = WEIGHTS + 1, DRAINED = DONE + 1;  // P^T; O^T += of a tile; O^T has been read
  static constexpr int RAW = DRAINED + 1, QUERY = RAW + 1, QUERY_FREE = QUERY + 1, SCALED = QUERY_FREE + 1;  // queries as they are, as operands; their scales read
  static constexpr int FACTORS = SCALED + 1, FACTORS_FREE = FACTORS + kSlots;  // of a tile's tokens: made, read
  static constexpr int WORK = FACTORS_FREE + kSlots, WORK_FREE = WORK + 2, PAGES = WORK_FREE + 2, PAGES_FREE = PAGES + 2, END = PAGES_FREE + 2,
                       BARS = END + 1;
};

// A piece of work: tiles [0, n) of 64 tokens from token t0 on (a multiple of 16), of which [lo, len) are seen.
struct Work {
  int b, t0, n, lo, len, part, more;  // part: number of its partial result, or -1: the whole sequence; more = 0: there is none
};

template <int DC, int N>
struct Small {
  float ref_z[N], ref_o[N], scale[N], scale_r[Cfg<DC, N>::BYTES ? N : 1], tmp[N], red[4][N];
  int bias[kDigits][Cfg<DC, N>::BYTES ? N : 1];
  int pages[2][4 * kBatch];
  float4 factors[Cfg<DC, N>::TURNED ? kSlots : 1][Cfg<DC, N>::TURNED ? kTok : 1];
  Work work[2];
  uint64_t bars[Cfg<DC, N>::BARS];
  int sums[kWarps], start_b, start_p, far, stop;
  uint32_t over[Cfg<DC, N>::SOFT];  // heads of each softmax warp whose exponentials exceed 2^kMost
  uint32_t tmem;
};

// Instrumented instantiation only (the library's own tests, see TestHooks): limit of the waits for a tile in SM cycles, and the
// tile of each thread block whose operands are never announced.
struct Hook {
  int wait_cycles, fault_tile;
};

// pred over the softmax threads: true for all if true for one
template <int THREADS>
__device__ __forceinline__ bool any_of_group(bool p) {
  uint32_t r;
  asm volatile(
      "{\n.reg .pred p, q;\nsetp.ne.u32 p, %1, 0;\nbarrier.cta.red.or.pred q, 1, %2, p;\nselp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(p)), "n"(THREADS)
      : "memory");
  return r != 0;
}
template <int THREADS>
__device__ __forceinline__ void group_sync() {
  asm volatile("barrier.cta.sync 1, %0;\n" ::"n"(THREADS) : "memory");
}

struct Max {
  __device__ static float of(float a, float b) { return fmaxf(a, b); }
};
struct Sum {
  __device__ static float of(float a, float b) { return a + b; }
};
// Reduces v[i] (i: head `base` + i) over the 16 lanes of a half warp into row[head].  The lanes share the heads out as they go.
template <typename Op, int HN>
__device__ __forceinline__ void reduce_half(float (&v)[HN], int lane, int base, float* row) {
  int n = HN;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) {
    if (n > 1) {
      n /= 2;
      const bool up = lane & off;
#pragma unroll
      for (int i = 0; i < HN / 2; ++i) {
        if (i >= n) continue;
        const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
        v[i] = Op::of(keep, __shfl_xor_sync(0xffffffffu, give, off));
      }
      base += up ? n : 0;
    } else {
      v[0] = Op::of(v[0], __shfl_xor_sync(0xffffffffu, v[0], off));
    }
  }
#pragma unroll
  for (int i = 0; i < (HN >= 16 ? HN / 16 : 1); ++i) row[base + i] = v[i];
}

__device__ __forceinline__ int tiles_of(int len, int window) {
  return len > 0 ? (len - (window_begin(len, window) & ~15) + kTok - 1) / kTok : 0;
}

// Which code a lane of TMEM has: channels `channel` .. + UNITS - 1 of every token, from byte `byte` on of its codes.
template <int UNITS>
struct Lane {
  int unit, half, piece, low, first;  // 128 channels, 64 of them, 8 of them, 4 of them; the first of the lane's in those
  __device__ Lane(int quarter, int lane)
      : unit(quarter / (4 / UNITS)), half(lane >> 4), piece((lane & 15) >> 1), low(lane & 1), first((quarter % (4 / UNITS)) * UNITS) {}
  __device__ int channel() const { return 128 * unit + 64 * half + 8 * piece + 4 * low + first; }
  __device__ int word() const { return 128 * unit + 16 * piece + 8 * half + 4 * low; }  // (byte of the four codes that hold them)
};

// bytes (low, high) of two codes as stored -> exact fp16 numbers
__device__ __forceinline__ uint32_t codes16(uint32_t bytes, uint32_t selector) {
  const __half2 k = __half2half2(__ushort_as_half(0x6480));  // 1024 + 128
  const uint32_t w = __byte_perm(bytes, 0x64646464u, selector);
  const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&w), k);
  return *reinterpret_cast<const uint32_t*>(&x);
}

// (a code is read by one thread of an SM, so L1 need not keep it: 128K tokens of 16 heads 36.5 us instead of 38.5)
__device__ __forceinline__ uint32_t load_once(const uint8_t* p) {
  uint32_t v;
  asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];\n" : "=r"(v) : "l"(p) : "memory");
  return v;
}

// BYTES: the cache's codes and positional parts; otherwise the queries' two parts
struct LatentMaps {
  CUtensorMap c, r;
};

// What a token's scales are used as: {a / 127, s, log2(a / 127), 2^-48 127 / a}; {0, 0, -inf, 0} of one that is not seen.
// (One without a range has codes of 0 and counts as the smallest: 2^-64 / 127, about 2^-71.)
__device__ __forceinline__ float4 token_factors(float2 sc, bool seen) {
  const float unit = sc.x > 0.0f ? __fdiv_rn(sc.x, 127.0f) : 0.0f;
  const float lg = sc.x > 0.0f ? __log2f(unit) : -71.0f, inv = sc.x > 0.0f ? __fdiv_rn(127.0f * kDown, sc.x) : 2.3611832414348226e21f * kDown;
  return seen ? make_float4(unit, sc.y, lg, inv) : make_float4(0.0f, 0.0f, -INFINITY, 0.0f);
}
__device__ __forceinline__ float2 token_scales(const uint8_t* blocks, int blk, int d_c, int t) {
  return *reinterpret_cast<const float2*>(blocks + static_cast<long long>(blk) * latent_block_bytes(d_c) + latent_scale_offset(d_c, t & 15));
}

template <int DC, int N, bool TEST>
__global__ void __launch_bounds__(kThreads, 1) latent_kernel(const __grid_constant__ LatentMaps maps, const LatentArgs a, int groups,
                                                                        int per_group, const Hook hook) {
  using C = Cfg<DC, N>;
  extern __shared__ __align__(1024) uint8_t smem[];
  auto& sm = *reinterpret_cast<Small<DC, N>*>(smem + C::SMALL);
  static_assert(sizeof(Small<DC, N>) <= C::SMALL_BYTES, "");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t base = smem_addr(smem);
  auto bar = [&](int i) { return smem_addr(&sm.bars[i]); };
  volatile int* const stop = &sm.stop;
  const long long tile_wait = TEST ? hook.wait_cycles : kTileWait;
  const int group = blockIdx.x % groups, line = blockIdx.x / groups, lines = gridDim.x / groups;
  const int h0 = group * per_group, heads = min(per_group, a.H - h0);
  const bool bf16 = a.q_dtype == TQ_BF16;

  if (warp == kMmaWarp) tmem_alloc(smem_addr(&sm.tmem), C::COLS);
  if (tid == 0) {
    for (int i = 0; i < C::NB; ++i) {
      mbar_init(bar(C::FULL + i), C::BYTES ? 1 : C::CONV);
      for (int k = 0; k < C::PARTS; ++k) mbar_init(bar(C::EMPTY + i * C::PARTS + k), C::BYTES ? C::CONV + 1 : 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(C::SCORES + i), C::TURNED ? 2 : 1);
      mbar_init(bar(C::READ + i), C::SOFT);
      mbar_init(bar(C::VALUES + i), C::CONV);
      mbar_init(bar(C::VALUES_FREE + i), 1);
      mbar_init(bar(C::WORK + i), 1);
      mbar_init(bar(C::WORK_FREE + i), C::TURNED ? 15 : 13);
      mbar_init(bar(C::PAGES + i), 1);
      mbar_init(bar(C::PAGES_FREE + i), C::BYTES ? 2 : (C::TURNED ? C::CONV + 2 : 12));
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(bar(C::FACTORS + i), 2);
      mbar_init(bar(C::FACTORS_FREE + i), C::SOFT);
    }
    mbar_init(bar(C::WEIGHTS), C::SOFT);
    mbar_init(bar(C::DONE), 1);
    mbar_init(bar(C::DRAINED), C::SOFT);
    mbar_init(bar(C::RAW), 1);
    mbar_init(bar(C::QUERY), C::CONV);
    mbar_init(bar(C::QUERY_FREE), 1);
    mbar_init(bar(C::SCALED), C::SOFT);
    mbar_init(bar(C::END), 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    sm.stop = 0;
    sm.start_b = a.c.B;
    sm.start_p = 0;
  }
  pdl_launch_dependents();
  pdl_wait();

  // ---- this thread block's share of the line: [x0, x1), and the sequence it begins in
  // (thread i looks at sequences i, i + kThreads, ...; of so few that a round will do the lengths are kept for the warp that finds
  // the work, in the weights' place)
  const bool one_round = a.c.B <= kThreads;
  int* const lengths = reinterpret_cast<int*>(smem + C::P);
  auto cost_of = [&](int raw) { return tiles_of(min(max(raw, 0), a.c.S_cap), a.window) + kFixed; };
  int cost = 0, total = 0;
  if (tid < a.c.B) {
    const int raw = a.c.seq_lens[tid];
    if (one_round) lengths[tid] = raw;
    cost = cost_of(raw);
  }
  auto scan = [&](int v) {  // over the thread block's threads: up to and with this one; `total` of all
    auto up = [&](int x) {
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
      }
      return x;
    };
    v = up(v);
    __syncthreads();
    if (lane == 31) sm.sums[warp] = v;
    __syncthreads();
    const int w = up(lane < kWarps ? sm.sums[lane] : 0), before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
    total = __shfl_sync(0xffffffffu, w, 31);
    return warp > 0 ? v + before : v;
  };
  int sum = cost;
  if (!one_round)
    for (int b = tid + kThreads; b < a.c.B; b += kThreads) sum += cost_of(a.c.seq_lens[b]);
  tc_fence_before();
  int upto = scan(sum);
  tc_fence_after();
  const int length = total, share = max(1, (length + lines - 1) / lines);
  const int x0 = min(line * share, length), x1 = min(x0 + share, length);
  for (int b0 = 0, p0 = 0; b0 < a.c.B && p0 <= x0; b0 += kThreads) {
    if (!one_round) {
      const int b = b0 + tid;
      cost = b < a.c.B ? cost_of(a.c.seq_lens[b]) : 0;
      upto = scan(cost);
    }
    const int p = p0 + upto - cost;
    if (cost > 0 && p <= x0 && x0 < p + cost) {
      sm.start_b = b0 + tid;
      sm.start_p = p;
    }
    p0 += total;
  }
  __syncthreads();
  const uint32_t tmem = sm.tmem;

  // 512 threads have 128 registers each; the last four warps leave half of theirs to the softmax warps.  A quarter of an SM
  // has its own registers, so what is taken there has to be left there: in each one or two softmax warps, two or one of
  // conversion and one of the last four, 192 + 2 x 128 + 64 = 2 x 160 + 128 + 64 = 4 x 128.
  static_assert(kWarps == 16 && kMmaWarp == 12 && (C::SOFT == 4 || C::SOFT == 8), "register split");
  if (warp < C::SOFT) {
    if constexpr (C::SOFT == 4) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;\n");
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 160;\n");
  } else if (warp >= kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;\n");
  }

  // the it-th piece of work, for every warp but the one that finds it; false: none, or the block winds down
  auto next_work = [&](int it, Work& w, bool live) {
    if (live) live = warp_wait_on(bar(C::WORK + (it & 1)), (it >> 1) & 1, stop, kBlockWait);
    w = sm.work[it & 1];
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(C::WORK_FREE + (it & 1)));
    return live;
  };

  if (warp < C::SOFT) {
    // =========================================================================================== softmax, epilogue
    // The warps meet at named barriers, so none leaves the others: a warp whose wait ran out goes on without waiting
    // (what it computes means nothing then), and they leave together between pieces of work.
    const int wq = warp & 3, column0 = (warp >> 2) * 2 * C::HN;  // quarter of TMEM, first head of the warp
    const int row = 16 * wq + (lane & 15), hbase = column0 + (lane >> 4) * C::HN;
    const uint32_t quarter = static_cast<uint32_t>(32 * wq) << 16;
    uint8_t* const p_row = smem + C::P + row * 128;
    float* const parts = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + info_bytes(a.c.B));
    bool live = true;
    uint32_t tile = 0, batch = 0, pieces = 0;  // tiles, batches of pages, pieces of work with tiles so far
    auto wait = [&](uint32_t b, uint32_t parity) {
      if (live) live = warp_wait_on(b, parity, stop, tile_wait);
    };
    Work w;
    for (int it = 0;; ++it) {
      const bool got = next_work(it, w, live);
      if (any_of_group<32 * C::SOFT>(!got) || !w.more) break;
      float l[C::HN], ref[C::HN], scale[C::HN], scale_r[C::BYTES ? C::HN : 1];
      bool far = false;
      int bias[C::BYTES ? kDigits : 1][C::HN];
#pragma unroll
      for (int i = 0; i < C::HN; ++i) {
        l[i] = 0.0f;
        scale[i] = a.attn_scale * kLog2e;
      }
      // Factors of this thread's token.  TURNED: another warp's, announced with the scores.  Otherwise scales are asked for a tile
      // ahead, their block is looked up two tiles ahead: while MMAs read shared memory a look-up takes about as long as they do,
      // and nothing here may wait for one.
      float4 own;
      auto block = [&](int i) {
        if (i % kBatch == 0) wait(bar(C::PAGES + (batch & 1)), (batch >> 1) & 1);
        const int blk = sm.pages[batch & 1][4 * (i % kBatch) + wq];
        if (i % kBatch == kBatch - 1 || i == w.n - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::PAGES_FREE + (batch & 1)));
          ++batch;
        }
        return live ? blk : 0;
      };
      float2 next;
      int after = 0;
      if constexpr (!C::TURNED) {
        if (w.n > 0) next = token_scales(a.c.blocks, block(0), DC, row);
        if (w.n > 1) after = block(1);
      }
      for (int i = 0; i < w.n; ++i, ++tile) {
        if constexpr (!C::TURNED) {
          const int at = w.t0 + kTok * i + row;
          own = token_factors(next, at >= w.lo && at < w.len);
          if (i + 1 < w.n) next = token_scales(a.c.blocks, after, DC, row);
          if (i + 2 < w.n) after = block(i + 2);
        }
        const int buf = tile % 2;
        const uint32_t s_at = tmem + quarter + C::S_COL + buf * C::SN + column0;
        if (i == 0 && (bf16 || C::BYTES)) {
          wait(bar(C::QUERY), pieces & 1);
#pragma unroll
          for (int x = 0; x < C::HN; ++x) {
            scale[x] = sm.scale[hbase + x];
            if constexpr (C::BYTES) {
              scale_r[x] = sm.scale_r[hbase + x];
#pragma unroll
              for (int d = 0; d < kDigits; ++d) bias[d][x] = sm.bias[d][hbase + x];
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::SCALED));
        }
        wait(bar(C::SCORES + buf), (tile / 2) & 1);
        tc_fence_after();
        float z[C::HN], e[C::HN];
        tmem_ld_halves<C::HN>(s_at + C::SN - N, reinterpret_cast<uint32_t*>(e));
        if constexpr (C::TURNED) own = sm.factors[tile % kSlots][row];
        if constexpr (C::BYTES) {
          uint32_t d[kDigits][C::HN];
          tmem_ld_halves<kDigits * C::HN>(s_at, d[0]);
          tmem_wait_ld();
          // whole numbers of 22 bits, without what the codes' offset of 128 adds: exact in fp32 (1.5 2^23 + x), and put together
#pragma unroll
          for (int x = 0; x < C::HN; ++x) {
            auto digit = [&](int k) { return __uint_as_float(d[k][x] + static_cast<uint32_t>(bias[k][x])) - 12582912.0f; };
            z[x] = digit(kDigits - 1);
#pragma unroll
            for (int k = kDigits - 2; k >= 0; --k) z[x] = fmaf(z[x], 128.0f, digit(k));
          }
        } else {
          tmem_ld_halves<C::HN>(s_at, reinterpret_cast<uint32_t*>(z));
          tmem_wait_ld();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(C::READ + buf));
          if (C::TURNED) mbar_arrive(bar(C::FACTORS_FREE + tile % kSlots));
        }
        const float unit = own.x, pos = own.y, lg = own.z, inv = own.w;
        const bool seen = lg > -INFINITY;
        if (__any_sync(0xffffffffu, !seen)) {
          // (rows that no token was appended to may hold anything)
#pragma unroll
          for (int x = 0; x < C::HN; ++x) {
            z[x] = seen ? z[x] : 0.0f;
            e[x] = seen ? e[x] : 0.0f;
          }
        }
        const uint64_t unit2 = pair(unit, unit), pos2 = pair(pos, pos), lg2 = pair(lg, lg), inv2 = pair(inv, inv);
#pragma unroll
        for (int x = 0; x < C::HN; x += 2) {
          const uint64_t sum_r = mul2(pair(e[x], e[x + 1]), pos2), by = pair(scale[x], scale[x + 1]);
          float2 v;
          if constexpr (C::BYTES) v = unpair(fma2(mul2(pair(z[x], z[x + 1]), unit2), by, mul2(sum_r, pair(scale_r[x], scale_r[x + 1]))));
          else v = unpair(mul2(fma2(pair(z[x], z[x + 1]), unit2, sum_r), by));
          z[x] = v.x;
          z[x + 1] = v.y;
        }
        auto exponents = [&] {  // returns the largest
          float top = -INFINITY;
#pragma unroll
          for (int x = 0; x < C::HN; x += 2) {
            float2 v = unpair(add2(add2(pair(z[x], z[x + 1]), pair(-ref[x], -ref[x + 1])), lg2));
            if (far) v = make_float2(v.x - sm.ref_o[hbase + x], v.y - sm.ref_o[hbase + x + 1]);
            e[x] = v.x;
            e[x + 1] = v.y;
            top = fmaxf(top, fmaxf(v.x, v.y));
          }
          return top;
        };
        bool raise = i == 0;
        if (i > 0) raise = exponents() > kMost;
        if (any_of_group<32 * C::SOFT>(raise)) {
          // ref anew: the largest score, then the largest exponent beside it; but for the first tile only of heads that asked for
          // it themselves (no head's result depends on another's)
          if (i > 0) {
            uint32_t over = 0;
#pragma unroll
            for (int x = 0; x < C::HN; ++x) over |= static_cast<uint32_t>(e[x] > kMost) << x;
            over = __reduce_or_sync(0xffffffffu, over << (lane & 16 ? C::HN : 0));
            if (lane == 0) sm.over[warp] = over;
          }
          float v[C::HN];
#pragma unroll
          for (int x = 0; x < C::HN; ++x) v[x] = seen ? z[x] : -INFINITY;
          reduce_half<Max, C::HN>(v, lane, hbase, sm.red[wq]);
          group_sync<32 * C::SOFT>();
          float new_z = 0.0f;
          if (tid == 0) sm.far = 0;
          if (tid < N) sm.tmp[tid] = new_z = fmaxf(fmaxf(sm.red[0][tid], sm.red[1][tid]), fmaxf(sm.red[2][tid], sm.red[3][tid]));
          group_sync<32 * C::SOFT>();
#pragma unroll
          for (int x = 0; x < C::HN; ++x) v[x] = (z[x] - sm.tmp[hbase + x]) + lg;
          reduce_half<Max, C::HN>(v, lane, hbase, sm.red[wq]);
          group_sync<32 * C::SOFT>();
          if (tid < N) {
            const float new_o = fmaxf(fmaxf(sm.red[0][tid], sm.red[1][tid]), fmaxf(sm.red[2][tid], sm.red[3][tid])) - kTop;
            const float up = (new_z - sm.ref_z[tid]) + (new_o - sm.ref_o[tid]);
            const uint32_t* const asked = sm.over + 4 * (tid / (2 * C::HN));
            const bool take = i == 0 || ((asked[0] | asked[1] | asked[2] | asked[3]) >> (tid % (2 * C::HN)) & 1);
            sm.tmp[tid] = take ? ex2(-0.5f * up) : 1.0f;  // (half of it: sums may need a factor of 2^-128)
            if (take) {
              const bool apart = fabsf(new_z) > kFar;
              sm.ref_z[tid] = apart ? new_z : new_z + new_o;
              sm.ref_o[tid] = apart ? new_o : 0.0f;
            }
            if (sm.ref_o[tid] != 0.0f) sm.far = 1;
          }
          group_sync<32 * C::SOFT>();
          far = sm.far != 0;
#pragma unroll
          for (int x = 0; x < C::HN; ++x) ref[x] = sm.ref_z[hbase + x];
          if (i > 0) {
#pragma unroll
            for (int x = 0; x < C::HN; ++x) l[x] = l[x] * sm.tmp[hbase + x] * sm.tmp[hbase + x];
            wait(bar(C::DONE), (tile - 1) & 1);
            tc_fence_after();
#pragma unroll 1
            for (int x = 16 * (warp >> 2); x < C::UNITS * N; x += 4 * C::SOFT) {
              uint32_t o[16];
              tmem_ld16(tmem + quarter + C::O_COL + x, o);
              tmem_wait_ld();
#pragma unroll
              for (int y = 0; y < 16; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * sm.tmp[(x + y) % N] * sm.tmp[(x + y) % N]);
              tmem_st16(tmem + quarter + C::O_COL + x, o);
            }
            tmem_wait_st();
          }
          exponents();
        }
        const bool free = live && tile > 0 ? mbar_test_wait(bar(C::DONE), (tile - 1) & 1) : true;  // (looked at in time, too)
        uint32_t p[C::HN / 2];
#pragma unroll
        for (int x = 0; x < C::HN; x += 2) {
          const float e0 = ex2(e[x]), e1 = ex2(e[x + 1]);
          const float2 s = unpair(fma2(pair(e0, e1), inv2, pair(l[x], l[x + 1])));
          l[x] = s.x;
          l[x + 1] = s.y;
          const float2 weight = unpair(mul2(pair(e0, e1), pair(kDown, kDown)));
          p[x >> 1] = pack2<TQ_FP16>(weight.x, weight.y);
        }
        if (!__all_sync(0xffffffffu, free)) wait(bar(C::DONE), (tile - 1) & 1);
#pragma unroll
        for (int x = 0; x < C::HN / 8; ++x)
          *reinterpret_cast<uint4*>(p_row + (((hbase / 8 + x) ^ (row & 7)) << 4)) = make_uint4(p[4 * x], p[4 * x + 1], p[4 * x + 2], p[4 * x + 3]);
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::WEIGHTS));
      }
      // ---- epilogue: a thread has UNITS neighbouring channels, for all heads
      reduce_half<Sum, C::HN>(l, lane, hbase, sm.red[wq]);
      group_sync<32 * C::SOFT>();
      if (tid < N) {
        const float sum = (sm.red[0][tid] + sm.red[1][tid]) + (sm.red[2][tid] + sm.red[3][tid]);
        sm.tmp[tid] = w.part < 0 ? (w.n > 0 ? __fdiv_rn(1.0f, sum) : 0.0f) : 1.0f;
        if (w.part >= 0) {
          float* const more = parts + static_cast<long long>(w.part) * part_floats(DC, N) + N * DC;
          more[tid] = sm.ref_z[tid];
          more[N + tid] = sm.ref_o[tid];
          more[2 * N + tid] = sum;
        }
      }
      group_sync<32 * C::SOFT>();
      if (w.n > 0) wait(bar(C::DONE), (tile - 1) & 1);
      tc_fence_after();
      // TURNED: UNITS neighbouring channels (one of each row tile); otherwise one of every 128
      constexpr int VEC = C::TURNED ? C::UNITS : 1;
      const int channel = C::TURNED ? Lane<C::UNITS>(wq, lane).channel() : 32 * wq + lane;
#pragma unroll 1
      for (int h = 8 * (warp >> 2); h < N; h += 2 * C::SOFT) {
        uint32_t o[C::UNITS][8];
        if (w.n > 0) {
#pragma unroll
          for (int m = 0; m < C::UNITS; ++m) tmem_ld8(tmem + quarter + C::O_COL + m * N + h, o[m]);
          tmem_wait_ld();
        }
        float* const part = w.part >= 0 ? parts + static_cast<long long>(w.part) * part_floats(DC, N) + channel : nullptr;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
#pragma unroll
          for (int m = 0; m < C::UNITS; m += VEC) {
            float v[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[k] = w.n > 0 ? __uint_as_float(o[m + k][y]) * sm.tmp[h + y] : 0.0f;
            auto store32 = [&](float* dst) {
              if constexpr (VEC == 4) *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
              else if constexpr (VEC == 2) *reinterpret_cast<float2*>(dst) = make_float2(v[0], v[1]);
              else *dst = v[0];
            };
            if (part) {
              store32(part + (h + y) * DC + 128 * m);
            } else if (h + y < heads) {
              const long long to = (static_cast<long long>(w.b) * a.H + h0 + h + y) * DC + channel + 128 * m;
              if (a.out_dtype == TQ_FP32) {
                store32(static_cast<float*>(a.out) + to);
              } else {
                uint16_t* const dst = static_cast<uint16_t*>(a.out) + to;
                const uint32_t lo = bf16 ? pack2<TQ_BF16>(v[0], v[VEC > 1 ? 1 : 0]) : pack2<TQ_FP16>(v[0], v[VEC > 1 ? 1 : 0]);
                if constexpr (VEC == 4)
                  *reinterpret_cast<uint2*>(dst) = make_uint2(lo, bf16 ? pack2<TQ_BF16>(v[2], v[3]) : pack2<TQ_FP16>(v[2], v[3]));
                else if constexpr (VEC == 2) *reinterpret_cast<uint32_t*>(dst) = lo;
                else *dst = static_cast<uint16_t>(lo);
              }
            }
          }
        }
      }
      if (w.n > 0) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::DRAINED));
        ++pieces;
      }
    }
  } else if (warp < kMmaWarp) {
    // ================================================================================= queries, codes into operands
    // A warp has the codes of TOK tokens, a thread four neighbouring channels of every 128 (TURNED: of one 128, of those its
    // lane's; two sets of four warps), and 16 bytes of the positional part of every fourth token of the warp's.
    constexpr int TOK = C::TURNED ? 32 : 16, ROPES = 16 / C::CONV;
    constexpr int UNITS = C::TURNED ? C::UNITS : 4;      // as far as a lane is concerned
    constexpr int TURNS = C::TURNED ? 1 : C::UNITS;      // 128 channels each
    const int cw = warp - C::SOFT, set = C::TURNED ? cw >> 2 : cw;
    const Lane<UNITS> own(C::TURNED ? cw & 3 : 0, lane);
    const uint32_t quarter = static_cast<uint32_t>(32 * (cw & 3)) << 16;
    const int rope0 = 64 / C::CONV * cw + (lane >> 3), piece = lane & 7;  // positional part: 16 bytes of tokens rope0, rope0 + 4, ...
    // bytes of a word that are the lane's (d_c < 512): of one word; of two words, neighbours side by side
    const uint32_t mine = UNITS == 2 ? (own.first ? 0x4342u : 0x4140u) : 0x4440u + own.first;
    const uint32_t both = UNITS == 2 ? (own.first ? 0x7362u : 0x5140u) : 0x0040u + 0x11u * own.first;
    bool ok = true;
    uint32_t tile = 0, batch = 0, pieces = 0;
    Work w;
    uint4 rope[ROPES], ahead[ROPES];  // of the tile that is next, of the last one asked for
    auto rope_next = [&] {
#pragma unroll
      for (int x = 0; x < ROPES; ++x) rope[x] = ahead[x];
    };
    // asks for the values of tile i of the piece
    auto load = [&](int i, uint32_t (&code)[TURNS * TOK]) {
      if (i % kBatch == 0 && !warp_wait_on(bar(C::PAGES + (batch & 1)), (batch >> 1) & 1, stop, tile_wait)) return false;
      const int* const pages = sm.pages[batch & 1] + 4 * (i % kBatch);
      {
        const uint8_t* const blk = a.c.blocks + static_cast<long long>(pages[rope0 >> 4]) * latent_block_bytes(DC) + latent_rope_offset(DC, rope0 & 15);
#pragma unroll
        for (int x = 0; x < ROPES; ++x) ahead[x] = *reinterpret_cast<const uint4*>(blk + 4 * 2 * kRope * x + 16 * piece);
      }
#pragma unroll
      for (int x = 0; x < TOK; x += 16) {
        const uint8_t* const blk = a.c.blocks + static_cast<long long>(pages[(set * TOK + x) >> 4]) * latent_block_bytes(DC) + own.word();
#pragma unroll
        for (int u = 0; u < TURNS; ++u)
#pragma unroll
          for (int y = 0; y < 16; ++y) code[u * TOK + x + y] = load_once(blk + 128 * u + DC * y);
      }
      if (i % kBatch == kBatch - 1 || i == w.n - 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::PAGES_FREE + (batch & 1)));
        ++batch;
      }
      return true;
    };
    // codes and positional part of a tile into shared memory
    auto keys = [&](uint32_t x, const uint32_t (&code)[TURNS * TOK]) {
      const int buf = x % C::NB;
      const uint32_t parity = ((x / C::NB) & 1) ^ 1;
      if (!warp_wait_on(bar(C::EMPTY + buf * C::PARTS + C::PARTS - 1), parity, stop, tile_wait)) return false;
      const uint32_t dst = base + C::RING + buf * C::TILE;
#pragma unroll
      for (int y = 0; y < ROPES; ++y) {
        const int r = rope0 + 4 * y;
        *reinterpret_cast<uint4*>(smem + C::RING + buf * C::TILE + (C::PANELS - 1) * kPanel + r * 128 + ((piece ^ (r & 7)) << 4)) = rope[y];
      }
#pragma unroll
      for (int u = 0; u < TURNS; ++u) {
        if (!C::TURNED && !warp_wait_on(bar(C::EMPTY + buf * C::PARTS + u), parity, stop, tile_wait)) return false;
        const uint32_t to = dst + (2 * (own.unit + u) + own.half) * kPanel + set * (TOK * 128) + 16 * own.piece + 8 * own.low + 2 * own.first;
#pragma unroll
        for (int y = 0; y < TOK; ++y) {
          const uint32_t at = (to ^ ((y & 7) << 4)) + y * 128, c = code[u * TOK + y];
          if constexpr (UNITS == 4)
            asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" ::"r"(at), "r"(codes16(c, 0x4140)), "r"(codes16(c, 0x4342)) : "memory");
          else if constexpr (UNITS == 2)
            asm volatile("st.shared.b32 [%0], %1;\n" ::"r"(at), "r"(codes16(c, mine)) : "memory");
          else
            asm volatile("st.shared.b16 [%0], %1;\n" ::"r"(at), "h"(static_cast<uint16_t>(codes16(c, mine))) : "memory");
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0 && !(TEST && static_cast<int>(x) == hook.fault_tile)) mbar_arrive(bar(C::FULL + buf));
      return true;
    };
    // the codes' transpose into TMEM
    auto values = [&](uint32_t x, const uint32_t (&code)[TURNS * TOK]) {
      const int buf = x % 2;
      if (!warp_wait_on(bar(C::VALUES_FREE + buf), ((x / 2) & 1) ^ 1, stop, tile_wait)) return false;
      tc_fence_after();
      const uint32_t to = tmem + quarter + C::V_COL + buf * 32 * UNITS + set * (TOK / 2);
#pragma unroll
      for (int y = 0; y < TOK; y += 16) {
        uint32_t v[UNITS][8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t c0 = code[y + 2 * k], c1 = code[y + 2 * k + 1];
          if constexpr (UNITS == 4) {
            const uint32_t lo = __byte_perm(c0, c1, 0x5140), hi = __byte_perm(c0, c1, 0x7362);
            v[0][k] = codes16(lo, 0x4140);
            v[1][k] = codes16(lo, 0x4342);
            v[2][k] = codes16(hi, 0x4140);
            v[3][k] = codes16(hi, 0x4342);
          } else {
            const uint32_t lo = __byte_perm(c0, c1, both);
            v[0][k] = codes16(lo, 0x4140);
            if constexpr (UNITS == 2) v[1][k] = codes16(lo, 0x4342);
          }
        }
#pragma unroll
        for (int m = 0; m < UNITS; ++m) tmem_st8(to + 32 * m + y / 2, v[m]);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::VALUES + buf));
      return true;
    };
    // BYTES: the queries of sequence b as digits, t = round(2^(25 - E) q) = sum_k 128^k t_k with the largest magnitude in
    // [2^E, 2^(E + 1)) (|t| < 2^26, -64 <= t_k < 64), in the order of the codes' bytes; their sums, times the codes' offset; and the
    // positional part as fp16 numbers, times a power of two of its own.  Digits of HN heads stand together, as a thread reads them.
    auto digits = [&](int b, auto type) {
      constexpr int T = decltype(type)::value;
      constexpr int CHUNKS = (DC + kRope) / 8, PER = (CHUNKS + 31) / 32, HEADS = N / C::CONV;
      uint4 v[PER], following[PER];
      auto load = [&](int h) {
        const uint16_t* qc = static_cast<const uint16_t*>(a.q_c.data) + b * a.q_c.row_stride + (h0 + h) * a.q_c.head_stride;
        const uint16_t* qr = static_cast<const uint16_t*>(a.q_r.data) + b * a.q_r.row_stride + (h0 + h) * a.q_r.head_stride;
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const int c = lane + 32 * x;
          following[x] = make_uint4(0, 0, 0, 0);
          if (h < heads && c < CHUNKS) following[x] = *reinterpret_cast<const uint4*>(c < DC / 8 ? qc + 8 * c : qr + 8 * c - DC);
        }
      };
      load(cw);
      if (!warp_wait_on(bar(C::QUERY_FREE), (pieces & 1) ^ 1, stop, kBlockWait)) return false;
      if (!warp_wait_on(bar(C::SCALED), (pieces & 1) ^ 1, stop, kBlockWait)) return false;
#pragma unroll 1  // (code that is met for the first time takes longer than what it does)
      for (int k = 0; k < HEADS; ++k) {
        const int h = cw + k * C::CONV;
#pragma unroll
        for (int x = 0; x < PER; ++x) v[x] = following[x];
        if (k + 1 < HEADS) load(h + C::CONV);
        uint32_t top = 0, top_r = 0;
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const uint32_t most = __vmaxu2(__vmaxu2(v[x].x & 0x7fff7fffu, v[x].y & 0x7fff7fffu),
                                         __vmaxu2(v[x].z & 0x7fff7fffu, v[x].w & 0x7fff7fffu));
          if (lane + 32 * x < DC / 8) top = __vmaxu2(top, most);
          else top_r = __vmaxu2(top_r, most);
        }
        top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
        top_r = __reduce_max_sync(0xffffffffu, max(top_r & 0xffffu, top_r >> 16));
        const bool bad = max(top, top_r) >= (T == TQ_BF16 ? 0x7f80u : 0x7c00u);  // an infinity or a NaN: the head gives NaN
        auto exponent = [&](uint32_t most) {  // (of 2^-100 at least)
          const float f = unpack2<T>(most).x;
          return f > 0.0f && !bad ? max(static_cast<int>(__float_as_uint(f) >> 23) - 127, -100) : 0;
        };
        auto power = [](int x) { return __uint_as_float(static_cast<uint32_t>(127 + x) << 23); };
        const int ex = exponent(top), ex_r = exponent(top_r);
        if (lane == 0) {
          const float factor = bad ? __uint_as_float(0x7fc00000u) : a.attn_scale * kLog2e;
          sm.scale[h] = h >= heads ? 0.0f : factor * power(ex - 15);  // (2^10 of it are in the tokens' factors)
          sm.scale_r[h] = h >= heads ? 0.0f : factor * power(ex_r - 15);
        }
        const float up = power(25 - ex), up_r = power(15 - ex_r);
        int sums[kDigits] = {};
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const int c = lane + 32 * x;
          if (c >= CHUNKS) continue;
          const uint32_t y[4] = {v[x].x, v[x].y, v[x].z, v[x].w};
          const bool pos = c >= DC / 8;
          const float by = pos ? up_r : up;
          float f[8];
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float2 g = unpack2<T>(y[m]);
            f[2 * m] = g.x * by;
            f[2 * m + 1] = g.y * by;
          }
          if (pos) {
            *reinterpret_cast<uint4*>(smem + C::Q_POS + h * 128 + (((c - DC / 8) ^ (h & 7)) << 4)) =
                make_uint4(pack2<TQ_FP16>(f[0], f[1]), pack2<TQ_FP16>(f[2], f[3]), pack2<TQ_FP16>(f[4], f[5]), pack2<TQ_FP16>(f[6], f[7]));
            continue;
          }
          // t + 64 (1 + 128 + 128^2 + 128^3) has the digits + 64 as its own: 7 bits each, spread to bytes, 64 taken off again
          uint32_t w[8], word[kDigits][2];
#pragma unroll
          for (int m = 0; m < 8; ++m) {
            const uint32_t u = static_cast<uint32_t>(__float2int_rn(f[m])) + 0x08102040u;
            const uint32_t two = (u & 0x3fffu) | ((u << 2) & 0x3fff0000u), four = (two & 0x007f007fu) | ((two << 1) & 0x7f007f00u);
            w[m] = (four + 0x40404040u) ^ 0x80808080u;
          }
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const uint32_t lo0 = __byte_perm(w[4 * m], w[4 * m + 1], 0x5140), lo1 = __byte_perm(w[4 * m + 2], w[4 * m + 3], 0x5140);
            const uint32_t hi0 = __byte_perm(w[4 * m], w[4 * m + 1], 0x7362), hi1 = __byte_perm(w[4 * m + 2], w[4 * m + 3], 0x7362);
            word[0][m] = __byte_perm(lo0, lo1, 0x5410);
            word[1][m] = __byte_perm(lo0, lo1, 0x7632);
            word[2][m] = __byte_perm(hi0, hi1, 0x5410);
            word[3][m] = __byte_perm(hi0, hi1, 0x7632);
          }
          // channels 8 c ..: 128 channels c / 16, piece c % 8, half c % 16 / 8
#pragma unroll
          for (int d = 0; d < kDigits; ++d) {
            const int row = (h / C::HN * kDigits + d) * C::HN + h % C::HN;
            sums[d] = __dp4a(static_cast<int>(word[d][1]), 0x01010101, __dp4a(static_cast<int>(word[d][0]), 0x01010101, sums[d]));
            *reinterpret_cast<uint2*>(smem + C::Q + (c >> 4) * C::QPANEL + row * 128 + (((c & 7) ^ (row & 7)) << 4) + (c & 8)) = make_uint2(word[d][0], word[d][1]);
          }
        }
#pragma unroll
        for (int d = 0; d < kDigits; ++d) {
          const int sum = __reduce_add_sync(0xffffffffu, sums[d]);
          if (lane == 0) sm.bias[d][h] = 0x4b400000 - 128 * sum;  // (with the bits of 1.5 2^23)
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::QUERY));
      return true;
    };
    for (int it = 0; ok && next_work(it, w, true) && w.more; ++it) {
      if (w.n == 0) continue;
      if constexpr (C::BYTES) {
        ok = bf16 ? digits(w.b, std::integral_constant<int, TQ_BF16>{}) : digits(w.b, std::integral_constant<int, TQ_FP16>{});
        for (int i = 0; i < w.n && ok; ++i, ++tile) {
          const int buf = tile % C::NB;
          ok = warp_wait_on(bar(C::FULL + buf), (tile / C::NB) & 1, stop, tile_wait);
          if (!ok) break;
          uint32_t code[TOK];
          const uint32_t from = base + C::RING + buf * C::TILE + own.unit * kPanel + set * (TOK * 128) + 16 * own.piece + 8 * own.half + 4 * own.low;
#pragma unroll
          for (int y = 0; y < TOK; ++y) asm volatile("ld.shared.b32 %0, [%1];\n" : "=r"(code[y]) : "r"((from ^ ((y & 7) << 4)) + y * 128) : "memory");
          ok = values(tile, code);
          if (lane == 0) mbar_arrive(bar(C::EMPTY + buf));
        }
        ++pieces;
        continue;
      }
      // TURNED: two tiles in registers in turn, so that loads have a tile's time to arrive.  (Of the others, whose 64 tokens take
      // twice the registers, the next tile's are asked for when this one's are in shared memory.)
      uint32_t even[TURNS * TOK], odd[C::TURNED ? TOK : 1];
      if (bf16) {
        // queries of bf16 as fp16, each head times the power of two that brings its largest into [2^15, 2^16)
        ok = warp_wait_on(bar(C::RAW), pieces & 1, stop, kBlockWait) && warp_wait_on(bar(C::SCALED), (pieces & 1) ^ 1, stop, kBlockWait);
        if (!ok) break;
        constexpr int CHUNKS = (DC + kRope) / 8, PER = (CHUNKS + 31) / 32, AT_ONCE = N / C::CONV < 4 ? N / C::CONV : 4;
#pragma unroll 1
        for (int first = cw; first < N; first += AT_ONCE * C::CONV) {
          uint4 v[AT_ONCE][PER];
          uint32_t top[AT_ONCE];
          auto at = [&](int k, int c) {
            const int h = first + k * C::CONV;
            return reinterpret_cast<uint4*>(smem + C::Q + (c >> 3) * C::QPANEL + h * 128 + (((c & 7) ^ (h & 7)) << 4));
          };
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k) {
            top[k] = 0;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
              const int c = lane + 32 * x;
              v[k][x] = c < CHUNKS ? *at(k, c) : make_uint4(0, 0, 0, 0);
            }
          }
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k) {
#pragma unroll
            for (int x = 0; x < PER; ++x)
              top[k] = __vmaxu2(__vmaxu2(top[k], __vmaxu2(v[k][x].x & 0x7fff7fffu, v[k][x].y & 0x7fff7fffu)),
                                __vmaxu2(v[k][x].z & 0x7fff7fffu, v[k][x].w & 0x7fff7fffu));
            top[k] = __reduce_max_sync(0xffffffffu, max(top[k] & 0xffffu, top[k] >> 16));
          }
#pragma unroll
          for (int k = 0; k < AT_ONCE; ++k) {
            const bool bad = top[k] >= 0x7f80u;  // an infinity or a NaN: the head gives NaN
            const float most = unpack2<TQ_BF16>(top[k]).x;
            const int ex = most > 0.0f ? max(static_cast<int>(__float_as_uint(most) >> 23) - 127 - 15, -126) : 0;
            const float up = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
            if (lane == 0) sm.scale[first + k * C::CONV] = bad ? __uint_as_float(0x7fc00000u) : a.attn_scale * kLog2e * __uint_as_float(static_cast<uint32_t>(127 + ex) << 23);
#pragma unroll
            for (int x = 0; x < PER; ++x) {
              const int c = lane + 32 * x;
              if (c >= CHUNKS) continue;
              const uint32_t y[4] = {v[k][x].x, v[k][x].y, v[k][x].z, v[k][x].w};
              uint32_t o[4];
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                const float2 f = unpack2<TQ_BF16>(y[m]);
                o[m] = bad ? 0 : pack2<TQ_FP16>(__fmul_rn(f.x, up), __fmul_rn(f.y, up));
              }
              *at(k, c) = make_uint4(o[0], o[1], o[2], o[3]);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::QUERY));
      }
      ++pieces;
      ok = load(0, even);
      if (!ok) break;
      if constexpr (C::TURNED) {
        rope_next();
        if (w.n > 1) ok = load(1, odd);
        for (int i = 0; i < w.n && ok; i += 2) {
          ok = keys(tile + i, even) && values(tile + i, even);
          if (ok) rope_next();
          if (ok && i + 2 < w.n) ok = load(i + 2, even);
          if (!ok || i + 1 >= w.n) break;
          ok = keys(tile + i + 1, odd) && values(tile + i + 1, odd);
          if (ok) rope_next();
          if (ok && i + 3 < w.n) ok = load(i + 3, odd);
        }
      } else {
        for (int i = 0; i < w.n && ok; ++i) {
          rope_next();
          ok = keys(tile + i, even);
          if (ok && i + 1 < w.n) ok = load(i + 1, even);
        }
      }
      tile += w.n;
    }
    tmem_wait_st();
  } else if (warp == kMmaWarp) {
    // ========================================================================================================== MMAs
    // The warp stays together and its control flow is uniform, see mma_ss.
    auto uniform = [](uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); };
    const uint32_t leader = elect_one(), tm = uniform(tmem);
    const uint32_t id_s = instr_desc(false, kTok, N, false), id_o = instr_desc(false, 128, N, true);
    const uint32_t q_lo = desc_lo(base + C::Q, 0), p_lo = desc_lo(base + C::P, 0), k_lo = desc_lo(base + C::RING, 0);
    bool ok = true;
    uint32_t tile = 0, pieces = 0;
    // for the scores of tile x (TURNED: its tokens' factors, too), and for the outputs of tile y, the first of its piece or not
    auto can_score = [&](uint32_t x) {
      if (C::TURNED && !warp_wait_on(bar(C::FACTORS + x % kSlots), (x / kSlots) & 1, stop, tile_wait)) return false;
      return warp_wait_on(bar(C::FULL + x % C::NB), (x / C::NB) & 1, stop, tile_wait) && warp_wait_on(bar(C::READ + x % 2), ((x / 2) & 1) ^ 1, stop, tile_wait);
    };
    auto can_output = [&](uint32_t y, bool first) {
      if (C::TURNED && !warp_wait_on(bar(C::VALUES + y % 2), (y / 2) & 1, stop, tile_wait)) return false;
      if (first && !warp_wait_on(bar(C::DRAINED), (pieces & 1) ^ 1, stop, tile_wait)) return false;
      return warp_wait_on(bar(C::WEIGHTS), y & 1, stop, tile_wait);
    };
    auto scores = [&](uint32_t x, bool last) {
      tc_fence_after();
      const uint32_t buf = x % C::NB, sbuf = x % 2;
      const uint32_t d = uniform(tm + C::S_COL + sbuf * C::SN), k = uniform(k_lo + ((buf * C::TILE) >> 4));
      constexpr int STEPS = (C::PANELS - 1) * 4;  // of 32 bytes
#pragma unroll
      for (int y = 0; y < STEPS; ++y) {
        const uint32_t ka = k + (((y >> 2) * kPanel + (y & 3) * 32) >> 4), qa = q_lo + (((y >> 2) * C::QPANEL + (y & 3) * 32) >> 4);
        if constexpr (C::BYTES) mma_ss_bytes(leader, d, ka, qa, kDescHi, instr_desc_bytes(kTok, kDigits * N), y > 0);
        else mma_ss(leader, d, ka, qa, kDescHi, id_s, y > 0);
      }
#pragma unroll
      for (int y = 0; y < kRope / 16; ++y)
        mma_ss(leader, d + C::SN - N, k + (((C::PANELS - 1) * kPanel + y * 32) >> 4), q_lo + ((C::Q_POS - C::Q + y * 32) >> 4), kDescHi, id_s, y > 0);
      mma_commit(leader, bar(C::SCORES + sbuf));
      if (C::TURNED && leader) mbar_arrive(bar(C::SCORES + sbuf));  // (the tokens' factors)
      mma_commit(leader, bar(C::EMPTY + buf * C::PARTS + C::PARTS - 1));
      if (last) mma_commit(leader, bar(C::QUERY_FREE));
    };
    auto outputs = [&](uint32_t x, bool first) {
      tc_fence_after();
      const uint32_t vbuf = x % 2, buf = x % C::NB;
      const uint32_t add = uniform(!first);
      if constexpr (C::TURNED) {
        const uint32_t v = uniform(tm + C::V_COL + vbuf * 32 * C::UNITS);
#pragma unroll
        for (int m = 0; m < C::UNITS; ++m)
#pragma unroll
          for (int y = 0; y < kTok / 16; ++y)
            mma_ts(leader, tm + C::O_COL + m * N, v + 32 * m + 8 * y, p_lo + (y * 2048 >> 4), kDescHi, id_o, y > 0 || add);
        mma_commit(leader, bar(C::VALUES_FREE + vbuf));
      } else {
        const uint32_t v = uniform(k_lo + ((buf * C::TILE) >> 4) + ((kPanel >> 4) << 16));
#pragma unroll
        for (int m = 0; m < C::UNITS; ++m) {
#pragma unroll
          for (int y = 0; y < kTok / 16; ++y)
            mma_ss(leader, tm + C::O_COL + m * N, v + ((2 * m * kPanel + y * 2048) >> 4), p_lo + (y * 2048 >> 4), kDescHi, id_o | kMnMajorA, y > 0 || add);
          mma_commit(leader, bar(C::EMPTY + buf * C::PARTS + m));
        }
      }
      mma_commit(leader, bar(C::DONE));
    };
    Work w;
    for (int it = 0; ok && next_work(it, w, true); ++it) {
      const int n = uniform(w.n);
      if (!uniform(w.more)) break;
      if (n == 0) continue;
      ok = warp_wait_on(bar(bf16 || C::BYTES ? C::QUERY : C::RAW), pieces & 1, stop, kBlockWait);
      if constexpr (C::TURNED) {
        // Scores are two tiles ahead, issued behind the outputs: while they read shared memory nobody else does much, so all
        // barriers are looked at before.
        for (int i = 0; i < 2 && i < n && ok; ++i) {
          ok = can_score(tile + i);
          if (ok) scores(tile + i, i + 1 == n);
        }
        for (int i = 0; i < n && ok; ++i) {
          const bool more = i + 2 < n;
          ok = (!more || can_score(tile + i + 2)) && can_output(tile + i, i == 0);
          if (!ok) break;
          outputs(tile + i, i == 0);
          if (more) scores(tile + i + 2, i + 3 == n);
        }
      } else {
        // The scores of the next tile go before the outputs of this one, whose weights are made meanwhile.
        for (int i = 0; i <= n && ok; ++i) {
          if (i < n) {
            ok = can_score(tile + i);
            if (ok) scores(tile + i, i + 1 == n);
          }
          if (i > 0 && ok) {
            ok = can_output(tile + i - 1, i == 1);
            if (ok) outputs(tile + i - 1, i == 1);
          }
        }
      }
      tile += n;
      ++pieces;
    }
    // everything issued has completed before the block gives its memory back
    mma_commit(leader, bar(C::END));
    if (!__all_sync(0xffffffffu, wait_stage_inline(bar(C::END), 0, kTileWait))) *stop = 1;
  } else if (warp == kFeedWarp) {
    // ============================================================================== the work, pages, loads of queries
    int2* const info = static_cast<int2*>(a.workspace);
    int b = sm.start_b, p = sm.start_p, it = 0, known = 0, first = b;  // lane i holds the length of sequence first + i
    bool ok = true;
    uint32_t batch = 0, pieces = 0, tile = 0;
    auto post = [&](const Work& w) {
      ok = warp_wait_on(bar(C::WORK_FREE + (it & 1)), ((it >> 1) & 1) ^ 1, stop, kBlockWait);
      if (!ok) return;
      if (lane == 0) {
        sm.work[it & 1] = w;
        mbar_arrive(bar(C::WORK + (it & 1)));
      }
      ++it;
    };
    for (bool fresh = true; b < a.c.B && p < x1 && x0 < x1 && ok; ++b) {
      if (fresh || b - first == 32) {
        first = b;
        known = b + lane < a.c.B ? (fresh && one_round ? lengths[b + lane] : a.c.seq_lens[b + lane]) : 0;
        fresh = false;
      }
      const int raw = __shfl_sync(0xffffffffu, known, b - first), len = min(max(raw, 0), a.c.S_cap);
      const int n = tiles_of(len, a.window), lo = window_begin(len, a.window);
      const int k0 = max(0, x0 - p - kFixed), k1 = min(n, x1 - p - kFixed);
      if (k1 > k0 || (n == 0 && p >= x0)) {
        const int first_line = (p + kFixed) / share, parts = n > 0 ? (p + kFixed + n - 1) / share - first_line + 1 : 1;
        if (k0 == 0 && group == 0 && lane == 0) {
          info[b] = make_int2(first_line, parts);
          const int bits = (raw != len ? TQ_STATUS_BAD_LEN : 0) | (len == 0 ? TQ_STATUS_EMPTY_SEQ : 0);
          if (bits && a.status) atomicOr(a.status, bits);
        }
        Work w;
        w.b = b;
        w.n = max(0, k1 - k0);
        w.t0 = (lo & ~15) + kTok * k0;
        w.lo = lo;
        w.len = len;
        w.part = parts > 1 ? (2 * line + (k0 == 0)) * groups + group : -1;
        w.more = 1;
        post(w);
        const int last = (len - 1) >> 4;
        for (int i = 0; i < w.n && ok; i += kBatch, ++batch) {
          ok = warp_wait_on(bar(C::PAGES_FREE + (batch & 1)), ((batch >> 1) & 1) ^ 1, stop, kBlockWait);
          if (!ok) break;
          const int j = (w.t0 >> 4) + 4 * i + lane;
          bool good;
          const long long blk = latent_block(a.c, b, min(j, last), good);
          if (!good && a.status) atomicOr(a.status, TQ_STATUS_BAD_PAGE);
          sm.pages[batch & 1][lane] = static_cast<int>(blk);
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::PAGES + (batch & 1)));
          if constexpr (C::BYTES) {
            // (the tiles come by TMA; the scales are asked for by the warps that make factors of them)
            if (j <= last && lane < 4 * (w.n - i))
              asm volatile("prefetch.global.L2 [%0];\n" ::"l"(a.c.blocks + blk * latent_block_bytes(DC) + latent_scale_offset(DC, 0)) : "memory");
            // the tiles' values: a lane per block of 16 tokens and 128 channels, or positional part
            for (int x = 0; x < kBatch && i + x < w.n && ok; ++x, ++tile) {
              const int buf = tile % C::NB;
              ok = warp_wait_on(bar(C::EMPTY + buf), ((tile / C::NB) & 1) ^ 1, stop, kBlockWait);
              const int from = __shfl_sync(0xffffffffu, static_cast<int>(blk), 4 * x + (lane & 3)), unit = lane >> 2;
              if (!ok) break;
              if (lane == 0) mbar_expect_tx(bar(C::FULL + buf), C::TILE + (TEST && static_cast<int>(tile) == hook.fault_tile ? 16 : 0));
              __syncwarp();
              const uint32_t to = base + C::RING + buf * C::TILE + unit * kPanel + (lane & 3) * 2048;
              if (unit < C::UNITS) tma_load_4d(to, &maps.c, 0, 0, unit, from, bar(C::FULL + buf));
              else if (unit == C::UNITS) tma_load_3d(to, &maps.r, 0, 0, from, bar(C::FULL + buf));
            }
            continue;
          }
          if (i == 0) {
            // the queries: heads beyond the last one are zeros, those beyond the group's are not looked at
            ok = warp_wait_on(bar(C::QUERY_FREE), (pieces & 1) ^ 1, stop, kBlockWait);
            if (!ok) break;
            if (lane == 0) {
              mbar_expect_tx(bar(C::RAW), C::PANELS * C::QPANEL);
              for (int x = 0; x < DC / 64; ++x) tma_load_3d(base + C::Q + x * C::QPANEL, &maps.c, 64 * x, h0, b, bar(C::RAW));
              tma_load_3d(base + C::Q + (DC / 64) * C::QPANEL, &maps.r, 0, h0, b, bar(C::RAW));
            }
            ++pieces;
          }
          if (j <= last && lane < 4 * (w.n - i))
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(a.c.blocks + blk * latent_block_bytes(DC)), "r"(latent_block_bytes(DC)) : "memory");
        }
      }
      p += n + kFixed;
    }
    if (ok) post(Work{});
    // loads on their way land before the block ends (whoever waits for them may have given up)
    if (pieces > 0) wait_stage_inline(bar(C::RAW), (pieces - 1) & 1, kMaxWaitCycles);
    for (uint32_t x = 0; C::BYTES && x < C::NB && x < tile; ++x) {
      const uint32_t n = tile - 1 - x;
      wait_stage_inline(bar(C::FULL + n % C::NB), (n / C::NB) & 1, kMaxWaitCycles);
    }
  } else if (C::TURNED) {
    // ============================================================================================ factors of tokens
    const int row = 32 * (warp - kFactorWarp) + lane;
    bool ok = true;
    uint32_t tile = 0, batch = 0;
    Work w;
    for (int it = 0; ok && next_work(it, w, true) && w.more; ++it) {
      auto scales = [&](int i) {
        if (i % kBatch == 0) ok = ok && warp_wait_on(bar(C::PAGES + (batch & 1)), (batch >> 1) & 1, stop, kBlockWait);
        if (!ok) return make_float2(0.0f, 0.0f);
        const int blk = sm.pages[batch & 1][4 * (i % kBatch) + (row >> 4)];
        if (i % kBatch == kBatch - 1 || i == w.n - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::PAGES_FREE + (batch & 1)));
          ++batch;
        }
        return token_scales(a.c.blocks, blk, DC, row);
      };
      float2 next = w.n > 0 ? scales(0) : make_float2(0.0f, 0.0f);
      for (int i = 0; i < w.n && ok; ++i, ++tile) {
        const float2 sc = next;
        if (i + 1 < w.n) next = scales(i + 1);
        const int at = w.t0 + kTok * i + row, slot = tile % kSlots;
        float4 f = token_factors(sc, at >= w.lo && at < w.len);
        if (C::BYTES) f.x *= 9.765625e-4f;  // 2^-10, see digits
        ok = ok && warp_wait_on(bar(C::FACTORS_FREE + slot), ((tile / kSlots) & 1) ^ 1, stop, kBlockWait);
        if (!ok) break;
        sm.factors[slot][row] = f;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::FACTORS + slot));
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_free(tmem, C::COLS);
  if (tid == 0 && sm.stop && a.status) atomicOr(a.status, TQ_STATUS_TIMEOUT);
}

// ---- joining: out = sum_i f_i^2 O_i / sum_i f_i^2 l_i,  f_i = 2^((ref_i - max ref) / 2): halves, as sums are largest where ref is smallest
// How many parts a sequence has depends on its length and on all others', which are known here only.  Every thread block lists the
// sequences that were cut and takes its share of their rows; refs and outputs are asked for together.
//   More than kFew parts: a thread block has 64 channels of a head, 16 threads to a column of four; a thread looks at one
//   part's ref, and the f_i go through shared memory.
//   Fewer: a thread has four channels of a head and every part, and a warp looks at the refs for itself.
// Measured (whole calls in a graph): 8 sequences of 16K tokens, 32 heads, 18 parts each: 52 us in the first form, 48 in the second; 4
// of 32K, 128 heads, 19 parts: 94 and 83; 4 of 32K, 32 heads, 37 parts (first form): 47.  One of 128K among 63 of one token, 16
// heads: 33 us (71 when the form went by the number of sequences).
// A single sequence (ONE) is not listed and takes the first form: 128K tokens, 16 heads 28.2 us instead of 29.8.
constexpr int kJoin = 256, kFew = 24;

__device__ __forceinline__ void store_joined(const LatentArgs& a, long long to, const float4& sum, float l) {
  const float inv = __fdiv_rn(1.0f, l);
  const float4 v = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
  if (a.out_dtype == TQ_FP32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = v;
  else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to) =
      a.out_dtype == TQ_BF16 ? make_uint2(pack2<TQ_BF16>(v.x, v.y), pack2<TQ_BF16>(v.z, v.w)) : make_uint2(pack2<TQ_FP16>(v.x, v.y), pack2<TQ_FP16>(v.z, v.w));
}
__device__ __forceinline__ void add4(float4& sum, float f, const float4& v) {
  sum = make_float4(fmaf(f, v.x, sum.x), fmaf(f, v.y, sum.y), fmaf(f, v.z, sum.z), fmaf(f, v.w, sum.w));
}

template <int DC, int N, bool ONE>
__global__ void __launch_bounds__(kJoin, 4) latent_join_kernel(const LatentArgs a, int groups, int per_group, int lines) {
  __shared__ int4 s_seq[kJoin];  // sequences that were cut: number, first line, parts; from the front those of many parts
  __shared__ int2 s_first[kJoin];
  __shared__ int s_many[kJoin / 32], s_few[kJoin / 32];
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // first line of sequence b and its number of parts; 0: it was not cut.  (The last two conditions: what a call that gave up has
  // left behind.)
  auto cut_of = [&](int b) {
    int2 in = static_cast<const int2*>(a.workspace)[b];
    if (in.y < 2 || in.x < 0 || in.y > lines - in.x) in.y = 0;
    return in;
  };
  unsigned n_many = 0, n_few = 0;
  int4 only;
  if constexpr (ONE) {
    pdl_wait();
    const int2 in = cut_of(0);
    n_many = in.y > 0;
    only = make_int4(0, in.x, in.y, 0);
  } else {
    // at most one of those that begin in a line goes on into the next: by first line they have an order, the same in every
    // thread block
    s_first[tid] = make_int2(0, 0);
    __syncthreads();
    pdl_wait();
    for (int b = tid; b < a.c.B; b += kJoin) {
      const int2 in = cut_of(b);
      if (in.y > 0) s_first[in.x] = make_int2(b, in.y);
    }
    __syncthreads();
    const int2 cut = s_first[tid];
    const unsigned many = __ballot_sync(0xffffffffu, cut.y > kFew), few = __ballot_sync(0xffffffffu, cut.y > 0 && cut.y <= kFew);
    s_many[warp] = __popc(many);
    s_few[warp] = __popc(few);
    __syncthreads();
    int many_before = 0, few_before = 0;
#pragma unroll
    for (int i = 0; i < kJoin / 32; ++i) {
      if (i == warp) many_before = n_many, few_before = n_few;
      n_many += s_many[i];
      n_few += s_few[i];
    }
    const unsigned below = (1u << lane) - 1;
    if (cut.y > 0)
      s_seq[cut.y > kFew ? many_before + __popc(many & below) : kJoin - 1 - few_before - __popc(few & below)] = make_int4(cut.x, tid, cut.y, 0);
    __syncthreads();
  }

  const float* const parts = reinterpret_cast<const float*>(static_cast<const char*>(a.workspace) + info_bytes(a.c.B));
  const int stride = 2 * groups * part_floats(DC, N);
  // part i of head h (the first one stands a place further than the line would say)
  auto part_of = [&](const int4& in, int h, int i) {
    return parts + static_cast<long long>(2 * in.y * groups + h / per_group) * part_floats(DC, N) + static_cast<long long>(i) * stride +
           (i == 0 ? groups * part_floats(DC, N) : 0);
  };
  {
    constexpr int LANES = 16, WIDE = kJoin / LANES, CHUNKS = DC / 4 / WIDE, AHEAD = ONE ? 10 : 8;  // (148 parts; 8 leave registers for the rest)
    __shared__ float4 s_sum[kJoin / 32][WIDE];
    __shared__ float s_f[kJoin], s_max[2][kJoin / 32], s_l[kJoin / 32];
    const int own = tid / WIDE;
    for (unsigned x = blockIdx.x; x < n_many * a.H * CHUNKS; x += gridDim.x) {
      const int h = ONE ? x / CHUNKS : x / CHUNKS % a.H, head = h % per_group, column = (x % CHUNKS) * WIDE + tid % WIDE;
      const int4 in = ONE ? only : s_seq[x / CHUNKS / a.H];
      const int n = in.z;
      auto load = [&](int i) { return *reinterpret_cast<const float4*>(part_of(in, h, i) + head * DC + 4 * column); };
      // ref of the joined row: the largest score part, and the largest of the rest beside it
      const bool mine = tid < n;  // (there are fewer parts than threads)
      const float* const q = part_of(in, h, mine ? tid : 0) + N * DC + head;
      const float z = mine ? q[0] : -INFINITY, o = mine ? q[N] : 0.0f, sums = mine ? q[2 * N] : 0.0f;
      float4 first[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) first[k] = own + k * LANES < n ? load(own + k * LANES) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      auto block_max = [&](float v, float* s) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
        if (lane == 0) s[warp] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int i = 1; i < kJoin / 32; ++i) v = fmaxf(v, s[i]);
        return v;
      };
      const float most = block_max(z, s_max[0]);
      const float rest = mine ? (z - most) + o : -INFINITY;
      const float f = ex2(0.5f * (rest - block_max(rest, s_max[1])));
      float total = mine ? f * sums * f : 0.0f;
      if (mine) s_f[tid] = f * f;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
      if (lane == 0) s_l[warp] = total;
      __syncthreads();
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (own + k * LANES < n) add4(sum, s_f[own + k * LANES], first[k]);
      for (int i = own + AHEAD * LANES; i < n; i += LANES) add4(sum, s_f[i], load(i));
      // a warp's threads of a column, then the warps
#pragma unroll
      for (int off = WIDE; off < 32; off *= 2)
        add4(sum, 1.0f, make_float4(__shfl_xor_sync(0xffffffffu, sum.x, off), __shfl_xor_sync(0xffffffffu, sum.y, off),
                                    __shfl_xor_sync(0xffffffffu, sum.z, off), __shfl_xor_sync(0xffffffffu, sum.w, off)));
      if (lane < WIDE) s_sum[warp][lane] = sum;
      __syncthreads();
      if (own == 0) {
        float l = s_l[0];
#pragma unroll
        for (int i = 1; i < kJoin / 32; ++i) {
          add4(sum, 1.0f, s_sum[i][tid]);
          l += s_l[i];
        }
        store_joined(a, (static_cast<long long>(in.x) * a.H + h) * DC + 4 * column, sum, l);
      }
      __syncthreads();
    }
  }
  if constexpr (!ONE) {
    constexpr int COLUMNS = DC / 4, PER = kJoin / COLUMNS, AHEAD = 4;
    static_assert(COLUMNS % 32 == 0 && kFew <= 32, "a warp has one row, and a lane for each part");
    const int column = tid % COLUMNS;
    for (unsigned x = (gridDim.x - 1 - blockIdx.x) * PER + tid / COLUMNS; x < n_few * a.H; x += gridDim.x * PER) {
      const int h = x % a.H, head = h % per_group;
      const int4 in = s_seq[kJoin - 1 - x / a.H];
      const int n = in.z;
      auto load = [&](int i) { return *reinterpret_cast<const float4*>(part_of(in, h, i) + head * DC + 4 * column); };
      const bool mine = lane < n;
      const float* const q = part_of(in, h, mine ? lane : 0) + N * DC + head;
      const float z = mine ? q[0] : -INFINITY, o = mine ? q[N] : 0.0f, sums = mine ? q[2 * N] : 0.0f;
      float4 first[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) first[k] = k < n ? load(k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      auto warp_max = [](float v) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
        return v;
      };
      const float most = warp_max(z), rest = mine ? (z - most) + o : -INFINITY;
      const float f = ex2(0.5f * (rest - warp_max(rest)));
      float l = mine ? f * sums * f : 0.0f;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f * f, k);
        if (k < n) add4(sum, fk, first[k]);
      }
      for (int i = AHEAD; i < n; i += 4) {
        float4 next[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) next[k] = i + k < n ? load(i + k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float fk = __shfl_sync(0xffffffffu, f * f, i + k);
          if (i + k < n) add4(sum, fk, next[k]);
        }
      }
      store_joined(a, (static_cast<long long>(in.x) * a.H + h) * DC + 4 * column, sum, l);
    }
  }
}

// ---- host

// Heads of a thread block (of N columns), and groups of them: at most 64, shared out evenly.
struct Shape {
  int groups, per_group, n, lines;
};
Shape shape_of(int H) {
  Shape s;
  s.groups = (H + 63) / 64;
  s.per_group = (H + s.groups - 1) / s.groups;
  s.n = s.per_group <= 16 ? 16 : (s.per_group <= 32 ? 32 : 64);
  s.lines = std::min(device_sm_count() / s.groups, kJoin);  // (joining has a thread for each)
  if (s.lines < 1) s.lines = 1;
  return s;
}

// The cache's blocks: codes as [blocks][128 channels][token][128 bytes], positional parts as [blocks][token][64].
bool make_cache_maps(LatentMaps* maps, const tq_latent_cache& c) {
  const cuuint64_t bytes = static_cast<cuuint64_t>(latent_block_bytes(c.d_c)), blocks = static_cast<cuuint64_t>(latent_slots(c) / 16);
  const cuuint64_t dims[4] = {128, 16, static_cast<cuuint64_t>(c.d_c / 128), blocks}, strides[3] = {static_cast<cuuint64_t>(c.d_c), 128, bytes};
  const cuuint64_t rope_dims[3] = {kRope, 16, blocks}, rope_strides[2] = {2 * kRope, bytes};
  const cuuint32_t box[4] = {128, 16, 1, 1}, rope_box[3] = {kRope, 16, 1}, ones[4] = {1, 1, 1, 1};
  return encode_fn()(&maps->c, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, c.blocks, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
         encode_fn()(&maps->r, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, c.blocks + latent_rope_offset(c.d_c, 0), rope_dims, rope_strides, rope_box, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DC, int N, bool TEST = false>
cudaError_t launch_n(const LatentArgs& a, const Shape& s, cudaStream_t st, Hook hook = {}) {
  using C = Cfg<DC, N>;
  if constexpr (DC == 512 && !TEST) {
    const int limit = test_hooks().spin_limit.load(std::memory_order_relaxed), fault = test_hooks().fault_block.load(std::memory_order_relaxed);
    if (limit > 0 || fault >= 0) return launch_n<DC, N, true>(a, s, st, {limit > 0 ? limit : static_cast<int>(kTileWait), fault});
  }
  auto* kernel = latent_kernel<DC, N, TEST>;
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit) || !bit) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM)) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  // no more lines than there can be places
  const long long longest = static_cast<long long>(a.c.B) * ((a.max_len + kTok - 1) / kTok + 1 + kFixed);
  const int lines = longest < s.lines ? static_cast<int>(longest) : s.lines;
  LatentMaps maps;
  if (!encode_fn()) return cudaErrorNotSupported;
  const bool made = C::BYTES ? make_cache_maps(&maps, a.c)
                             : make_map(&maps.c, a.q_c.data, a.q_dtype, DC, a.H, a.c.B, a.q_c.row_stride, a.q_c.head_stride, N, 1) &&
                                   make_map(&maps.r, a.q_r.data, a.q_dtype, kRope, a.H, a.c.B, a.q_r.row_stride, a.q_r.head_stride, N, 1);
  if (!made) return cudaErrorInvalidValue;
  if (cudaError_t e = launch_kernel(kernel, dim3(static_cast<unsigned>(lines * s.groups)), dim3(kThreads), C::SMEM, st, maps, a, s.groups, s.per_group, hook))
    return e;
  if (lines == 1) return cudaSuccess;  // nothing is cut
  // (lines cut lines - 1 sequences at most, and (lines - 1) / kFew into more than kFew parts)
  const bool one = a.c.B == 1;
  const long long cut = std::min<long long>(a.c.B, lines - 1), many = one ? 1 : std::min<long long>(cut, (lines - 1) / kFew);
  const long long want = many * a.H * (DC / 64) + (one ? 0 : (cut * a.H * (DC / 4) + kJoin - 1) / kJoin);
  return launch_kernel(one ? latent_join_kernel<DC, N, true> : latent_join_kernel<DC, N, false>,
                       dim3(static_cast<unsigned>(std::min<long long>(want, (one ? 8LL : 4LL) * device_sm_count()))), dim3(kJoin), 0, st, a, s.groups, s.per_group, lines);
}

template <int DC>
cudaError_t launch_dc(const LatentArgs& a, cudaStream_t st) {
  const Shape s = shape_of(a.H);
  if (s.n == 16) return launch_n<DC, 16>(a, s, st);
  return s.n == 32 ? launch_n<DC, 32>(a, s, st) : launch_n<DC, 64>(a, s, st);
}

}  // namespace

size_t latent_workspace_bytes(int B, int H, int d_c) {
  const Shape s = shape_of(H);
  return info_bytes(B) + 2 * static_cast<size_t>(s.lines) * s.groups * part_floats(d_c, s.n) * 4;
}

cudaError_t launch_latent_decode(const LatentArgs& a, cudaStream_t st) {
  switch (a.c.d_c) {
    case 128: return launch_dc<128>(a, st);
    case 256: return launch_dc<256>(a, st);
    default: return launch_dc<512>(a, st);
  }
}

}  // namespace tq

// Decode attention over the 8-bit cache: one query token per sequence, softmax(alpha q . K^T) V over its cached tokens
// (or the last `window` of them), in one launch.
//
//   Scores:  alpha q . k^ = (alpha a_K / 127) sum_c q_c code_c -- the range of a block is one number per KV head and 16
//            tokens, so it multiplies the fp32 accumulator and the tensor cores see exact integer codes in fp16.
//   Output:  o = sum_j 2^(s_j) a_V(j) code_j / (127 sum_j 2^(s_j)).  The weight that enters the second MMA in fp16 is
//            w_j = 2^(s_j + log2 a_V(j) - M' + 7), with M' the running maximum of the whole exponent: a block whose
//            values are small is weighed against the largest contribution, not against the largest score.  The
//            denominator has a maximum M of its own, kept in fp32, and the factor 2^(M' - M) / 2^7 joins them at the end.
//            M' is kept as its distance R = M' - M, so that log2 a_V is never added to a score: next to one of 10^6 it
//            would lose its digits, and the values their scale.
//   Both maxima are raised only when a score exceeds them by more than 2^8: weights stay below 2^15, inside fp16.  The
//   7 puts the subnormals of fp16 as low as that allows: a weight is rounded by 2^-11 of itself down to 2^-21 of the
//   largest contribution, below that by 2^-32 of it (at most; 2^-25 without the 7, where a token of 2^-22.5 was off by
//   6 %, and a long tail of such tokens with it).
//
// What bounds it: HBM.  2 d + 0.5 bytes per token and KV head; per 16-token block a warp issues 2 x d / 16 MMAs, 3 d / 8
// integer and half-precision instructions that widen the codes, and 8 exponentials per lane (2 per score): a quarter
// of what an SM could do in the time that the block takes to arrive.  Measured at d = 128, 64 heads on 8: 128K tokens
// 51.7 us (5.2 TB/s over all; the loop itself takes 38 us, 7.1 TB/s, and the rest is the start, 2 us, the merge of the
// warps, 2.5, and the joining of cut units, 5); 16 sequences of 4K to 64K, 195 us (5.9 TB/s); d = 256, 32K tokens, 32
// heads on 16: 49 us.  1K tokens 9.3 us, latency: 8 thread blocks take a KV head each, five blocks deep in every warp,
// then merge their warps; nothing is cut.  One KV head or two leave most SMs without a share (see `cuts`): 100 000
// tokens, 8 heads on 1, 27 us where the bytes take 4; d = 512 has four warps of arithmetic only: 20 000 tokens, 16 heads
// on 2, 59 us where they take 6.
//
// Work split.  All (sequence, KV head, tile of 8 query heads) units' blocks lie on one line, sequences first; thread
// block i of N takes the positions [i L / N, (i + 1) L / N) of the L in all, whatever the lengths: ragged batches load
// every SM alike, one short sequence still spreads.  (Batches of short sequences are not cut: see by_block and by_warp.)
// With more units than thread blocks each unit also has `lead` positions before its blocks, for what its query, merge and
// output cost; without them a share of many short units took three times as long as one of a few long ones (45
// sequences of 320 to 5130 tokens, 128 heads on 16: 199 us instead of 100).
// A unit that lies in one thread block is finished there; the parts of a cut one go to the workspace, and the last to
// arrive joins them (counters in 256 bytes, a byte per thread block, whatever the shape).  A thread block has 15 warps of
// arithmetic (7 and 4 at d = 256 and 512: registers), each with a ring of three to six stages of one 16-token block, and
// one warp that fills the rings, one bulk copy per block (K codes, V codes and ranges are contiguous): 185 KB in flight
// per SM at d <= 128, 172 and 197 KB at 256 and 512, no barrier in the main loop, and the copies run on into the
// thread block's next unit while this one is merged.
#include <algorithm>
#include <type_traits>

#include "tq_async.cuh"
#include "tq_kv8.cuh"

namespace tq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNoMax = -3.0e38f;  // below every score of fp32 (bf16 inputs reach its whole range), and finite
constexpr float kSlack = 8.0f;  // log2 units a score may exceed the running maxima
constexpr float kRaise = 7.0f;  // log2 of the weight in fp16 that a contribution as large as M' has
constexpr float kLower = 1.0f / 128.0f;  // undoes it, in the accumulators: 2^(M' - M) may be the smallest normal number
constexpr int kMaxGrid = 160;   // thread blocks of a launch (one per SM)
static_assert(kMaxGrid <= kCounterBytes && kMaxGrid < 256, "arrival counters");

template <int D>
struct Cfg {
  static constexpr int NW = D <= 128 ? 15 : (D == 256 ? 7 : 4);  // warps of the arithmetic (registers: 16, 8, 8 warps fit)
  static constexpr int NST = D == 64 ? 6 : 3;                    // stages of a warp's ring
  static constexpr int STAGE = block8_bytes(D);
  static constexpr int THREADS = 32 * NW;                        // ... of the arithmetic; one more warp issues the copies
  static constexpr int LAUNCH = THREADS + 32;
  static constexpr int RING = NW * NST * STAGE;
  // the merge arrays lie behind the rings (copies for the next unit are in flight while a unit is merged); the outputs
  // of the warps go through them MQ query heads at a time
  static constexpr int ROW = D + 4;  // floats of one query's row: 8 rows x 2 words apart hit different banks
  static constexpr int MQ = 2;
  // the last to arrive keeps the weights of a unit's parts there, and the teams' sums behind them
  static constexpr int WTS = 2 * 8 * kMaxGrid * 4 + 16 * THREADS;
  static constexpr int MERGE = NW * MQ * ROW * 4 > WTS ? NW * MQ * ROW * 4 : WTS;
  static constexpr int STATS = RING + MERGE;             // [NW][8] x {M, R, l} and the factors of them
  static constexpr int BARS = STATS + NW * 8 * 3 * 4 + 8 * 4 * 4;
  static constexpr int QS = BARS + 2 * NW * NST * 8;         // d = 512: the query's B fragments, 8 bytes per lane and step
  static constexpr int QBYTES = D == 512 ? (D / 16) * 32 * 8 : 0;
  static constexpr int SMEM = QS + QBYTES;
  static_assert(BARS % 8 == 0 && QS % 8 == 0 && STAGE % 16 == 0 && SMEM <= 232448, "shared memory");
};

// The part of a cut unit that one thread block has done: `rows` rows of output, then their maxima and sums.
__host__ __device__ constexpr int part_floats(int d, int rows) { return rows * d + (2 * rows + 3) / 4 * 4; }
// How many there can be: a thread block cuts two units at most, and a line of U units in N shares has N + U - 1 pieces.
inline long long part_count(long long units, int grid) { return units < grid ? grid + units : 2LL * grid; }

struct Args {
  tq_kv8_cache c;
  const uint16_t* q;
  long long q_stride;
  int H_q, G, tiles, window;
  float scale_log2;  // alpha * log2(e) / 127
  int units;         // H_kv * tiles
  int grid;          // thread blocks launched
  int min_blocks;    // fewest cache blocks worth a thread block
  int lead;          // positions on the line before a unit's blocks (see the top)
  uint32_t* counters;  // a byte for each thread block
  float* parts;      // see part_floats
  int rows;          // query heads of a tile: at most 8
  bool compact;      // fewer units than thread blocks: part of (thread block i, unit u) at i + u, else two per thread block
  void* out;
  int32_t* status;
  // instrumented instantiation only (the library's own tests, see TestHooks): limit of the stage waits in SM cycles, and
  // the 16-token block of every unit whose copy announces 16 bytes too many: its barrier never completes, the data lands
  int wait_cycles, fault_block;
};

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
// stored bytes (code + 128) of a word -> two words of exact fp16 codes
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const __half2 bias = __half2half2(__ushort_as_half(0x6480));  // 1152
  uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
  const __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), bias), y = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
  lo = *reinterpret_cast<const uint32_t*>(&x);
  hi = *reinterpret_cast<const uint32_t*>(&y);
}

// Tokens [lo, hi) that a sequence attends.
struct Span {
  int lo, hi;
  __device__ int first() const { return lo >> 4; }
  __device__ int blocks() const { return hi > lo ? ((hi + 15) >> 4) - (lo >> 4) : 0; }
};
__device__ __forceinline__ Span span_of(const Args& a, int b) {
  int len = a.c.seq_lens[b];
  len = len < 0 ? 0 : (len > a.c.S_cap ? a.c.S_cap : len);
  return {window_begin(len, a.window), len};
}

// A walk over a thread block's share of the line: units, and in a unit the blocks [j0, j1).  With hop > 0 it takes whole
// units instead: unit g (sequences first), then every hop-th one after it.  Positions fit 31 bits (the entry point sees
// to that): they are held through the main loop, and 64-bit divisions cost half a microsecond of latency apiece.
struct Walk {
  int g, g1;  // start of the unit on the line and end of the share; unit and their number
  int hop;
  int b, u, h;      // sequence, unit in it, its KV head
  int j0, j1, n;    // blocks of this visit, blocks of the unit
  Span span;
  __device__ void open(const Args& a, int j) {
    span = span_of(a, b);
    h = a.tiles == 1 ? u : u / a.tiles;
    n = span.blocks();
    j0 = j;
    j1 = hop > 0 ? n : min(n, g1 - g - a.lead);
  }
  // the first unit with a token, from g on
  __device__ bool seek(const Args& a) {
    for (; g < g1; g += hop) {
      b = g / a.units;
      u = g - b * a.units;
      open(a, 0);
      if (n > 0) return true;
    }
    return false;
  }
  __device__ bool next(const Args& a) {
    if (hop > 0) {
      g += hop;
      return seek(a);
    }
    g += a.lead + n;
    if (g >= g1) return false;
    if (++u == a.units) {
      u = 0;
      do {
        if (++b >= a.c.B) {  // lengths that change while the kernel runs break the caller's promise: stop
          g = g1;
          return false;
        }
      } while (span_of(a, b).blocks() == 0);
    }
    open(a, 0);
    return j1 > 0;  // (no: the share ends before the unit's blocks)
  }
};

__device__ __forceinline__ const uint8_t* block_at(const Args& a, int b, int h, int j) {
  if (a.c.page_table == nullptr)
    return a.c.blocks + ((static_cast<long long>(b) * a.c.H_kv + h) * (a.c.S_cap >> 4) + j) * block8_bytes(a.c.d);
  const int shift = __ffs(a.c.page_tokens) - 5;  // log2 of the blocks of a page
  int p = a.c.page_table[static_cast<long long>(b) * a.c.max_pages + (j >> shift)];
  if (p < 0 || p >= a.c.num_pages) {
    if (a.status) atomicOr(a.status, TQ_STATUS_BAD_PAGE);
    p = 0;
  }
  return a.c.blocks + (((static_cast<long long>(p) * a.c.H_kv + h) << shift) + (j & ((1 << shift) - 1))) * block8_bytes(a.c.d);
}

template <int OT>
__device__ __forceinline__ void store_out(void* out, long long at, float x) {
  if (OT == TQ_FP32) static_cast<float*>(out)[at] = x;
  else if (OT == TQ_BF16) static_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);
  else static_cast<__half*>(out)[at] = __float2half_rn(x);
}

template <int OT>
__device__ __forceinline__ void store_out2(void* out, long long at, float x, float y) {
  if (OT == TQ_FP32) *reinterpret_cast<float2*>(static_cast<float*>(out) + at) = make_float2(x, y);
  else *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + at) = pack2<OT>(x, y);
}

// The line of L positions cut into N shares: share i starts at floor(i L / N).
struct Shares {
  int each, rest, N;
  float per;
  __device__ Shares(int L, int n) : each(L / n), rest(L - each * n), N(n) { per = static_cast<float>(n) / static_cast<float>(L); }
  __device__ int start(int i) const { return each * i + i * rest / N; }
  __device__ int owner(int g) const {
    int i = static_cast<int>(static_cast<float>(g) * per);  // off by one at most
    i = i < N ? i : N - 1;
    if (start(i) > g) --i;
    else if (i + 1 < N && start(i + 1) <= g) ++i;
    return i;
  }
};

template <int D, int QT, int OT, bool TEST = false>
__global__ void __launch_bounds__(Cfg<D>::LAUNCH, 1) decode8_kernel(const Args a) {
  using C = Cfg<D>;
  constexpr int KK = D / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_start, s_warp[C::NW + 1], s_top[C::NW + 1];
  __shared__ int s_b, s_last, s_dead, s_from, s_to, s_line[3];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gid = lane >> 2, t4 = lane & 3;
  float* const merge = reinterpret_cast<float*>(smem + C::RING);
  float* const stats = reinterpret_cast<float*>(smem + C::STATS);  // [3][NW][8]
  float* const sums = stats + 3 * C::NW * 8;                       // [8] x {M, R, l, factor}
  // warp w's ring of NST stages, and the barriers "stage s is full" and "stage s may be filled" behind all rings
  uint32_t base;
  asm("{ .reg .u64 p; cvta.to.shared.u64 p, %1; cvt.u32.u64 %0, p; }\n" : "=r"(base) : "l"(smem));
  auto full = [&](int w, int s) { return base + C::BARS + (w * C::NST + s) * 8; };
  auto empty = [&](int w, int s) { return base + C::BARS + (C::NW * C::NST + w * C::NST + s) * 8; };
  if (tid == 0) s_dead = 0;
  for (int i = tid; i < 2 * C::NW * C::NST; i += C::LAUNCH) mbar_init(base + C::BARS + 8 * i, 1);
  asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait();

  const bool few = a.c.B <= 32;  // a warp sums the lengths up by itself: every warp does, and no barrier is needed

  // ---- where this thread block's share starts: blocks of all sequences, then the sequence that holds the start
  int most = 0;                       // longest unit on the line
  auto scan = [&](int v, int& sum) {  // inclusive sum over the threads; `sum`: that of all
    int x = v;
    const int top = __reduce_max_sync(0xffffffffu, v);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (few) {
      sum = __shfl_sync(0xffffffffu, x, 31);
      most = top;
      return x;
    }
    if (lane == 31) {
      s_warp[warp] = x;
      s_top[warp] = top;
    }
    __syncthreads();
    int add = 0, all = 0;
#pragma unroll
    for (int w = 0; w <= C::NW; ++w) {
      const int y = s_warp[w];
      if (w < warp) add += y;
      all += y;
      most = max(most, s_top[w]);
    }
    __syncthreads();
    sum = all;
    return x + add;
  };
  auto on_line = [&](int n) { return n > 0 ? n + a.lead : 0; };  // a unit's length
  int L = 0;
  int own_n = 0;  // a unit of the thread's sequence on the line, and of all up to it, in the last round
  int own_upto = 0;
  for (int round = 0; round < a.c.B; round += C::LAUNCH) {
    const int b = few ? lane : round + tid;
    own_n = 0;
    if (b < a.c.B) {
      own_n = on_line(span_of(a, b).blocks());
      const int len = a.c.seq_lens[b];
      if (blockIdx.x == 0 && a.status && (!few || warp == 0) && (len <= 0 || len > a.c.S_cap))
        atomicOr(a.status, (len < 0 || len > a.c.S_cap ? TQ_STATUS_BAD_LEN : 0) | (len <= 0 ? TQ_STATUS_EMPTY_SEQ : 0));
    }
    if (a.c.B == 1) {  // nothing to sum up
      own_n = __shfl_sync(0xffffffffu, own_n, 0);
      L = own_upto = most = own_n;
      break;
    }
    int all;
    own_upto = scan(own_n, all);
    L += all;
  }
  L *= a.units;
  const int U = a.c.B * a.units;
  const int worth = (L - 1) / a.min_blocks + 1;
  int N = worth < 1 ? 1 : (worth < a.grid ? worth : a.grid);
  if (a.lead > 0) N = max(1, min(L, a.grid));
  // Short sequences are not cut.  With no more units than thread blocks, the longest of which is at most 66 blocks (6 us)
  // above a share, a thread block takes one unit: joining a cut one costs that (16 units of 63 blocks: 19 us cut into 17
  // shares).  With more units a warp takes whole units, without a merge, where the longest, at 0.5 us per block, is done
  // before the shares would be, at 0.075 us per position and 8 us for the joining (18 x 8 units of up to 8 blocks: 168 us
  // in shares without leads; 58 x 16 of up to 99: 132 us so, 51 by warps).
  const bool by_block = U <= static_cast<int>(gridDim.x) && most <= L / N + 66;
  const bool by_warp = D < 512 && a.lead > 0 && !by_block &&  // (d = 512: the warps share the query's fragments)
                       most - a.lead <= L / N / 7 + 16;

  // Few units: shares that end where units do save the thread blocks in between a second query and merge (6 us).  Each
  // unit of a sequence gets floor(its part of the line x N) of them; that lengthens the longest share, by 0.09 us per
  // block, and is done up to 66 blocks (10 sequences of 207 to 3321 tokens, one KV head: 14.8 us, not so 20).  No unit
  // gets more than half the root of its blocks: one thread block joins the parts, at 0.15 to 0.6 us each (30 000 tokens,
  // one KV head of 256: 67 parts 55 us, 16 parts 30).  The 66 do not count what this second limit lengthens: 8192 blocks
  // of one KV head make 45 shares of 182, where 148 would have 56 each.  (Batches of more than 32 stay on the line,
  // because only there does a warp have all sums, not because it serves them better: 60 sequences of 147 to 2357 tokens,
  // one KV head, 28 us; 22 of 171 to 2738, two KV heads, in shares that end with units 14.6, on the line 26.)
  int cuts = 0, cuts_upto = 0;  // shares of each unit of the lane's sequence, and of those up to it
  bool snapped = false;
  if (few && !by_block && a.lead == 0 && U <= N) {
    const int n = lane < a.c.B ? own_n : 0;
    const float part = static_cast<float>(n) / static_cast<float>(L / a.units);  // (1 exactly for a single sequence)
    const int even = max(1, static_cast<int>(part * static_cast<float>(N / a.units)));
    cuts = min(min(n, even), max(1, static_cast<int>(0.5f * sqrtf(static_cast<float>(n)))));  // (none of them is empty)
    cuts_upto = cuts;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, cuts_upto, o);
      if (lane >= o) cuts_upto += y;
    }
    const bool fits = __shfl_sync(0xffffffffu, cuts_upto, 31) * a.units <= N;
    snapped = fits && __all_sync(0xffffffffu, n == 0 || (n - 1) / even + 1 <= L / N + 66);
    if (snapped) N = __shfl_sync(0xffffffffu, cuts_upto, 31) * a.units;
  }

  // sequences without a token: their rows are zero
  if (!few || __any_sync(0xffffffffu, lane < a.c.B && own_n == 0))
    for (int b = blockIdx.x; b < a.c.B; b += gridDim.x) {
      if (span_of(a, b).blocks() != 0) continue;
      for (int i = tid; i < a.H_q * D; i += C::LAUNCH) store_out<OT>(a.out, static_cast<long long>(b) * a.H_q * D + i, 0.0f);
    }
  if (L == 0 || (!by_block && !by_warp && static_cast<int>(blockIdx.x) >= N)) return;

  const Shares shares(L, N);
  const int g0 = shares.start(min(static_cast<int>(blockIdx.x), N));
  if (tid == 0) {  // for the merges of cut units: kept out of the main loop's registers
    s_line[0] = L;
    s_line[1] = N;
    s_line[2] = g0;
    s_from = -1;
  }
  int first_b;
  int first_at;
  auto claim = [&](int b, int n, int upto) {  // the sequence that holds the start of the share
    if (n > 0 && upto * a.units > g0 && (upto - n) * a.units <= g0) {
      s_b = b;
      s_start = (upto - n) * a.units;
    }
  };
  if (by_block || by_warp || snapped) {
    first_b = 0;
    first_at = 0;
  } else if (few) {
    // the owner's lane tells its warp
    const bool holds = own_n > 0 && own_upto * a.units > g0 && (own_upto - own_n) * a.units <= g0;
    const int from = __ffs(static_cast<int>(__ballot_sync(0xffffffffu, holds))) - 1;
    first_b = from;
    first_at = __shfl_sync(0xffffffffu, (own_upto - own_n) * a.units, from);
  } else if (a.c.B <= C::LAUNCH) {
    claim(tid, own_n, own_upto);
  } else {
    int carry = 0;
    for (int round = 0; round < a.c.B; round += C::LAUNCH) {
      const int b = round + tid;
      const int n = b < a.c.B ? on_line(span_of(a, b).blocks()) : 0;
      int all;
      const int upto = scan(n, all);
      claim(b, n, carry + upto);
      carry += all;
    }
  }
  if (!few && !by_block && !by_warp) {
    __syncthreads();
    first_b = s_b;
    first_at = s_start;
  }
  Walk use;
  bool any = true;
  if (by_block || by_warp) {
    use.g = by_block ? static_cast<int>(blockIdx.x) : (warp < C::NW ? warp : lane) * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
    use.g1 = warp == C::NW && lane >= C::NW ? 0 : U;
    use.hop = by_block ? static_cast<int>(gridDim.x) : static_cast<int>(gridDim.x) * C::NW;
    any = use.seek(a);
  } else if (snapped) {
    const int i = blockIdx.x;
    const int from = __ffs(static_cast<int>(__ballot_sync(0xffffffffu, cuts_upto * a.units > i))) - 1;
    const int c = __shfl_sync(0xffffffffu, cuts, from), at = i - (__shfl_sync(0xffffffffu, cuts_upto, from) - c) * a.units;
    use.hop = 0;
    use.b = from;
    use.u = at / c;
    const int x = at - use.u * c, n = __shfl_sync(0xffffffffu, own_n, from);
    const int each = n / c, rest = n - each * c;  // part x has the blocks [floor(n x / c), floor(n (x + 1) / c))
    const int lo = each * x + rest * x / c, hi = each * (x + 1) + rest * (x + 1) / c;
    use.g = (__shfl_sync(0xffffffffu, own_upto, from) - n) * a.units + use.u * n;
    use.g1 = use.g + hi;
    use.open(a, lo);
    if (tid == 0) {
      s_from = i - x;
      s_to = i - x + c - 1;
    }
  } else {
    use.hop = 0;
    use.g1 = shares.start(blockIdx.x + 1);
    use.b = first_b;
    const int n = on_line(span_of(a, use.b).blocks());
    const int r = g0 - first_at;
    use.u = r / n;
    const int at = r - use.u * n;
    use.g = g0 - at;
    use.open(a, max(0, at - a.lead));
    any = use.j1 > use.j0;
  }

  if (warp == C::NW) {
    // ---- copies: lane w fills warp w's ring, ahead of its arithmetic and on into the next units
    bool more = any && lane < C::NW;
    const int at = by_warp ? 0 : lane, step = by_warp ? 1 : C::NW;
    int j = any ? use.j0 + at : 0, stage = 0;
    uint32_t phase = 1;  // the first pass over a ring finds every stage free
    long long since = clock64();
    while (true) {
      while (more && j >= use.j1) {  // the warp's next block may lie in a later unit
        more = use.next(a);
        j = use.j0 + at;
      }
      if (!__any_sync(0xffffffffu, more)) break;
      bool sent = false;
      if (more && mbar_test_wait(empty(lane, stage), phase)) {
        const uint8_t* src = block_at(a, use.b, use.h, use.span.first() + j);
        mbar_expect_tx(full(lane, stage), C::STAGE + (TEST && use.span.first() + j == a.fault_block ? 16 : 0));
        bulk_g2s(base + (lane * C::NST + stage) * C::STAGE, src, C::STAGE, full(lane, stage));
        j += step;
        if (++stage == C::NST) {
          stage = 0;
          phase ^= 1;
        }
        sent = true;
      }
      if (__any_sync(0xffffffffu, sent)) {
        since = clock64();
      } else {
        if (clock64() - since > 4 * kMaxWaitCycles) break;  // its readers have given up (they report it)
        __nanosleep(64);
      }
    }
    // Whatever is still on its way lands before the warp ends (bounded): a reader that has given up did not wait for it.
    // (A stage that was never filled answers at once.)
    if (lane < C::NW)
      for (int s = 0; s < C::NST; ++s) {
        const int x = (stage + s) % C::NST;
        wait_stage(full(lane, x), x >= stage ? phase : phase ^ 1);
      }
    return;
  }
  auto join_warps = [&]() { asm volatile("bar.sync 1, %0;\n" ::"n"(C::THREADS) : "memory"); };

  int stage = 0;
  uint32_t phase = 0;
  bool dead = false;

  for (bool go = any; go; go = use.next(a)) {
    const int h = use.h, tile = use.u - h * a.tiles;
    const int head0 = h * a.G + tile * 8;
    const int heads = a.G - tile * 8 < 8 ? a.G - tile * 8 : 8;

    // ---- B fragments of the scores: query gid, channels 32 kk + 8 t4 .. + 7 (both k = 16 steps).  bf16 queries are
    // scaled by a power of two per query into the range of fp16: exact down to 2^-28 of the query's largest value.
    uint32_t qf[D == 512 ? 1 : KK][4];
    float back = 1.0f;  // undoes that scale
    {
      const bool real = gid < heads;
      const uint16_t* src = a.q + static_cast<long long>(use.b) * a.q_stride + static_cast<long long>(head0 + gid) * D + 8 * t4;
      float mul = 1.0f;
      if (QT == TQ_BF16) {
        float top = 0.0f;
        for (int kk = 0; kk < KK; ++kk) {
          const uint4 x = real ? __ldg(reinterpret_cast<const uint4*>(src + 32 * kk)) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          for (int e = 0; e < 4; ++e) {
            const float2 f = unpack2<QT>(w[e]);
            top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = static_cast<int>(__float_as_uint(top) >> 23) - 127;  // exponent; 128: infinite
        if (top > 0.0f && e < 128) {
          int by = 13 - e;
          by = by > 126 ? 126 : by;
          mul = __uint_as_float(static_cast<uint32_t>(127 + by) << 23);
          back = __uint_as_float(static_cast<uint32_t>(127 - by) << 23);
        }
      }
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint4 x = real ? __ldg(reinterpret_cast<const uint4*>(src + 32 * kk)) : make_uint4(0, 0, 0, 0);
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
        if (QT == TQ_BF16) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = unpack2<QT>(w[e]);
            w[e] = pack2<TQ_FP16>(f.x * mul, f.y * mul);
          }
        }
        if (D == 512) {
          uint2* to = reinterpret_cast<uint2*>(smem + C::QS);
          if (warp == 0) {
            to[(2 * kk) * 32 + lane] = make_uint2(w[0], w[1]);
            to[(2 * kk + 1) * 32 + lane] = make_uint2(w[2], w[3]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) qf[D == 512 ? 0 : kk][e] = w[e];
        }
      }
      if (D == 512) join_warps();
    }
    const float back0 = __shfl_sync(0xffffffffu, back, 8 * t4), back1 = __shfl_sync(0xffffffffu, back, 8 * t4 + 4);

    float o[2 * KK][4];  // channels 16 m + gid (+ 8), queries 2 t4 (+ 1)
#pragma unroll
    for (int m = 0; m < 2 * KK; ++m) o[m][0] = o[m][1] = o[m][2] = o[m][3] = 0.0f;
    float M0 = kNoMax, M1 = kNoMax, R0 = kNoMax, R1 = kNoMax, l0 = 0.0f, l1 = 0.0f;

    for (int j = use.j0 + (by_warp ? 0 : warp); j < use.j1; j += by_warp ? 1 : C::NW) {
      if (!dead && !wait_stage(full(warp, stage), phase, TEST ? a.wait_cycles : kMaxWaitCycles)) {
        dead = true;
        s_dead = 1;
        if (a.status && lane == 0) atomicOr(a.status, TQ_STATUS_TIMEOUT);
      }
      dead = __any_sync(0xffffffffu, dead);
      if (dead) break;
      const uint8_t* blk = smem + (warp * C::NST + stage) * C::STAGE;
      float s[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint4 x = *reinterpret_cast<const uint4*>(blk + 512 * kk + 16 * lane);
        uint32_t f0[4], f1[4];  // rows gid: words x, y; rows gid + 8: words z, w; x and z are the first k = 16 step
        widen(x.x, f0[0], f0[2]);
        widen(x.z, f0[1], f0[3]);
        widen(x.y, f1[0], f1[2]);
        widen(x.w, f1[1], f1[3]);
        if (D == 512) {
          const uint2* from = reinterpret_cast<const uint2*>(smem + C::QS);
          const uint2 b0 = from[(2 * kk) * 32 + lane], b1 = from[(2 * kk + 1) * 32 + lane];
          mma16816(s[0], f0, b0.x, b0.y);
          mma16816(s[1], f1, b1.x, b1.y);
        } else {
          mma16816(s[0], f0, qf[kk][0], qf[kk][1]);
          mma16816(s[1], f1, qf[kk][2], qf[kk][3]);
        }
      }
      const float2 range = *reinterpret_cast<const float2*>(blk + 32 * D);
      const float f = range.x * a.scale_log2;
      const float f0 = f * back0, f1 = f * back1;
      float s0 = (s[0][0] + s[1][0]) * f0, s1 = (s[0][1] + s[1][1]) * f1;  // token gid
      float s2 = (s[0][2] + s[1][2]) * f0, s3 = (s[0][3] + s[1][3]) * f1;  // token gid + 8
      const int tok = (use.span.first() + j) * 16 + gid;
      if (tok < use.span.lo || tok >= use.span.hi) s0 = s1 = -INFINITY;
      if (tok + 8 < use.span.lo || tok + 8 >= use.span.hi) s2 = s3 = -INFINITY;
      float lg;  // log2 of the value range; -inf for a block of zeros
      asm("lg2.approx.f32 %0, %1;\n" : "=f"(lg) : "f"(range.y));
      const float b0 = fmaxf(s0, s2), b1 = fmaxf(s1, s3);
      if (__any_sync(0xffffffffu, b0 > M0 + kSlack || b1 > M1 + kSlack || b0 - M0 + lg > R0 + kSlack || b1 - M1 + lg > R1 + kSlack)) {
        float m0 = b0, m1 = b1;
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
          m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, x));
          m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, x));
        }
        const float n0 = fmaxf(M0, m0), n1 = fmaxf(M1, m1), d0 = M0 - n0, d1 = M1 - n1;
        const float r0 = fmaxf(kNoMax, fmaxf(R0 + d0, m0 - n0 + lg)), r1 = fmaxf(kNoMax, fmaxf(R1 + d1, m1 - n1 + lg));
        l0 *= ex2(d0);
        l1 *= ex2(d1);
        const float c0 = ex2(d0 + R0 - r0), c1 = ex2(d1 + R1 - r1);
        M0 = n0;
        M1 = n1;
        R0 = r0;
        R1 = r1;
#pragma unroll
        for (int m = 0; m < 2 * KK; ++m) {
          o[m][0] *= c0;
          o[m][1] *= c1;
          o[m][2] *= c0;
          o[m][3] *= c1;
        }
      }
      s0 -= M0;
      s1 -= M1;
      s2 -= M0;
      s3 -= M1;
      l0 += ex2(s0) + ex2(s2);
      l1 += ex2(s1) + ex2(s3);
      const float w0 = lg - R0 + kRaise, w1 = lg - R1 + kRaise;
      const uint32_t v0 = transpose8x8(pack2<TQ_FP16>(ex2(s0 + w0), ex2(s1 + w1)));  // tokens 2 t4, + 1 of query gid
      const uint32_t v1 = transpose8x8(pack2<TQ_FP16>(ex2(s2 + w0), ex2(s3 + w1)));  // tokens 2 t4 + 8, + 9
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint4 x = *reinterpret_cast<const uint4*>(blk + 16 * D + 512 * kk + 16 * lane);
        uint32_t e[4];
        widen(x.x, e[0], e[2]);
        widen(x.y, e[1], e[3]);
        mma16816(o[2 * kk], e, v0, v1);
        widen(x.z, e[0], e[2]);
        widen(x.w, e[1], e[3]);
        mma16816(o[2 * kk + 1], e, v0, v1);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(warp, stage));
      if (++stage == C::NST) {
        stage = 0;
        phase ^= 1;
      }
    }

    // ---- join the warps: maxima and sums first, then the outputs, MQ query heads at a time
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, x);
      l1 += __shfl_xor_sync(0xffffffffu, l1, x);
    }
    if (by_warp) {
      // the warp's own unit: straight out of the accumulators
      const float f0 = ex2(R0) / (127.0f * l0), f1 = ex2(R1) / (127.0f * l1);
      const long long at = (static_cast<long long>(use.b) * a.H_q + head0 + 2 * t4) * D + gid;
#pragma unroll
      for (int m = 0; m < 2 * KK; ++m) {
        if (2 * t4 < heads) {
          store_out<OT>(a.out, at + 16 * m, o[m][0] * kLower * f0);
          store_out<OT>(a.out, at + 16 * m + 8, o[m][2] * kLower * f0);
        }
        if (2 * t4 + 1 < heads) {
          store_out<OT>(a.out, at + D + 16 * m, o[m][1] * kLower * f1);
          store_out<OT>(a.out, at + D + 16 * m + 8, o[m][3] * kLower * f1);
        }
      }
      continue;
    }
    if (gid == 0) {
      float* st = stats + warp * 8 + 2 * t4;
      st[0] = M0;
      st[1] = M1;
      st[C::NW * 8] = R0;
      st[C::NW * 8 + 1] = R1;
      st[2 * C::NW * 8] = l0;
      st[2 * C::NW * 8 + 1] = l1;
    }
    const bool whole = use.j0 == 0 && use.j1 == use.n;
    const int u0 = use.g + a.lead;  // the unit's first block on the line, and the thread blocks that share the unit
    join_warps();
    int from = 0, to = 0, slot = 0;  // the thread blocks that share the unit; which of this one's two parts it is
    if (!whole) {
      slot = use.g <= s_line[2] ? 0 : 1;
      from = s_from;
      to = s_to;
      if (from < 0) {
        const Shares shares(s_line[0], s_line[1]);
        from = shares.owner(u0);
        to = shares.owner(u0 + use.n - 1);
      }
    }
    for (int q = warp; q < 8; q += C::NW) {
      const bool has = lane < C::NW;
      const float wm = has ? stats[lane * 8 + q] : kNoMax;
      float m = wm, r = has ? stats[(C::NW + lane) * 8 + q] : kNoMax;
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m, x), r2 = __shfl_xor_sync(0xffffffffu, r, x), n = fmaxf(m, m2);
        r = fmaxf(r + (m - n), r2 + (m2 - n));
        m = n;
      }
      float l = has ? stats[(2 * C::NW + lane) * 8 + q] * ex2(wm - m) : 0.0f;
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
      if (lane == 0) {
        sums[q] = m;
        sums[8 + q] = r;
        sums[16 + q] = l;
        sums[24 + q] = ex2(r) / (127.0f * l);
      }
    }
    join_warps();
    const long long unit = static_cast<long long>(use.b) * a.units + use.u;
    const int stride = part_floats(D, a.rows);
    float* const mine = a.parts + (a.compact ? blockIdx.x + unit : 2LL * blockIdx.x + slot) * stride;
    const float c0 = ex2(M0 - sums[2 * t4] + R0 - sums[8 + 2 * t4]) * kLower, c1 = ex2(M1 - sums[2 * t4 + 1] + R1 - sums[8 + 2 * t4 + 1]) * kLower;
    auto emit = [&](int q, int ch, float x, float y) {
      x *= sums[24 + q];
      y *= sums[24 + q];
      if (whole) store_out2<OT>(a.out, (static_cast<long long>(use.b) * a.H_q + head0 + q) * D + ch, x, y);
      else *reinterpret_cast<float2*>(mine + q * D + ch) = make_float2(x, y);
    };
    // rows of the warps' queries q0 .. q0 + MQ - 1 in `area`, summed over the warps
    auto join = [&](float* area, int q0, auto mq) {
      constexpr int MQ = decltype(mq)::value;
      if (MQ == 8 || 2 * t4 == q0) {
        float* row = area + (warp * MQ + (MQ == 8 ? 2 * t4 : 0)) * C::ROW;
#pragma unroll
        for (int m = 0; m < 2 * KK; ++m) {
          row[16 * m + gid] = o[m][0] * c0;
          row[16 * m + gid + 8] = o[m][2] * c0;
          row[C::ROW + 16 * m + gid] = o[m][1] * c1;
          row[C::ROW + 16 * m + gid + 8] = o[m][3] * c1;
        }
      }
      join_warps();
      for (int i = tid; i < MQ * (D / 2); i += C::THREADS) {
        const int q = i / (D / 2), ch = 2 * (i - q * (D / 2));
        float2 x = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < C::NW; ++w) {
          const float2 y = *reinterpret_cast<const float2*>(area + (w * MQ + q) * C::ROW + ch);
          x.x += y.x;
          x.y += y.y;
        }
        if (q0 + q < heads) emit(q0 + q, ch, x.x, x.y);
      }
      join_warps();
    };
    // On the thread block's last visit nothing is on its way into the rings any more (every warp has used what it asked
    // for, and the barriers above are behind that): all eight rows at once through the rings' memory.
    if ((use.hop > 0 ? use.g + use.hop : u0 + use.j1) >= use.g1 && !s_dead) {
      join(reinterpret_cast<float*>(smem), 0, std::integral_constant<int, 8>{});
    } else {
      for (int q0 = 0; q0 < heads; q0 += C::MQ) join(merge, q0, std::integral_constant<int, C::MQ>{});
    }
    if (!whole) {
      if (tid < a.rows) {
        mine[a.rows * D + tid] = sums[tid];
        mine[a.rows * D + a.rows + tid] = sums[16 + tid];
      }
      join_warps();
      if (tid == 0) {
        // The unit's counter is the byte of the thread block that holds its first part (at most one cut unit begins there).
        // This releases the block's writes, which the barrier orders before it, and acquires those of the blocks before.
        uint32_t* const word = a.counters + (from >> 2);
        const uint32_t shift = 8 * (from & 3);
        uint32_t got;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;\n" : "=r"(got) : "l"(word), "r"(1u << shift) : "memory");
        s_last = static_cast<int>(got >> shift & 0xff) == to - from;
        if (s_last) atomicSub(word, static_cast<uint32_t>(to - from + 1) << shift);  // left as it was found
      }
      join_warps();
      if (s_last) {
        // the first part is its thread block's second one
        const int skip = a.compact || Shares(s_line[0], s_line[1]).start(from) >= use.g ? 0 : 1;
        const int np = to - from + 1;
        auto part_of = [&](int p) {
          return a.parts + (a.compact ? from + p + unit : 2LL * (from + p) + (p == 0 ? skip : 0)) * stride;
        };
        // The maxima and sums of all parts at once, one query head per warp for the weights; then the rows.  The loads are
        // independent of each other, and the first CH rows are on their way while the weights are made (a running maximum
        // would wait for a round trip to L2 per part: 17 us of a 64 us launch).
        // Few rows and many parts: `teams` of threads share the parts of a row.
        constexpr int CH = D <= 128 ? 9 : 16;
        float* const wts = merge;  // [2][8][np]
        float4 rows[CH];
        const int items = heads * (D / 4);
        int teams = 1;
        while (2 * teams * items <= C::THREADS && 2 * teams <= np) teams *= 2;
        const int each = (np + teams - 1) / teams;
        auto fetch = [&](int i, int p0, int end) {
          const int q = i / (D / 4), ch = 4 * (i - q * (D / 4));
#pragma unroll
          for (int p = 0; p < CH; ++p)
            if (p0 + p < end) rows[p] = __ldcg(reinterpret_cast<const float4*>(part_of(p0 + p) + q * D + ch));
        };
        const int team = teams > 1 ? tid / items : 0, item = teams > 1 ? tid - team * items : tid;
        const int p_first = team * each, p_end = min(np, p_first + each);
        if (team < teams && item < items) fetch(item, p_first, p_end);
        for (int i = tid; i < 8 * np; i += C::THREADS) {
          const int p = i >> 3, q = i & 7;
          if (q >= a.rows) continue;
          const float* src = part_of(p) + a.rows * D + q;
          wts[q * np + p] = __ldcg(src);
          wts[8 * np + q * np + p] = __ldcg(src + a.rows);
        }
        join_warps();
        for (int q = warp; q < heads; q += C::NW) {
          float m = kNoMax, l = 0.0f;
          for (int p = lane; p < np; p += 32) m = fmaxf(m, wts[q * np + p]);
#pragma unroll
          for (int x = 16; x; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
          for (int p = lane; p < np; p += 32) {
            const float w = wts[(8 + q) * np + p] * ex2(wts[q * np + p] - m);
            wts[q * np + p] = w;
            l += w;
          }
#pragma unroll
          for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
          if (lane == 0) sums[q] = 1.0f / l;
        }
        join_warps();
        auto sum_of = [&](int i, bool first) {
          const int q = i / (D / 4);
          const float inv = sums[q];  // in every weight, not behind the sum: rows may be near the largest number
          float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int p0 = p_first; p0 < p_end; p0 += CH) {
            if (!first || p0 > p_first) fetch(i, p0, p_end);
#pragma unroll
            for (int p = 0; p < CH; ++p)
              if (p0 + p < p_end) {
                const float w = wts[q * np + p0 + p] * inv;
                x.x += w * rows[p].x;
                x.y += w * rows[p].y;
                x.z += w * rows[p].z;
                x.w += w * rows[p].w;
              }
          }
          return x;
        };
        auto put = [&](int i, const float4& x) {
          const int q = i / (D / 4), ch = 4 * (i - q * (D / 4));
          const long long at = (static_cast<long long>(use.b) * a.H_q + head0 + q) * D + ch;
          store_out2<OT>(a.out, at, x.x, x.y);
          store_out2<OT>(a.out, at + 2, x.z, x.w);
        };
        if (teams == 1) {
          for (int i = tid; i < items; i += C::THREADS) put(i, sum_of(i, i == tid));
        } else {
          float4* const half = reinterpret_cast<float4*>(merge + (2 * 8 * np + 3) / 4 * 4);  // [teams][items], behind the weights
          if (team < teams) half[tid] = sum_of(item, true);
          join_warps();
          if (team == 0) {
            float4 x = half[item];
            for (int t = 1; t < teams; ++t) {
              const float4 y = half[t * items + item];
              x.x += y.x;
              x.y += y.y;
              x.z += y.z;
              x.w += y.w;
            }
            put(item, x);
          }
        }
      }
      join_warps();
    }
  }
}

template <int D, int QT, int OT, bool TEST = false>
cudaError_t launch_dqo(const Args& a, cudaStream_t st) {
  using C = Cfg<D>;
  if constexpr (D == 128 && QT == TQ_FP16 && OT == TQ_FP32 && !TEST) {
    const int limit = test_hooks().spin_limit.load(std::memory_order_relaxed), fault = test_hooks().fault_block.load(std::memory_order_relaxed);
    if (limit > 0 || fault >= 0) {
      Args x = a;
      x.wait_cycles = limit > 0 ? limit : static_cast<int>(kMaxWaitCycles);
      x.fault_block = fault;
      return launch_dqo<D, QT, OT, true>(x, st);
    }
  }
  auto* kernel = decode8_kernel<D, QT, OT, TEST>;
  static std::atomic<uint64_t> ready{0};  // devices on which the shared-memory limit has been raised
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit) || !bit) {
    if (cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM)) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  Args x = a;
  // a thread block's fixed costs are those of some four blocks per warp
  x.min_blocks = 4 * C::NW;
  return launch_kernel(kernel, dim3(static_cast<unsigned>(a.grid)), dim3(C::LAUNCH), C::SMEM, st, x);
}

template <int D>
cudaError_t launch_d(const Args& a, int q_type, int out_type, cudaStream_t st) {
  if (q_type == TQ_BF16) return out_type == TQ_FP32 ? launch_dqo<D, TQ_BF16, TQ_FP32>(a, st) : launch_dqo<D, TQ_BF16, TQ_BF16>(a, st);
  return out_type == TQ_FP32 ? launch_dqo<D, TQ_FP16, TQ_FP32>(a, st) : launch_dqo<D, TQ_FP16, TQ_FP16>(a, st);
}

}  // namespace

// Thread blocks of a launch: one per SM, or as many as the longest sequences could give work to.
int decode8_grid(int B, int H_kv, int G, int d, int max_len) {
  const long long warps = d <= 128 ? Cfg<128>::NW : (d == 256 ? Cfg<256>::NW : Cfg<512>::NW);
  const long long blocks = static_cast<long long>(B) * H_kv * ((G + 7) / 8) * ((max_len + 15LL) / 16 + 1);
  const long long units = static_cast<long long>(B) * H_kv * ((G + 7) / 8);
  const long long worth = std::max(units, (blocks + warps - 1) / warps), most = std::min(device_sm_count(), kMaxGrid);
  return static_cast<int>(std::min(worth, most));
}

// Bytes of the partial results of a call on the current device, whatever its lengths.
size_t decode8_parts_bytes(int B, int H_kv, int G, int d) {
  const long long units = static_cast<long long>(B) * H_kv * ((G + 7) / 8);
  return static_cast<size_t>(part_count(units, std::min(device_sm_count(), kMaxGrid))) * part_floats(d, G < 8 ? G : 8) * sizeof(float);
}

cudaError_t launch_decode8(const tq_kv8_cache& c, const void* q, int q_type, long long q_stride, int H_q, float attn_scale,
                           int window, int grid, uint32_t* counters, float* parts, void* out, int out_type, int32_t* status,
                           cudaStream_t st) {
  Args a = {};
  a.c = c;
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.H_q = H_q;
  a.G = H_q / c.H_kv;
  a.tiles = (a.G + 7) / 8;
  a.window = window;
  a.scale_log2 = attn_scale * kLog2e / 127.0f;
  a.units = c.H_kv * a.tiles;
  a.rows = a.G < 8 ? a.G : 8;
  a.compact = static_cast<long long>(c.B) * a.units < grid;
  // A unit's query, merge and output cost as much as 57 blocks with 8 query heads (d = 128: 7800 cycles, 143 per block),
  // 33 with 2 (d = 64: 3400, 103 per block).
  a.lead = a.compact ? 0 : 25 + 4 * a.rows;
  a.grid = grid;
  a.counters = counters;
  a.parts = parts;
  a.out = out;
  a.status = status;
  switch (c.d) {
    case 64: return launch_d<64>(a, q_type, out_type, st);
    case 128: return launch_d<128>(a, q_type, out_type, st);
    case 256: return launch_d<256>(a, q_type, out_type, st);
    default: return launch_d<512>(a, q_type, out_type, st);
  }
}

}  // namespace tq

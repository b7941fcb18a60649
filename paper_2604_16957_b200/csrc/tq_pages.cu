// Page bookkeeping of a serving step: the pages of finished sequences go back to the pool, new tokens get pages and
// slots.  Everything is computed from device-side lengths, so a step needs no host round trip and can be replayed
// from a CUDA graph.
//
// The free list is a stack free_pages[0 .. count).  With len_b cached and new_b new tokens, pages of P tokens and
//   need_b = ceil((len_b + new_b) / P) - ceil(len_b / P),   N_b = sum of need over the sequences before b,
// the i-th fresh page of sequence b is free_pages[count - 1 - N_b - i]: two prefix sums (tokens and pages) over
// the batch and one table look-up per token, nothing sequential.
//
// These launches are made of latencies (17 bytes per sequence, 8 per page and per slot): one thread block scans the
// batch, 1024 sequences a round, warp shuffles and one exchange through shared memory.  The slots of many tokens
// (8 bytes each) are written by a second launch over the whole GPU; up to kOneLaunchSlots of them the scanning block
// writes them itself, which saves the hand-over.
#include "tq_internal.cuh"

namespace tq {
namespace {

constexpr int kScan = 1024;                    // most threads of the scanning block; a thread per sequence and round
constexpr int kFill = 256;                     // threads of a block of the slot launch
// Most slots that the scanning block writes itself.  Measured (us per call in a chain): 16 slots 3.2 in one launch, 3.7
// in two; 512: 3.3 and 3.7; 1024: 5.9 and 3.9; 8192: 12.2 and 3.9.
constexpr long long kOneLaunchSlots = 512;

struct Sums {
  long long tokens, pages;
};

// Inclusive sums over the block's threads (thread order).  `warp_sums` holds 32 entries; all threads call it.
__device__ __forceinline__ Sums block_inclusive(Sums v, Sums* warp_sums, Sums& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, v.tokens, o), p = __shfl_up_sync(0xffffffffu, v.pages, o);
    if (lane >= o) {
      v.tokens += t;
      v.pages += p;
    }
  }
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  Sums before = {0, 0}, all = {0, 0};
  for (int w = 0; w < warps; ++w) {
    const Sums s = warp_sums[w];
    if (w < warp) {
      before.tokens += s.tokens;
      before.pages += s.pages;
    }
    all.tokens += s.tokens;
    all.pages += s.pages;
  }
  __syncthreads();  // warp_sums may be written again
  total = all;
  v.tokens += before.tokens;
  v.pages += before.pages;
  return v;
}

__device__ __forceinline__ long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// What the slot launch needs of a sequence: its old length (-1: refused) and the pages taken before it.
struct Row {
  int32_t old, pages_before;
};

__device__ __forceinline__ int read_count(const int32_t* free_count, int num_pages, int32_t* status) {
  int count = *free_count;
  if (count < 0 || count > num_pages) {
    if (status && threadIdx.x == 0) atomicOr(status, TQ_STATUS_BAD_PAGE);
    count = count < 0 ? 0 : num_pages;
  }
  return count;
}

// Offsets and rows of a batch of up to kScan sequences, kept in shared memory: the search for a token's sequence would
// otherwise be a chain of trips to L2.
struct Batch {
  int32_t offsets[kScan + 1];
  Row rows[kScan];
};

// Slot of packed token n, and the table entry of a page that token is the first of.
__device__ __forceinline__ long long slot_of(const PageArgs& a, const int32_t* offsets, const Row* rows, int count, long long n,
                                             int32_t* status) {
  if (n >= offsets[a.B]) return -1;  // padding behind the last token
  int lo = 0, hi = a.B;              // the sequence with offsets[lo] <= n < offsets[lo + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= n) lo = mid;
    else hi = mid;
  }
  const Row r = rows[lo];
  if (r.old < 0) return -1;  // refused
  const int pos = r.old + static_cast<int>(n - offsets[lo]);  // below the capacity, which fits 31 bits
  if (a.page_table == nullptr) return static_cast<long long>(lo) * a.page_tokens * a.max_pages + pos;
  const int shift = __ffs(a.page_tokens) - 1;  // a power of two
  const int logical = pos >> shift, within = pos & (a.page_tokens - 1);
  const int first = static_cast<int>((static_cast<unsigned>(r.old) + a.page_tokens - 1) >> shift);
  int page;
  if (logical >= first) {
    page = a.free_pages[count - 1 - r.pages_before - (logical - first)];
    if (within == 0) a.page_table[static_cast<long long>(lo) * a.max_pages + logical] = page;
  } else {
    page = a.page_table[static_cast<long long>(lo) * a.max_pages + logical];
  }
  if (page < 0 || page >= a.num_pages) {
    if (status) atomicOr(status, TQ_STATUS_BAD_PAGE);
    return -1;
  }
  return static_cast<long long>(page) * a.page_tokens + within;
}

__global__ void __launch_bounds__(kScan) assign_scan_kernel(PageArgs a, int32_t* ws, bool fill, int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ Sums warp_sums[kScan / 32];
  __shared__ int granted;
  __shared__ Batch batch;
  Row* rows = reinterpret_cast<Row*>(ws + 2);
  const bool paged = a.page_table != nullptr;
  const int count = paged ? read_count(a.free_count, a.num_pages, status) : 0;
  const long long cap = static_cast<long long>(a.page_tokens) * a.max_pages;
  if (threadIdx.x == 0) {
    granted = 0;
    ws[0] = count;  // the slot launch reads it here: free_count_out may be free_count
  }
  Sums carry = {0, 0};
  for (int base = 0; base < a.B; base += blockDim.x) {
    const int b = base + threadIdx.x;
    long long old = 0, fresh = 0, need = 0;
    bool fits = false;
    int bad = 0;
    if (b < a.B) {
      old = a.seq_lens[b];
      fresh = a.new_lens[b];
      if (fresh < 0 || old < 0 || old > cap) bad |= TQ_STATUS_BAD_LEN;
      if (fresh < 0) fresh = 0;
      fits = bad == 0 && old + fresh <= cap;
      if (paged && fits) need = ceil_div(old + fresh, a.page_tokens) - ceil_div(old, a.page_tokens);
    }
    // A refused sequence still owns its rows of the packed tokens (their slots are -1), but no pages.  Sums of
    // tokens are kept in 64 bits and cut at n_slots on the way out.
    Sums total;
    const Sums upto0 = block_inclusive({fresh, need}, warp_sums, total);
    const Sums upto = {upto0.tokens + carry.tokens, upto0.pages + carry.pages};
    if (b < a.B) {
      bool ok = fits;
      if (!fits && bad == 0) bad |= TQ_STATUS_CACHE_FULL;
      if (upto.tokens > a.n_slots) {
        if (fresh > 0) bad |= TQ_STATUS_BAD_LEN;
        ok = ok && fresh == 0;
      }
      if (ok && need > 0 && upto.pages > count) {
        bad |= TQ_STATUS_POOL_EMPTY;
        ok = false;
      }
      if (bad && status) atomicOr(status, bad);
      const long long end = upto.tokens < a.n_slots ? upto.tokens : a.n_slots;
      a.token_offsets[b + 1] = static_cast<int32_t>(end);
      if (a.B <= kScan) batch.offsets[b + 1] = static_cast<int32_t>(end);
      a.seq_lens_out[b] = static_cast<int32_t>(ok ? old + fresh : old);
      const long long before = upto.pages - need;
      const Row r = {ok ? static_cast<int32_t>(old) : -1, static_cast<int32_t>(before < 0x7fffffff ? before : 0x7fffffff)};
      rows[b] = r;
      if (a.B <= kScan) batch.rows[b] = r;
      if (ok && need > 0) atomicMax(&granted, static_cast<int>(upto.pages));
    }
    carry.tokens += total.tokens;
    carry.pages += total.pages;
  }
  if (threadIdx.x == 0) a.token_offsets[0] = batch.offsets[0] = 0;
  __syncthreads();
  if (threadIdx.x == 0 && paged) *a.free_count_out = count - granted;
  if (!fill) return;
  const int32_t* offsets = a.B <= kScan ? batch.offsets : a.token_offsets;
  const Row* where = a.B <= kScan ? batch.rows : rows;
  for (long long n = threadIdx.x; n < a.n_slots; n += blockDim.x) a.slots[n] = slot_of(a, offsets, where, count, n, status);
}

__global__ void __launch_bounds__(kFill) assign_fill_kernel(PageArgs a, const int32_t* ws, int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ Batch batch;
  const Row* rows = reinterpret_cast<const Row*>(ws + 2);
  const int32_t* offsets = a.token_offsets;
  const int count = ws[0];
  if (a.B <= kScan) {
    for (int b = threadIdx.x; b <= a.B; b += kFill) {
      batch.offsets[b] = a.token_offsets[b];
      if (b < a.B) batch.rows[b] = rows[b];
    }
    __syncthreads();
    offsets = batch.offsets;
    rows = batch.rows;
  }
  const long long step = static_cast<long long>(gridDim.x) * kFill;
  for (long long n = static_cast<long long>(blockIdx.x) * kFill + threadIdx.x; n < a.n_slots; n += step)
    a.slots[n] = slot_of(a, offsets, rows, count, n, status);
}

// Pages of finished sequences, sequences and pages in ascending order, are pushed onto the stack.
__global__ void __launch_bounds__(kScan) release_kernel(PageArgs a, const uint8_t* finished, int32_t* free_pages,
                                                        int32_t* status) {
  pdl_launch_dependents();
  pdl_wait();
  __shared__ Sums warp_sums[kScan / 32];
  __shared__ int s_at[kScan];
  const bool paged = a.page_table != nullptr;
  const int count = paged ? read_count(a.free_count, a.num_pages, status) : 0;
  const long long cap = static_cast<long long>(a.page_tokens) * a.max_pages;
  // More than 1024 sequences: the total is needed before anything is written, so the lengths are read twice.
  long long all = 0;
  for (int round = (a.B > static_cast<int>(blockDim.x) ? 0 : 1); round < 2; ++round) {
    long long carry = 0;
    for (int base = 0; base < a.B; base += blockDim.x) {
      const int b = base + threadIdx.x;
      long long len = 0, pages = 0;
      bool gone = false;
      if (b < a.B) {
        len = a.seq_lens[b];
        gone = finished[b] != 0;
        if (len < 0 || len > cap) {
          if (status) atomicOr(status, TQ_STATUS_BAD_LEN);
          len = len < 0 ? 0 : cap;
        }
        if (gone && paged) pages = ceil_div(len, a.page_tokens);
      }
      Sums total;
      const Sums upto = block_inclusive({0, pages}, warp_sums, total);
      if (round == 1) {
        if (a.B <= static_cast<int>(blockDim.x)) all = total.pages;
        // more pages than the pool has: the table or the stack is not what it should be, and nothing is released
        const bool refuse = count + all > a.num_pages && paged;
        if (refuse && status && threadIdx.x == 0) atomicOr(status, TQ_STATUS_BAD_PAGE);
        if (b < a.B) a.seq_lens_out[b] = static_cast<int32_t>(gone && !refuse ? 0 : len);
        if (paged) {
          s_at[threadIdx.x] = static_cast<int>(count + carry + upto.pages - pages);
          const int leaving = __syncthreads_count(pages > 0);  // sequences whose pages go back
          // A thread per page, whichever sequence it is of (the last one whose pages start at or before it), or, where no
          // warp is left without one, a warp per sequence.  Release and assign together: one sequence of 600 pages 6.0 us,
          // by warps 8.1; 201 sequences of 54 pages 13.9 us, by warps 9.3.  Four loads of a thread are on their way at a
          // time.
          const int here = min(a.B - base, static_cast<int>(blockDim.x)), warps = blockDim.x >> 5;
          const int first = s_at[0], end = refuse ? first : first + static_cast<int>(total.pages);
          auto move = [&](int from, int to, int step, auto source) {  // the stack's entries from, from + step, ... below to
            for (int at = from; at < to; at += 4 * step) {
              int page[4];
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (at + x * step < to) page[x] = *source(at + x * step);
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                if (at + x * step >= to) break;
                if ((page[x] < 0 || page[x] >= a.num_pages) && status) atomicOr(status, TQ_STATUS_BAD_PAGE);
                free_pages[at + x * step] = page[x];
              }
            }
          };
          auto row = [&](int r) { return a.page_table + static_cast<long long>(base + r) * a.max_pages; };
          if (leaving < warps) {
            move(first + threadIdx.x, end, blockDim.x, [&](int e) {
              int r = 0;
              for (int hi = here; hi - r > 1;) {
                const int mid = (r + hi) >> 1;
                if (s_at[mid] <= e) r = mid;
                else hi = mid;
              }
              return row(r) + (e - s_at[r]);
            });
          } else if (!refuse) {
            for (int r = threadIdx.x >> 5; r < here; r += warps) {
              const int at = s_at[r], to = r + 1 < here ? s_at[r + 1] : end;
              move(at + (threadIdx.x & 31), to, 32, [&](int e) { return row(r) + (e - at); });
            }
          }
          __syncthreads();
        }
      }
      carry += total.pages;
    }
    if (round == 0) all = carry;
  }
  if (threadIdx.x == 0 && paged) *a.free_count_out = static_cast<int32_t>(count + all > a.num_pages ? count : count + all);
}

// As many threads as there is work for: a small block starts sooner and its barriers are shorter.
unsigned threads_for(long long work) {
  return static_cast<unsigned>(work >= kScan ? kScan : (work < 128 ? 128 : (work + 31) / 32 * 32));
}

}  // namespace

cudaError_t launch_pages_assign(const PageArgs& a, int32_t* ws, int32_t* status, cudaStream_t st) {
  const bool fill = a.n_slots <= kOneLaunchSlots;
  const long long work = fill && a.n_slots > a.B ? a.n_slots : a.B;
  cudaError_t e = launch_kernel(assign_scan_kernel, dim3(1), dim3(threads_for(work)), 0, st, a, ws, fill, status);
  if (e != cudaSuccess || fill) return e;
  const long long want = (a.n_slots + kFill - 1) / kFill, most = 8LL * device_sm_count();
  return launch_kernel(assign_fill_kernel, dim3(static_cast<unsigned>(want < most ? want : most)), dim3(kFill), 0, st, a,
                       const_cast<const int32_t*>(ws), status);
}

cudaError_t launch_pages_release(const PageArgs& a, const uint8_t* finished, int32_t* free_pages, int32_t* status,
                                 cudaStream_t st) {
  // (a thread per released page, up to kScan at a time)
  return launch_kernel(release_kernel, dim3(1), dim3(threads_for(a.page_table ? 8LL * a.B : a.B)), 0, st, a, finished, free_pages, status);
}

}  // namespace tq

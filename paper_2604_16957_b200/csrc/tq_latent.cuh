// The block of 16 tokens of the latent cache (tq.h: TQ_BLOCK_LATENT_BYTES) and the arguments of the operators on it.
//
// Byte order.  The decode kernel turns codes into the fp16 operands of tcgen05.mma: rows of 64 channels, 128 bytes, in
// which 16-byte piece p of token t lies at p ^ (t % 8).  A 16-byte load brings the codes of two such pieces; with
// channels 8 j .. 8 j + 7 of two neighbouring rows of 64 in it, the eight threads of a token store to eight different
// pieces of a row at a time, without bank conflicts.  (Sixteen neighbouring channels would meet two by two.)
#pragma once
#include "tq_kv8.cuh"

namespace tq {

constexpr int kRope = TQ_LATENT_ROPE;  // channels of the positional key

__host__ __device__ constexpr int latent_block_bytes(int d_c) { return TQ_BLOCK_LATENT_BYTES(d_c); }
__host__ __device__ constexpr int latent_code_offset(int d_c, int t, int c) {
  return d_c * t + 128 * (c >> 7) + 16 * ((c & 63) >> 3) + 8 * ((c & 127) >> 6) + (c & 7);
}
__host__ __device__ constexpr int latent_rope_offset(int d_c, int t) { return 16 * d_c + 2 * kRope * t; }
__host__ __device__ constexpr int latent_scale_offset(int d_c, int t) { return 16 * d_c + 32 * kRope + 8 * t; }

// Block number b of a sequence's 16-token block j (contiguous or paged); a table entry outside the pool is treated as
// page 0 and `ok` is false.
__device__ __forceinline__ long long latent_block(const tq_latent_cache& c, int b, int j, bool& ok) {
  ok = true;
  if (!c.page_table) return static_cast<long long>(b) * (c.S_cap >> 4) + j;
  const int shift = __ffs(c.page_tokens) - 5;  // log2 of the blocks of a page
  int p = c.page_table[static_cast<long long>(b) * c.max_pages + (j >> shift)];
  if (p < 0 || p >= c.num_pages) {
    ok = false;
    p = 0;
  }
  return (static_cast<long long>(p) << shift) + (j & ((1 << shift) - 1));
}
__host__ __device__ inline long long latent_slots(const tq_latent_cache& c) {
  return c.page_table ? static_cast<long long>(c.num_pages) * c.page_tokens : static_cast<long long>(c.B) * c.S_cap;
}

}  // namespace tq

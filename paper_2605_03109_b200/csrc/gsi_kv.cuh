// Keys and values in 4 bits: the pages' layout and what the kernels of a cache take (gsi_kv.cu, gsi_kv_attend.cu).
#pragma once

#include <cuda_fp16.h>

#include "gsi_common.cuh"

namespace gsi {
namespace kv {

constexpr int kTile = 16;          // tokens of a tile
constexpr int kGroup = 64;         // channels that share a pair (s, mid)
constexpr int kCodeBytes = 512;    // codes of a block: 16 tokens x 64 channels, 16 bytes a lane of a warp
constexpr int kBlockBytes = 576;   // ... and 16 pairs
constexpr int kMaxShares = 148 * 16;   // warps of the attention's grid
constexpr int kMaxShared = 1 << 16;    // (x + 1/2) / shared is right to a row for x < shared + kMaxRows
constexpr int kMaxRows = 16;          // rows of the attention that a warp takes at a time
// What a warp leaves of rows that it shares with others, for heads of that many blocks.
constexpr int kPartFloats(int groups) { return (groups <= 2 ? kMaxRows : kMaxRows / 2) * (groups * kGroup + 8); }

// Layout within a block, of token t (0..15) and channel c (0..63).  K is the A operand of m16n8k16 with tokens as
// its rows: lane 4 (t % 8) + c / 16 holds 16 channels of tokens t % 8 and t % 8 + 8.  V is the A operand with
// channels as its rows and tokens as the contraction: the two halves of a 32-bit word are the tokens of a pair,
// so that a mask takes the same channel of both, and lane 4 (c / 8) + t % 8 / 2 holds 8 channels of four tokens.
__host__ __device__ __forceinline__ int k_byte(int t, int c) { return ((t % 8) * 4 + c / 16) * 16 + (t / 8) * 8 + c % 16 / 2; }
__host__ __device__ __forceinline__ int v_byte(int t, int c) {
  return ((c / 8) * 4 + t % 8 / 2) * 16 + (t / 8) * 8 + c % 8 / 4 * 4 + t % 2 * 2 + c % 4 / 2;
}
__host__ __device__ __forceinline__ int pair_byte(int t) { return kCodeBytes + (2 * (t % 8) + t / 8) * 4; }

// n / d for 0 <= n < 2^31: n m / 2^(31 + l) with 2^(l - 1) < d <= 2^l and m = ceil(2^(31 + l) / d), which is less than 2^32
// and off by less than 2^l / 2^31 of a unit of the quotient.
struct Divisor {
  unsigned d, mul, shift;
  static Divisor of(int d) {
    unsigned l = 0;
    while ((1ull << l) < (unsigned long long)d) ++l;
    return {(unsigned)d, (unsigned)(((1ull << (31 + l)) + d - 1) / d), 31 + l};
  }
  __host__ __device__ __forceinline__ int quotient(int n) const { return (int)((unsigned long long)(unsigned)n * mul >> shift); }
};

struct Shape {
  int n_heads, head_dim, groups, page_tokens, page_tiles, n_pages, max_seqs, max_pages, max_tokens;
  Divisor by_page, by_page_tiles;                 // of tokens, of tiles
  long long tile_bytes, head_bytes, page_bytes;   // a tile of a head (K and V), a head of a page, a page
};

// First byte of tile `tile` of a head in a page.
__host__ __device__ __forceinline__ long long tile_at(const Shape& s, int page, int head, int tile) {
  return page * s.page_bytes + head * s.head_bytes + tile * s.tile_bytes;
}

struct Control {          // at the front of the workspace
  int status;
  unsigned plan_ticket;   // blocks of a plan or release that have read its state
};

struct PlanArgs {
  const int* n_new;
  int n_seqs, upto, commit;   // upto: the requests that q_start and kv_len are written for
  int *lens, *n_free;
  const int* free_pages;
  int *table, *q_start, *kv_len, *slots, *positions, *counts;
};
struct ReleaseArgs {
  const unsigned char* done;
  int n_seqs;
  int *lens, *n_free, *free_pages, *table;
};
struct RowsArgs {   // append: from k, v; read: to k, v
  void *k, *v;
  gsi_dtype_t dtype;
  long long k_token, k_head, v_token, v_head;   // strides in elements
  const int* slots;
  int n;
  unsigned char* pages;
};
struct AttendArgs {
  const void* q;
  void* out;
  gsi_dtype_t dtype;
  long long q_token, q_head, out_token, out_head;
  int n_rows, n_q_heads, shared;   // shared: q heads of a head of the cache (up to kMaxShared)
  float per_shared;                // 1 / shared
  bool q_vec;                      // eight channels of q lie on 16 bytes
  float scale;   // of scores in powers of two
  const int *q_start, *kv_len, *table;
  int n_seqs, likely;   // likely: how many of them have rows, for the choice of a form
  const unsigned char* pages;
  bool clear;          // rows behind the last request's become zeros
  float* parts;        // [kMaxShares][2]: what a warp has of a segment begun before its share, and of one that ends behind it
  unsigned* tickets;   // [kMaxShares]
};

cudaError_t launch_plan(const Shape& s, const PlanArgs& a, Control* ctl, cudaStream_t stream);
cudaError_t launch_release(const Shape& s, const ReleaseArgs& a, Control* ctl, cudaStream_t stream);
cudaError_t launch_append(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream);
cudaError_t launch_read(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream);
cudaError_t prepare_attend(const Shape& s);   // once for a handle, on its device
cudaError_t launch_attend(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream);

// Sums over the block of two values per thread: exclusive prefixes (in thread order) and totals.
struct Scan2 {
  long long a, b;
};
__device__ __forceinline__ Scan2 block_scan(Scan2 v, Scan2* total, Scan2* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  Scan2 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, x.a, o), b = __shfl_up_sync(0xffffffffu, x.b, o);
    if (lane >= o) {
      x.a += a;
      x.b += b;
    }
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  Scan2 before{0, 0}, all{0, 0};
  for (int w = 0; w < warps; ++w) {
    if (w < warp) {
      before.a += s_warp[w].a;
      before.b += s_warp[w].b;
    }
    all.a += s_warp[w].a;
    all.b += s_warp[w].b;
  }
  __syncthreads();
  *total = all;
  return {before.a + x.a - v.a, before.b + x.b - v.b};
}

__device__ __forceinline__ float load_as_float(const void* p, gsi_dtype_t t, long long i) {
  if (t == GSI_F32) return static_cast<const float*>(p)[i];
  if (t == GSI_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, gsi_dtype_t t, long long i, float v) {
  if (t == GSI_F32) static_cast<float*>(p)[i] = v;
  else if (t == GSI_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}

}  // namespace kv
}  // namespace gsi

// Attention over keys and values in 4 bits.
//
// What bounds it: the cache's bytes, 1.125 per channel of a token and head, read once.  At the memory's rate that is 46
// channels a cycle and SM, and unpacking, two contractions and the softmax come to about two instructions a channel and
// lane, so the contractions run on mma.sync straight from the bytes as they lie in the cache (a tile's block is a
// warp's A operand, 16 bytes a lane, no shuffles), with rows of q (row r of the operand's eight columns: row of the step
// x q head that shares the head) as the B operand:
//   scores^T [16 tokens][8 rows]    = codes of K [16][64] x q^T,  one block after the other; s and mid - 8 s of a token
//                                     multiply the block's sums and the sum of q over the block
//   out^T    [64 channels][8 rows] += (codes of V - 8)^T [64][16] x (p s)^T, p and s in one operand, as s differs by token;
//                                     the mid part, sum of p mid, is the same for the 64 channels and stays outside
// tcgen05 has nothing to add at eight columns, and its operands would have to be unpacked into shared memory first.
//
// Codes of K enter as f16 subnormals, code 2^-24 (a mask, exact; the channels in the upper half of a byte as 16 code,
// against q / 16).  Those of V enter as code - 8 (mask, one f16 instruction, exact): sums of random signs,
// where sums of codes would cancel against the mid part.  fp32 rows take two columns each, the two f16 terms of q 2^k
// (|q 2^k| < 2^14) and of p s: 22 bits; 16-bit rows take one: q exact, p s in 11 bits.  The tensor cores truncate as
// they add, so fp32 rows hand their sums over to fp32 additions every kFlush tiles.
#include <type_traits>

#include "gsi_kv.cuh"
#include "gsi_umma.cuh"

namespace gsi {
namespace kv {

namespace {

using umma::mbar_arrive;
using umma::mbar_expect_tx;
using umma::mbar_init;
using umma::mbar_wait;
using umma::s32;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kGrid = 296;       // two blocks an SM
constexpr int kFlush = 16;      // tiles between sums in fp32 (T = 2)
constexpr int kSnap = 8;        // tiles: the share of a CTA ends with a segment that ends as near
constexpr int kMostShares = 64; // CTAs that share a segment
constexpr float kLazy = 8.f;    // a running maximum is left where it is while 2^score stays below 2^kLazy above it
constexpr float kOne = 64.f;    // p s <= 2^kLazy kOne s / vs < 2^15

// G: blocks of 64 channels; T: f16 terms of an operand; NT: column tiles of eight
template <int G, int T, int NT>
struct Cfg {
  static constexpr int kDim = G * kGroup;
  static constexpr int kRows = NT * 8 / T;   // rows of a CTA
  static constexpr int kLaneRows = T == 1 ? 2 : 1;   // ... of a lane per column tile
  static constexpr int kTileBytes = G * 2 * kBlockBytes;
  static constexpr int kStages = G == 1 ? 6 : G == 2 ? 4 : 2;
  static constexpr int kAreaStride = kDim + 8;
  static constexpr int kAreaRows = T == 2 ? NT * 4 : 4;   // rows of a warp that are summed at a time
  static constexpr int kRing = kWarps * kStages * kTileBytes;
  static constexpr int kQ = NT * G * 1024;
  static constexpr int kArea = kWarps * kAreaRows * kAreaStride * 4;
  static constexpr int kSums = (G + 1) * kMaxRows * 4;          // sums of q by block, factors of the scores
  static constexpr int kMl = 2 * kWarps * kMaxRows * 4;         // maxima and sums of the warps
  static constexpr int kBars = kWarps * kStages * 8;
  static constexpr int kSmem = kRing + kQ + kArea + kSums + kMl + kBars;
  static constexpr int kPart = kMaxRows * (kDim + 2);           // floats of a part
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_fast(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ float2 unpack_half2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Nibbles 0 and 4 (kOdd: 1 and 5) of a word, minus 8, as f16.
template <bool kOdd>
__device__ __forceinline__ uint32_t centred(uint32_t w) {
  const uint32_t v = (w & (kOdd ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;   // 1024 + code (16 code)
  __half2 h = *reinterpret_cast<const __half2*>(&v);
  if constexpr (kOdd) h = __hfma2(h, __half2half2(__ushort_as_half(0x2C00)), __half2half2(__ushort_as_half(0xD480)));   // / 16 - 72
  else h = __hadd2(h, __half2half2(__ushort_as_half(0xE408)));   // - 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void copy_tile(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(s32(bar))
               : "memory");
}

// What a step has of one sequence.  Units of work: (head, tile of rows, tile of tokens), the last the fastest.
struct Seq {
  int q0, m, len, seen, tiles, n_row_tiles;   // seen: by the row before its first
  __device__ __forceinline__ long long segments(const Shape& s) const { return (long long)n_row_tiles * s.n_heads; }
};
template <int kRows>
__device__ __forceinline__ Seq load_seq(const Shape& s, const AttendArgs& a, int i) {
  Seq q;
  q.q0 = __ldg(a.q_start + i);
  const int end = __ldg(a.q_start + i + 1);
  q.m = q.q0 < 0 ? 0 : max(min(end, a.n_rows) - q.q0, 0);
  q.len = max(__ldg(a.kv_len + i), 0);
  q.seen = q.m ? q.len - (end - q.q0) : 0;
  // (a length outside the table: one tile more than the table has, which is not there)
  const long long room = (long long)s.max_pages * s.page_tiles;
  q.tiles = (int)max(1ll, min(((long long)q.len + kTile - 1) / kTile, room + 1));
  q.n_row_tiles = (int)(((long long)q.m * a.shared + kRows - 1) / kRows);
  return q;
}

template <int G, int T, int NT>
__global__ void __launch_bounds__(kThreads, 2) k_kv_attend(Shape s, AttendArgs a, Control* ctl) {
  using C = Cfg<G, T, NT>;
  constexpr int kLR = C::kLaneRows;
  extern __shared__ __align__(128) unsigned char smem[];
  unsigned char* s_q = smem + C::kRing;
  float* s_area = reinterpret_cast<float*>(s_q + C::kQ);
  float* s_sum = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(s_area) + C::kArea);   // [G][kMaxRows]
  float* s_factor = s_sum + G * kMaxRows;
  float* s_m = s_factor + kMaxRows;                // [kWarps][kMaxRows]
  float* s_l = s_m + kWarps * kMaxRows;
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(s_l + kWarps * kMaxRows);
  __shared__ Scan2 s_warp[kWarps];
  __shared__ long long s_at[2], s_base[2];   // the CTA's first unit and the one behind its last; the first unit of its first sequence
  __shared__ int s_seq, s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, t4 = lane & 3;

  if (lane == 0)
    for (int i = 0; i < C::kStages; ++i) mbar_init(s_bar + warp * C::kStages + i, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");

  // ---- shares: the units of all sequences in order, in even pieces that end with a segment where one ends near
  const int per = (a.n_seqs + kThreads - 1) / kThreads, first = tid * per, last = min(first + per, a.n_seqs);
  Scan2 sum{0, 0}, total;
  for (int i = first; i < last; ++i) {
    const Seq q = load_seq<C::kRows>(s, a, i);
    sum.a += q.segments(s) * q.tiles;
    sum.b += q.segments(s);
  }
  const Scan2 before = block_scan(sum, &total, s_warp);
  if (total.a == 0) return;
  const long long shares = max(1ll, min(min((long long)gridDim.x, max(total.a / kWarps, total.b)), total.b * kMostShares));
  const int b = blockIdx.x;
  if (b >= shares) return;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const long long x = total.a * (b + e) / shares;
    if (x >= total.a) {
      if (tid == 0) s_at[e] = total.a;
    } else if (x >= before.a && x < before.a + sum.a) {
      long long base = before.a;
      int i = first;
      Seq q = load_seq<C::kRows>(s, a, i);
      for (long long n; x >= base + (n = q.segments(s) * q.tiles);) {
        base += n;
        q = load_seq<C::kRows>(s, a, ++i);
      }
      const long long begin = base + (x - base) / q.tiles * q.tiles, from = x - begin, to = begin + q.tiles - x;
      s_at[e] = from < kSnap && from <= to ? begin : to < kSnap ? begin + q.tiles : x;
      if (e == 0) {
        s_base[0] = base;
        s_seq = i;
      }
    }
  }
  __syncthreads();
  const long long u0 = s_at[0], u1 = s_at[1];
  if (u0 >= u1) return;
  int seq = s_seq;
  long long base = s_base[0];
  Seq q = load_seq<C::kRows>(s, a, seq);
  while (u0 >= base + q.segments(s) * q.tiles) {   // (the share begins where the sequence ended)
    base += q.segments(s) * q.tiles;
    q = load_seq<C::kRows>(s, a, ++seq);
  }

  // ---- the warp's tiles: units u0 + warp + 8 j, through a ring of its own; lane j % 32 knows where tile j lies
  const uint32_t ring = s32(smem) + warp * C::kStages * C::kTileBytes;
  uint64_t* bars = s_bar + warp * C::kStages;
  const int mine = u1 - u0 > warp ? (int)((u1 - u0 - warp + kWarps - 1) / kWarps) : 0;   // its tiles
  int look_seq = seq;
  long long look_base = base;
  const unsigned char* where = nullptr;
  unsigned bad[2] = {0u, 0u};
  auto look_up = [&](int batch) {
    const long long u = u0 + warp + (long long)kWarps * (batch * 32 + lane);
    bool wrong = false;
    where = nullptr;
    if (u < u1) {
      Seq x = load_seq<C::kRows>(s, a, look_seq);
      for (long long n; u >= look_base + (n = x.segments(s) * x.tiles);) {
        look_base += n;
        x = load_seq<C::kRows>(s, a, ++look_seq);
      }
      const long long local = u - look_base, segment = local / x.tiles;
      const int tile = (int)(local - segment * x.tiles), head = (int)(segment / x.n_row_tiles);
      if ((long long)tile * kTile < x.len) {
        const int index = tile / s.page_tiles;
        const int page = index < s.max_pages ? __ldg(a.table + (long long)look_seq * s.max_pages + index) : -1;
        wrong = (unsigned)page >= (unsigned)s.n_pages;
        if (!wrong) where = a.pages + tile_at(s, page, head, tile - index * s.page_tiles);
      }
    }
    bad[batch & 1] = __ballot_sync(0xffffffffu, wrong);
  };
  int issued = 0;
  auto issue = [&]() {
    if (issued >= mine) return;
    if ((issued & 31) == 0) look_up(issued >> 5);
    if (lane == (issued & 31)) {
      uint64_t* bar = bars + issued % C::kStages;
      if (where) {
        mbar_expect_tx(bar, C::kTileBytes);
        copy_tile(ring + (issued % C::kStages) * C::kTileBytes, where, C::kTileBytes, bar);
      } else {
        mbar_arrive(bar);
      }
    }
    ++issued;
    __syncwarp();
  };
  for (int i = 0; i < C::kStages; ++i) issue();

  int j = 0;         // the warp's next tile
  bool gave_up = false;    // a copy did not arrive

  // ---- segments of the share
  for (long long u = u0; u < u1;) {
    while (u >= base + q.segments(s) * q.tiles) {
      base += q.segments(s) * q.tiles;
      q = load_seq<C::kRows>(s, a, ++seq);
    }
    const long long segment = (u - base) / q.tiles, begin = base + segment * q.tiles, end = begin + q.tiles, upto = min(end, u1);
    const int head = (int)(segment / q.n_row_tiles), row0 = (int)(segment - (long long)head * q.n_row_tiles) * C::kRows;
    const int n_rows = min(C::kRows, q.m * a.shared - row0);
    // row r of the tile: row i of the step, q head
    auto step_row = [&](int r) { return (row0 + r) / a.shared; };
    auto q_head = [&](int r) { return head * a.shared + (row0 + r) % a.shared; };
    auto sees = [&](int r) { return q.seen + step_row(min(r, n_rows - 1)) + 1; };

    // the rows as B operand: a warp takes a row, a lane 2 G channels
    for (int r = warp; r < C::kRows; r += kWarps) {
      float v[2 * G], top = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) {
        const int c = i * 32 + lane;
        v[i] = r < n_rows && c < s.head_dim
                   ? load_as_float(a.q, a.dtype, (q.q0 + step_row(r)) * a.q_token + q_head(r) * a.q_head + c) : 0.f;
        top = fmaxf(top, fabsf(v[i]));
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      int k = 0;
      if (top > 0.f && top <= 3.402823466e38f) {
        int e;
        frexpf(top, &e);
        k = 14 - e;
      }
      float part[G];
#pragma unroll
      for (int g = 0; g < G; ++g) part[g] = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) {
        const int c = (i & 1) * 32 + lane, g = i >> 1, nib = c & 7;   // channel of the block, of its word
        const float x = scalbnf(v[i], k);
        part[g] += x;
        const float y = (nib & 1) ? x * 0.0625f : x;
        const __half hi = __float2half_rn(y);
        // word (c % 16) / 8 of lane c / 16: its two steps' registers (nib / 2) % 2, b0 or b1 nib % 2, half nib / 4
        const int col = T == 2 ? (r & 3) * 2 : r & 7, nt = T == 2 ? r >> 2 : r >> 3;
        __half* to = reinterpret_cast<__half*>(s_q + ((nt * G + g) * 2 + (c % 16) / 8) * 512 + (col * 4 + c / 16) * 16) + (nib / 2 % 2) * 4 +
                     (nib & 1) * 2 + nib / 4;
        *to = hi;
        if constexpr (T == 2) to[32] = __float2half_rn(y - __half2float(hi));   // the next column: 4 lanes of 16 bytes on
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        part[g] = warp_sum(part[g]);
        if (lane == 0) s_sum[g * kMaxRows + r] = part[g] * 0x1p-24f;
      }
      if (lane == 0) s_factor[r] = (float)fmin(ldexp((double)a.scale * 1.4426950408889634, 24 - k), 0x1p100);
    }
    __syncthreads();

    float O[NT][G][4][4], z[NT][kLR][G], m[NT][kLR], l[NT][kLR], m_flush[NT];
    float vs = 0.f, vinv = 0.f;   // a power of two not below any s of V so far, and kOne / vs
    bool flushed = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) O[n][g][i][e] = 0.f;
#pragma unroll
      for (int r = 0; r < kLR; ++r) {
        m[n][r] = -INFINITY;
        l[n][r] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) z[n][r][g] = 0.f;
      }
      m_flush[n] = -INFINITY;
    }
    auto row_of = [&](int n, int r) { return T == 2 ? n * 4 + t4 : n * 8 + t4 * 2 + r; };
    int vis[NT][kLR];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < kLR; ++r) vis[n][r] = sees(row_of(n, r));
    const int least = sees(0), most = sees(n_rows - 1);

    auto tile_pass = [&](uint32_t at, int tile, bool wrong, auto masked) {
      constexpr bool kMasked = decltype(masked)::value;
      const int pos = tile * kTile + gr;
      float S[NT][kLR][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < kLR; ++r) S[n][r][0] = S[n][r][1] = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4 w = lds128(at + g * kBlockBytes + lane * 16);
        const uint2 pw = lds64(at + g * kBlockBytes + kCodeBytes + gr * 8);
        float acc[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = h ? w.y : w.x, y = h ? w.w : w.z;
          const uint32_t x8 = x >> 8, y8 = y >> 8;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4 bq = lds128(s32(s_q) + ((n * G + g) * 2 + h) * 512 + lane * 16);
            mma_f16(acc[n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, bq.x, bq.y);
            mma_f16(acc[n], x8 & 0x000F000Fu, y8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x00F000F0u, bq.z, bq.w);
          }
        }
        const float2 p0 = unpack_half2(pw.x), p1 = unpack_half2(pw.y);   // (s, mid) of tokens gr and gr + 8
        const float c0 = fmaf(-8.f, p0.x, p0.y), c1 = fmaf(-8.f, p1.x, p1.y);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < kLR; ++r) {
            const float qs = s_sum[g * kMaxRows + row_of(n, r)];
            const float a0 = T == 2 ? acc[n][0] + acc[n][1] : acc[n][r], a1 = T == 2 ? acc[n][2] + acc[n][3] : acc[n][2 + r];
            S[n][r][0] = fmaf(p0.x, a0, fmaf(c0, qs, S[n][r][0]));
            S[n][r][1] = fmaf(p1.x, a1, fmaf(c1, qs, S[n][r][1]));
          }
      }
      // pairs of V, their largest step, and whether a maximum has to move
      const uint32_t v_at = at + G * kBlockBytes;
      uint2 pv[G];
      __half2 top0 = __half2half2(__ushort_as_half(0)), top1 = top0;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        pv[g] = lds64(v_at + g * kBlockBytes + kCodeBytes + gr * 8);
        if constexpr (kMasked) {   // (behind the last token lies anything)
          if (pos >= q.len) pv[g].x = 0u;
          if (pos + 8 >= q.len) pv[g].y = 0u;
        }
        if (wrong) pv[g] = make_uint2(0u, 0u);
        top0 = __hmax2(top0, *reinterpret_cast<const __half2*>(&pv[g].x));
        top1 = __hmax2(top1, *reinterpret_cast<const __half2*>(&pv[g].y));
      }
      const float step = fmaxf(__low2float(top0), __low2float(top1));
      bool move = step > vs;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < kLR; ++r) {
          const float f = s_factor[row_of(n, r)];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            S[n][r][e] *= f;
            if (wrong) S[n][r][e] = NAN;
            if (kMasked && pos + 8 * e >= vis[n][r]) S[n][r][e] = -INFINITY;
            move = move || S[n][r][e] > m[n][r] + kLazy;
          }
        }
      if (__any_sync(0xffffffffu, move)) {
        float largest = step;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
        const float next_vs = fmaxf(vs, __uint_as_float((__float_as_uint(largest) + 0x7FFFFFu) & 0x7F800000u));
        const float v_keep = next_vs > 0.f ? vs / next_vs : 1.f;
        vs = next_vs;
        vinv = vs > 0.f ? kOne / vs : 0.f;
        float keep[NT][kLR];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < kLR; ++r) {
            float x = fmaxf(S[n][r][0], S[n][r][1]);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            const float next = fmaxf(m[n][r], x);
            keep[n][r] = next == m[n][r] ? 1.f : exp2_fast(m[n][r] - next);
            m[n][r] = next;
            l[n][r] *= keep[n][r];
#pragma unroll
            for (int g = 0; g < G; ++g) z[n][r][g] *= keep[n][r];
            keep[n][r] *= v_keep;
          }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) O[n][g][i][e] *= keep[n][kLR == 2 ? e & 1 : 0];
      }
      float p[NT][kLR][2];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < kLR; ++r) {
          const float from = m[n][r] == -INFINITY ? 0.f : m[n][r];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            p[n][r][e] = exp2_fast(S[n][r][e] - from);
            l[n][r] += p[n][r][e];
          }
        }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4 w = lds128(v_at + g * kBlockBytes + lane * 16);
        const float2 p0 = unpack_half2(pv[g].x), p1 = unpack_half2(pv[g].y);
        const float s0 = p0.x * vinv, s1 = p1.x * vinv;
        uint32_t b0[NT], b1[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x[kLR][2];
#pragma unroll
          for (int r = 0; r < kLR; ++r) {
            x[r][0] = p[n][r][0] * s0;
            x[r][1] = p[n][r][1] * s1;
            float z0 = p[n][r][0] * p0.y, z1 = p[n][r][1] * p1.y;
            if constexpr (kMasked) {   // (a token that this row does not see need not be a number)
              if (pos >= vis[n][r]) x[r][0] = z0 = 0.f;
              if (pos + 8 >= vis[n][r]) x[r][1] = z1 = 0.f;
            }
            z[n][r][g] += z0 + z1;
          }
          if constexpr (T == 2) {
            const __half h0 = __float2half_rn(x[0][0]), h1 = __float2half_rn(x[0][1]);
            b0[n] = pack_half2(__half2float(h0), x[0][0] - __half2float(h0));
            b1[n] = pack_half2(__half2float(h1), x[0][1] - __half2float(h1));
          } else {
            b0[n] = pack_half2(x[0][0], x[kLR - 1][0]);
            b1[n] = pack_half2(x[0][1], x[kLR - 1][1]);
          }
          b0[n] = transpose8x8(b0[n]);
          b1[n] = transpose8x8(b1[n]);
        }
        const uint32_t x8 = w.x >> 8, y8 = w.y >> 8, z8 = w.z >> 8, w8 = w.w >> 8;
        const uint32_t A[4][4] = {{centred<false>(w.x), centred<false>(w.y), centred<false>(w.z), centred<false>(w.w)},
                                  {centred<true>(w.x), centred<true>(w.y), centred<true>(w.z), centred<true>(w.w)},
                                  {centred<false>(x8), centred<false>(y8), centred<false>(z8), centred<false>(w8)},
                                  {centred<true>(x8), centred<true>(y8), centred<true>(z8), centred<true>(w8)}};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16(O[n][g][i], A[i][0], A[i][1], A[i][2], A[i][3], b0[n], b1[n]);
      }
    };

    // rows of the area: this warp's, row `r` (of kAreaRows), from channel 8 gr of block g on
    auto area = [&](int w, int r, int g) { return s_area + (w * C::kAreaRows + r) * C::kAreaStride + g * kGroup + gr * 8; };
    // channels 8 gr .. + 7 of block g: the four steps' rows gr, then their rows gr + 8
    auto lane_sums = [&](int n, int g, int r, float (&v)[8]) {
      const float f = vs * (1.f / kOne);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = (T == 2 ? O[n][g][i][0] + O[n][g][i][1] : O[n][g][i][r]) * f;
        v[i + 4] = (T == 2 ? O[n][g][i][2] + O[n][g][i][3] : O[n][g][i][2 + r]) * f;
      }
    };
    auto add_flushed = [&](int n, int g, float keep, float (&v)[8]) {   // (T = 2)
      const float4* from = reinterpret_cast<const float4*>(area(warp, n * 4 + t4, g));
      const float4 x = from[0], y = from[1];
      v[0] = fmaf(x.x, keep, v[0]), v[1] = fmaf(x.y, keep, v[1]), v[2] = fmaf(x.z, keep, v[2]), v[3] = fmaf(x.w, keep, v[3]);
      v[4] = fmaf(y.x, keep, v[4]), v[5] = fmaf(y.y, keep, v[5]), v[6] = fmaf(y.z, keep, v[6]), v[7] = fmaf(y.w, keep, v[7]);
    };
    auto to_area = [&](int r, int g, const float (&v)[8]) {
      float4* to = reinterpret_cast<float4*>(area(warp, r, g));
      to[0] = make_float4(v[0], v[1], v[2], v[3]);
      to[1] = make_float4(v[4], v[5], v[6], v[7]);
    };

    int since = 0;
    for (; j < mine; ++j) {
      const long long at_u = u0 + warp + (long long)kWarps * j;
      if (at_u >= upto) break;
      const int stage = j % C::kStages;
      if (!gave_up && !mbar_wait(bars + stage, (uint32_t)(j / C::kStages) & 1u)) gave_up = true;
      gave_up = __any_sync(0xffffffffu, gave_up);
      const int tile = (int)(at_u - begin);
      if (tile * kTile < most && !gave_up) {
        const bool wrong = bad[(j >> 5) & 1] >> (j & 31) & 1u;
        if (wrong && lane == 0) ctl->status = GSI_ERR_INVALID_ARG;
        const uint32_t at = ring + stage * C::kTileBytes;
        if ((tile + 1) * kTile <= least) tile_pass(at, tile, wrong, std::false_type{});
        else tile_pass(at, tile, wrong, std::true_type{});
        if (T == 2 && ++since == kFlush) {
          since = 0;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const float keep = m_flush[n] == -INFINITY ? 0.f : exp2_fast(m_flush[n] - m[n][0]);
#pragma unroll
            for (int g = 0; g < G; ++g) {
              float v[8];
              lane_sums(n, g, 0, v);
              if (flushed) add_flushed(n, g, keep, v);
              to_area(n * 4 + t4, g, v);
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[n][g][i][e] = 0.f;
            }
            m_flush[n] = m[n][0];
          }
          flushed = true;
        }
      }
      __syncwarp();
      if (!gave_up) issue();
    }

    // ---- the warps' sums, and those of the CTAs that share the segment
    if (gave_up) {
      if (lane == 0) ctl->status = GSI_ERR_TIMEOUT;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < kLR; ++r) l[n][r] = NAN;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < kLR; ++r) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], o);
#pragma unroll
          for (int g = 0; g < G; ++g) z[n][r][g] += __shfl_xor_sync(0xffffffffu, z[n][r][g], o);
        }
        if (gr == 0) {
          s_m[warp * kMaxRows + row_of(n, r)] = m[n][r];
          s_l[warp * kMaxRows + row_of(n, r)] = l[n][r];
        }
      }
    const bool whole = u == begin && upto == end;
    float* part = a.parts + ((long long)b * 2 + (begin >= u0)) * C::kPart;
    constexpr int kPasses = T == 2 ? 1 : NT * 2;
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      // area row i of the pass is row `base_row + i * stride` of the tile
      const int base_row = T == 2 ? 0 : pass / 2 * 8 + (pass & 1);
      constexpr int kStride = T == 2 ? 1 : 2;
      if (base_row >= n_rows) break;
      if constexpr (T == 2) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float keep = m_flush[n] == -INFINITY ? 0.f : exp2_fast(m_flush[n] - m[n][0]);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float v[8];
            lane_sums(n, g, 0, v);
            if (flushed) add_flushed(n, g, keep, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += z[n][0][g];
            if (n * 4 + t4 < n_rows) to_area(n * 4 + t4, g, v);
          }
        }
      } else {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          float v[8];
          lane_sums(pass / 2, g, pass & 1, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += z[pass / 2][pass & 1][g];
          to_area(t4, g, v);
        }
      }
      __syncthreads();
      const int rows = min(C::kAreaRows, (n_rows - base_row + kStride - 1) / kStride);
      for (int i = tid; i < rows * C::kDim; i += kThreads) {
        const int ar = i / C::kDim, c = i - ar * C::kDim, r = base_row + ar * kStride;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w * kMaxRows + r]);
        const float from = top == -INFINITY ? 0.f : top;
        float sum_l = 0.f, v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float mw = s_m[w * kMaxRows + r], lw = s_l[w * kMaxRows + r];
          if (mw == -INFINITY && lw == 0.f) continue;   // (it saw nothing)
          const float f = exp2_fast(mw - from);
          sum_l += lw * f;
          v += s_area[(w * C::kAreaRows + ar) * C::kAreaStride + c] * f;
        }
        if (whole) {
          if (c < s.head_dim)
            store_from_float(a.out, a.dtype, (q.q0 + step_row(r)) * a.out_token + q_head(r) * a.out_head + c, sum_l == 0.f ? 0.f : v / sum_l);
        } else {
          __stcg(part + r * C::kDim + c, v);
          if (c == 0) {
            __stcg(part + kMaxRows * C::kDim + r, top);
            __stcg(part + kMaxRows * (C::kDim + 1) + r, sum_l);
          }
        }
      }
      __syncthreads();
    }
    if (!whole) {
      // the boundaries between shares that lie within the segment: shares first_b .. first_b + n_parts - 1 have a part
      const long long b1 = ((begin + kSnap) * shares + total.a - 1) / total.a, b2 = ((end - kSnap + 1) * shares + total.a - 1) / total.a - 1;
      const int first_b = (int)b1 - 1, n_parts = (int)(b2 - b1) + 2;
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        s_last = atomicAdd(a.tickets + first_b, 1u) == (unsigned)n_parts - 1;
        if (s_last) a.tickets[first_b] = 0u;
      }
      __syncthreads();
      if (s_last) {
        __threadfence();
        for (int i = tid; i < n_rows * C::kDim; i += kThreads) {
          const int r = i / C::kDim, c = i - r * C::kDim;
          float top = -INFINITY, sum_l = 0.f, v = 0.f;
          for (int x0 = 0; x0 < n_parts; x0 += 8) {
            float pm[8], pl[8], px[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              const float* from = a.parts + ((long long)(first_b + min(x0 + x, n_parts - 1)) * 2 + (x0 + x == 0)) * C::kPart;
              pm[x] = __ldcg(from + kMaxRows * C::kDim + r);
              pl[x] = __ldcg(from + kMaxRows * (C::kDim + 1) + r);
              px[x] = __ldcg(from + r * C::kDim + c);
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
              if (x0 + x >= n_parts || (pm[x] == -INFINITY && pl[x] == 0.f)) continue;
              const float next = fmaxf(top, pm[x]), from = next == -INFINITY ? 0.f : next;
              const float keep = exp2_fast(top - from), f = exp2_fast(pm[x] - from);
              top = next;
              sum_l = sum_l * keep + pl[x] * f;
              v = v * keep + px[x] * f;
            }
          }
          if (c < s.head_dim)
            store_from_float(a.out, a.dtype, (q.q0 + step_row(r)) * a.out_token + q_head(r) * a.out_head + c, sum_l == 0.f ? 0.f : v / sum_l);
        }
      }
      __syncthreads();
    }
    u = upto;
  }
  if (gave_up)   // (copies in flight land before the block's memory is another's)
    for (int i = j; i < issued; ++i) mbar_wait(bars + i % C::kStages, (uint32_t)(i / C::kStages) & 1u);
}

template <int G, int T, int NT>
cudaError_t launch(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  using C = Cfg<G, T, NT>;
  static_assert(C::kSmem <= 113 * 1024, "two blocks of an SM");
  static_assert(C::kRows <= kMaxRows && C::kRing % 16 == 0 && C::kArea % 16 == 0 && (C::kSums + C::kMl) % 8 == 0, "layout");
  if (!a.q) return cudaFuncSetAttribute(k_kv_attend<G, T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  k_kv_attend<G, T, NT><<<kGrid, kThreads, C::kSmem, stream>>>(s, a, ctl);
  return cudaGetLastError();
}

}  // namespace

namespace {

cudaError_t launch_of(int groups, bool two, bool wide, const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  switch (groups * 4 + two * 2 + wide) {
    case 4: return launch<1, 1, 1>(s, a, ctl, stream);
    case 5: return launch<1, 1, 2>(s, a, ctl, stream);
    case 6: return launch<1, 2, 1>(s, a, ctl, stream);
    case 7: return launch<1, 2, 2>(s, a, ctl, stream);
    case 8: return launch<2, 1, 1>(s, a, ctl, stream);
    case 9: return launch<2, 1, 2>(s, a, ctl, stream);
    case 10: return launch<2, 2, 1>(s, a, ctl, stream);
    case 11: return launch<2, 2, 2>(s, a, ctl, stream);
    case 12: return launch<3, 1, 1>(s, a, ctl, stream);
    case 14: return launch<3, 2, 1>(s, a, ctl, stream);
    case 16: return launch<4, 1, 1>(s, a, ctl, stream);
    case 18: return launch<4, 2, 1>(s, a, ctl, stream);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace

cudaError_t prepare_attend(const Shape& s) {
  for (int i = 0; i < (s.groups <= 2 ? 4 : 2); ++i) {
    const bool wide = i >= 2;
    const cudaError_t e = launch_of(s.groups, i & 1, wide, s, AttendArgs{}, nullptr, nullptr);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  // Rows of one column tile, or of two where sequences bring more on average and the registers have room for their sums.
  const bool two = a.dtype == GSI_F32;
  const bool wide = s.groups <= 2 && (long long)a.n_rows * a.shared > (two ? 4ll : 8ll) * a.n_seqs;
  return launch_of(s.groups, two, wide, s, a, ctl, stream);
}

}  // namespace kv
}  // namespace gsi

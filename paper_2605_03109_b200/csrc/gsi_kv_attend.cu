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
// where sums of codes would cancel against the mid part.  fp32 rows take two columns each.  Those of q are whole numbers, q 2^k
// = hi + lo / 4096 with |hi|, |lo| <= 2^11 (so q is held to 2^-24 of its row's largest): a block's sums of codes times
// whole numbers stay below 2^21, and the tensor cores, which truncate as they add, add them exactly (with two f16 terms instead the
// scores were three times as far off).  Those of p s are two f16 terms, 22 bits.  The sums of out are handed over to
// fp32 additions every kFlush sets of tiles.  16-bit rows take one column: q exact (to 2^-35 of its row's largest).  p s of fp16 rows
// are two terms, one after the other (with one, outputs of drafts were 2.8e-4 off instead of 2.1e-4); of bf16 rows one term, 11 bits,
// 2^-12 where the output's own rounding takes 2^-9 (128 requests with shared heads: 1.67e-3 off with one, 1.66e-3 with two; 135 us against 146).
//
// Measured: one row of fp32, heads of 128, 240 warp instructions a tile (K and V of 16 tokens), issue slots 60 % and DRAM 94 % busy
// once all warps run: 1.21 GB in 200 us, 6.0 TB/s.  A call has 6 us before its first tiles (lengths, shares, table, q) and
// some 5 us of uneven ends; 604 MB of 64 ragged requests take 117 us, 119-127 in a loop at the card's power limit.
#include <type_traits>

#include "gsi_kv.cuh"
#include "gsi_umma.cuh"

namespace gsi {
namespace kv {

namespace {

using umma::mbar_init;
using umma::mbar_wait;
using umma::s32;

constexpr int kScan = 256;      // threads that look through the sequences
constexpr int kGrid = 148;      // a block an SM (of two, the one that came first ran ahead by an eighth)
constexpr float kLow = 4096.f;  // units of the second term of q in one of the first
constexpr float kLazy = 8.f;    // a running maximum is left where it is while 2^score stays below 2^kLazy above it
// p s enters as f16 terms: times kOne / (the largest p s so far, as a power of two), and anew where one passes kTop.  That is a
// matter of a row and a block of channels: a step that is large in another block, or a token that the row does not see, or hardly,
// takes no bits away.  Terms of 2^-30 of the largest p s are still held; below kLeast none is.
constexpr float kOne = 64.f, kTop = 32768.f, kLeast = 0x1p-100f;
// kOne / v of a power of two v in [kLeast, 2^100], and 1 / v
__device__ __forceinline__ float over_power(float v) { return __uint_as_float((260u << 23) - __float_as_uint(v)); }
__device__ __forceinline__ float inverse_power(float v) { return __uint_as_float((254u << 23) - __float_as_uint(v)); }
constexpr float kNone = -3e38f; // the maximum of no score

// G: blocks of 64 channels; T: f16 terms of an operand; NT: column tiles of eight; L: lane quarters of a tile.
// The columns of a column tile are 2 L for each of 4 / L tiles of tokens, so that lane quarter t has the scores of tile t / L
// (rows t % L, T = 2; 2 (t % L) and the next, T = 1).  Few rows so share the scalar work of a tile's scores, where they would
// leave most columns empty (one row: 188 -> 160 us for the 64 requests above).  A unit of work is one such set of tiles (two, where
// a set is one tile and the registers have room: chunks of prompts 60 -> 54 us) of one head and a tile of rows.
// A kernel for each type: with fp16 and bf16 told apart at run time 64 requests of bf16 rows, 32 heads of 128, took 129 us instead of 115.
template <gsi_dtype_t kType>
constexpr int kColumns = kType == GSI_F32 ? 2 : 1;
template <int G, int T, int L, int NT>
struct Cfg {
  // Twelve warps where sixteen would spill by the hundred bytes within the loop; what is spilled comes back behind the tiles in flight
  // (one request of 32771 tokens, 16 heads of 256: 52 us with sixteen, 49 with twelve; drafts of 5 fp16 rows 46.8 and 40.3; 64 requests, 8 x 2 heads
  // of 128, bf16: 48.5 and 43.3; chunks of fp32 rows, heads of 64: 50.4 and 50.3).  Heads of 128 with sixteen 16-bit rows still spill 192.
  static constexpr int kWarps = G >= 3 || (L == 4 && G * NT >= 2) || (T == 1 && G == 2) ? 12 : 16;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kShares = kGrid * kWarps;
  static constexpr int kDim = G * kGroup;
  static constexpr int kSet = 4 / L, kSets = L == 4 && G * NT <= 2 ? 2 : 1;   // tiles side by side in the columns, and one after the other
  static constexpr int kTiles = kSet * kSets;          // of a unit
  static constexpr int kLaneRows = T == 1 ? 2 : 1;     // rows of a lane per column tile
  static constexpr int kRows = NT * L * kLaneRows;     // rows of a unit
  static constexpr int kHalf = G * kBlockBytes;        // K of a tile, or V
  static constexpr int kStages = (kWarps == 16 ? 9216 : 14336) / (2 * kHalf) / kTiles;   // units under way
  static constexpr int kRing = kStages * kTiles * 2 * kHalf;
  // A tile comes in one copy; where only one unit has room, in two, so that K of the next one comes while V is read.
  static constexpr bool kSplit = kStages == 1;
  static constexpr int kStride = kSplit ? kHalf : 2 * kHalf;      // from tile to tile
  static constexpr int kToV = kSplit ? kTiles * kHalf : kHalf;    // from a tile's K to its V
  static constexpr int kQ = NT * G * 1024;
  static constexpr int kSums = ((3 * G + 1) * kRows * 4 + 15) / 16 * 16;   // per block: -8 times the sums of q's terms, the sum of q; factors
  static constexpr int kBars = kStages * (kSplit ? 2 : 1) * 8;
  static constexpr int kWarpBytes = (kRing + kQ + kSums + kBars + 15) / 16 * 16;
  static constexpr int kSmem = kWarps * kWarpBytes;
  static_assert(kShares <= kMaxShares, "the workspace's parts and tickets");
  static constexpr int kSnap = kTiles == 1 ? 2 : 1;        // units: the share of a warp ends with a segment that ends as near
  static constexpr int kCost = kSets == 2 ? 3 : L + 1;     // units that a segment itself counts as in a share (L: 111 us, L + 1: 109)
  // Sets of tiles between sums in fp32, as the tensor cores truncate: 2^-23 of a sum each.  16-bit rows are rounded to 2^-12 or 2^-9 in
  // the end (with 32 for them too: 128 requests with shared heads 136 -> 139 us).
  static constexpr int kFlush = T == 2 ? 32 : 128;
  static constexpr int kPart = kPartFloats(G);
  static constexpr int kPartRows = kPart / (kDim + 8);
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ float2 lds_float2(uint32_t at) {
  const uint2 v = lds64(at);
  return make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
}
__device__ __forceinline__ float lds_float(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at));
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
  uint32_t v;   // 1024 + code (16 code): (w & mask) | 1024
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w), "r"(kOdd ? 0x00F000F0u : 0x000F000Fu), "r"(0x64006400u));
  __half2 h = *reinterpret_cast<const __half2*>(&v);
  if constexpr (kOdd) h = __hfma2(h, __half2half2(__ushort_as_half(0x2C00)), __half2half2(__ushort_as_half(0xD480)));   // / 16 - 72
  else h = __hadd2(h, __half2half2(__ushort_as_half(0xE408)));   // - 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void copy_tile(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint64_t policy) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar), "l"(policy)
               : "memory");
}
// Tiles that are read once leave the L2 first: what the next call or the next segment needs (this code, tables, q, parts) would
// otherwise come from memory, behind the tiles in flight.
__device__ __forceinline__ uint64_t first_out() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}
__device__ __forceinline__ uint64_t as_usual() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}

// What a step has of one sequence.  Its units: (head, tile of rows, tokens), the last the fastest; those of one head and
// tile of rows are a segment.
struct Seq {
  int q0, m, len, seen, units, n_row_tiles;   // seen: by the row before its first; units: of a segment
  __device__ __forceinline__ long long segments(const Shape& s) const { return (long long)n_row_tiles * s.n_heads; }
  __device__ __forceinline__ long long all(const Shape& s) const { return segments(s) * units; }
};
// a / b of numbers that are not negative and seldom large
__device__ __noinline__ long long large_quotient(long long a, long long b) { return a / b; }
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if ((a | b) >> 32) return large_quotient(a, b);
  return (unsigned)a / (unsigned)b;
}
// Where a share begins: its first unit; the sequence, the first unit of that and the segments before it.
struct Begin {
  long long u, base, segments;
  int seq;
};
template <int kRows, int kTiles>
__device__ __forceinline__ Seq load_seq(const Shape& s, const AttendArgs& a, int i) {
  Seq q;
  q.q0 = a.q_start[i];
  const int end = a.q_start[i + 1];
  q.m = q.q0 < 0 ? 0 : max(min(end, a.n_rows) - q.q0, 0);
  q.len = max(a.kv_len[i], 0);
  q.seen = q.m ? q.len - (end - q.q0) : 0;
  // (a length outside the table: one tile more than the table has, which is not there)
  const long long room = (long long)s.max_pages * s.page_tiles;
  q.units = ((int)max(1ll, min(((long long)q.len + kTile - 1) / kTile, room + 1)) + kTiles - 1) / kTiles;
  q.n_row_tiles = (int)(((long long)q.m * a.shared + kRows - 1) / kRows);
  return q;
}

constexpr int kFew = 8;   // parts that the last warp of a segment sums by itself

// A segment that more warps share, whose last warp is of this block.
struct Pending {
  int first, parts, rows;
  long long out[kMaxRows];
};

template <int G, gsi_dtype_t kType, int L, int NT>
__global__ void __launch_bounds__(Cfg<G, kColumns<kType>, L, NT>::kThreads, 1) k_kv_attend(Shape s, AttendArgs a, Control* ctl) {
  constexpr int T = kColumns<kType>;
  using C = Cfg<G, T, L, NT>;
  constexpr int kTerms = kType == GSI_F16 ? 2 : 1;   // of p s that follow one another, where a row has one column
  constexpr int kLR = C::kLaneRows, N = C::kTiles, kSet = C::kSet, kSets = C::kSets, kWarps = C::kWarps, kThreads = C::kThreads;
  static_assert(C::kRing >= (int)sizeof(Scan2) * kScan, "prefixes lie in the first warp's rings");
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Scan2 s_warp[kWarps];
  Scan2* s_before = reinterpret_cast<Scan2*>(smem);   // units and segments before a thread's sequences (where the rings will be)
  __shared__ Begin s_begin[kWarps * 2];
  __shared__ Pending s_pending[kWarps * 2];
  __shared__ int s_n_pending;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gr = lane >> 2, t4 = lane & 3;
  unsigned char* ring = smem + warp * C::kWarpBytes;
  unsigned char* s_q = ring + C::kRing;
  float* s_start = reinterpret_cast<float*>(s_q + C::kQ);   // [G][kRows][2]
  float* s_sum = s_start + 2 * G * C::kRows;                // [G][kRows]
  float* s_factor = s_sum + G * C::kRows;                   // [kRows]
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_q + C::kQ + C::kSums);   // of the stages (K, then V, where they come apart)
  auto load = [&](int i) { return load_seq<C::kRows, N>(s, a, i); };

  if (lane == 0)
    for (int i = 0; i < C::kBars / 8; ++i) mbar_init(bars + i, N);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  if (tid == 0) s_n_pending = 0;
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait();

  if (a.clear) {
    const long long width = (long long)a.n_q_heads * s.head_dim;
    for (long long row = max(a.q_start[a.n_seqs], 0) + (long long)blockIdx.x; row < a.n_rows; row += gridDim.x)
      for (long long i = tid; i < width; i += kThreads)
        store_from_float(a.out, kType, row * a.out_token + i / s.head_dim * a.out_head + i % s.head_dim, 0.f);
  }

  // ---- shares: the units of all sequences in order, in even pieces that end with a segment where one ends near.  A segment
  // counts as kCost units more: its rows have to be fetched and its sums to be put away.
  Scan2 total;
  long long weight, shares;
  bool full;
  int my_share, stride;
  // Few shares: one a block.  Otherwise a block's are neighbours: long segments are then the work of a few blocks each, and
  // not all of them wait for the slowest one.
  auto share_out = [&]() {
    weight = total.a + C::kCost * total.b;
    shares = max(1ll, min((long long)C::kShares, max(quotient(weight, C::kSnap + C::kCost), total.b)));
    full = shares == C::kShares;
    my_share = full ? blockIdx.x * kWarps : blockIdx.x;
    stride = full ? 1 : kGrid;
  };
  // the first unit of the share that begins at x of a sequence's weight, from the sequence's first on
  auto unit_at = [&](long long x, int units) {
    const long long segment = quotient(x, units + C::kCost);
    const int unit = max((int)(x - segment * (units + C::kCost)) - C::kCost, 0), left = units - unit;
    return segment * units + (unit < C::kSnap && unit <= left ? 0 : left < C::kSnap ? units : unit);
  };
  auto clear_rows = [&]() {   // (while the lengths are on their way)
    for (int i = lane; i < (C::kQ + C::kSums) / 16; i += 32) reinterpret_cast<uint4*>(s_q)[i] = make_uint4(0u, 0u, 0u, 0u);
  };
  long long u0 = 0, u1 = 0, base = 0, segment = 0;   // the warp's units; its first sequence's first unit; the next segment, counted over all sequences
  int seq = 0;
  if (a.n_seqs <= 32) {   // a lane a sequence, no wait between the warps (12 heads of 64, 33 tokens: 7.5 -> 6.8 us; up to
                          // 128 sequences, four a lane: no gain)
    Scan2 mine{0, 0};
    int units = 1;
    if (lane < a.n_seqs) {
      const Seq x = load(lane);
      mine = {x.all(s), x.segments(s)};
      units = x.units;
    }
    clear_rows();
    Scan2 upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long na = __shfl_up_sync(0xffffffffu, upto.a, o), nb = __shfl_up_sync(0xffffffffu, upto.b, o);
      if (lane >= o) upto = {upto.a + na, upto.b + nb};
    }
    total = {__shfl_sync(0xffffffffu, upto.a, 31), __shfl_sync(0xffffffffu, upto.b, 31)};
    if (total.a == 0) return;
    share_out();
    if (my_share >= shares) return;
    const Scan2 before{upto.a - mine.a, upto.b - mine.b};
    const long long from = before.a + C::kCost * before.b;
#pragma unroll
    for (int e = 1; e >= 0; --e) {
      const long long x = quotient(weight * min((long long)my_share + warp * stride + e, shares), shares);
      // the last sequence that begins there or before (of those without units, which begin where the next one does, none is the last)
      const int at = 31 - __clz(__ballot_sync(0xffffffffu, lane < a.n_seqs && from <= x));
      base = __shfl_sync(0xffffffffu, before.a, at);
      segment = __shfl_sync(0xffffffffu, before.b, at);
      const long long u = x >= weight ? total.a : base + unit_at(x - base - C::kCost * segment, __shfl_sync(0xffffffffu, units, at));
      (e ? u1 : u0) = u;
      seq = at;
    }
  } else {
    const int per = (a.n_seqs + kScan - 1) / kScan;
    Scan2 sum{0, 0};
    for (int i = tid * per; tid < kScan && i < min(tid * per + per, a.n_seqs); ++i) {
      const Seq x = load(i);
      sum.a += x.all(s);
      sum.b += x.segments(s);
    }
    clear_rows();
    const Scan2 before = block_scan(sum, &total, s_warp);
    if (tid < kScan) s_before[tid] = before;
    if (total.a == 0) return;
    share_out();
    if (my_share >= shares) return;
    __syncthreads();
    if (tid < kWarps * 2) {   // the shares of the block's warps, and those behind them
      const long long x = quotient(weight * (my_share + (tid >> 1) * stride + (tid & 1)), shares);
      Begin at{total.a, 0, 0, 0};
      if (x < weight) {
        int lo = 0, hi = kScan;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (s_before[mid].a + C::kCost * s_before[mid].b <= x) lo = mid;
          else hi = mid;
        }
        at = {0, s_before[lo].a, s_before[lo].b, lo * per};
        Seq q = load(at.seq);
        for (;;) {
          const long long n = q.segments(s);
          if (x < at.base + C::kCost * at.segments + n * (q.units + C::kCost)) break;
          at.base += n * q.units;
          at.segments += n;
          q = load(++at.seq);
        }
        at.u = at.base + unit_at(x - at.base - C::kCost * at.segments, q.units);
      }
      s_begin[tid] = at;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    const Begin& at = s_begin[warp * 2];
    u0 = at.u, u1 = s_begin[warp * 2 + 1].u, base = at.base, segment = at.segments, seq = at.seq;
  }
  const int share = my_share + warp * stride;

  if (share < shares) {
    __syncwarp();   // (what clear_rows wrote lies under other lanes' rows of q; votes and shuffles order no memory)
    const int mine = (int)(u1 - u0);   // the warp's units
    Seq q;
    int head = 0, row_tile = 0, unit = 0;   // of the next unit
    if (mine > 0) {
      q = load(seq);
      while (u0 >= base + q.all(s)) {   // (the share begins where the sequence ended)
        base += q.all(s);
        segment += q.segments(s);
        q = load(++seq);
      }
      const int first = (int)quotient(u0 - base, q.units);
      segment += first;
      unit = (int)(u0 - base - (long long)first * q.units);
      head = (int)((unsigned)first / (unsigned)q.n_row_tiles);
      row_tile = first - head * q.n_row_tiles;
    }

    // Rows of q: a lane takes eight channels, a word of K's codes, kRowLanes lanes a row.  The first ones are asked for ahead of the
    // tiles, which would hold them up; rows of later segments are prefetched.
    constexpr int kRowLanes = G == 1 ? 8 : G == 2 ? 16 : 32, kRowsAtOnce = 32 / kRowLanes;
    const int my_word = lane % kRowLanes, my_row = lane / kRowLanes;
    uint32_t q_raw[T == 2 ? 8 : 4];   // as they lie there
    auto fetch = [&](long long from, bool there) {
#pragma unroll
      for (int i = 0; i < (T == 2 ? 8 : 4); ++i) q_raw[i] = 0u;
      const int n = there ? s.head_dim - my_word * 8 : 0;
      from += my_word * 8;
      if (n >= 8 && a.q_vec) {
        const uint4* at = reinterpret_cast<const uint4*>(static_cast<const char*>(a.q) + from * (T == 2 ? 4 : 2));
        const uint4 v = at[0];
        q_raw[0] = v.x, q_raw[1] = v.y, q_raw[2] = v.z, q_raw[3] = v.w;
        if constexpr (T == 2) {
          const uint4 y = at[1];
          q_raw[4] = y.x, q_raw[5] = y.y, q_raw[6] = y.z, q_raw[7] = y.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) {
            if constexpr (T == 2) q_raw[i] = static_cast<const uint32_t*>(a.q)[from + i];
            else q_raw[i / 2] |= (uint32_t)static_cast<const uint16_t*>(a.q)[from + i] << 16 * (i & 1);
          }
      }
    };
    auto channel = [&](int i) {
      if (T == 2) return __uint_as_float(q_raw[i]);
      const uint32_t w = q_raw[i / 2 % (T == 2 ? 8 : 4)];
      if (kType == GSI_BF16) return __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
      return __half2float(__ushort_as_half((unsigned short)(w >> 16 * (i & 1))));
    };
    // row r of a tile of rows, from the step's row `step0` and the q head `in0` of those that share the head on
    auto step_of = [&](int in0, int r) { return __float2int_rd((in0 + r + 0.5f) * a.per_shared); };
    auto q_from = [&](const Seq& x, int of_head, int step0, int in0, int r) {
      const int i = step_of(in0, r);
      return (long long)(x.q0 + step0 + i) * a.q_token + (long long)(of_head * a.shared + in0 + r - i * a.shared) * a.q_head;
    };
    auto prefetch = [&](const Seq& x, int of_head, int of_tile) {
      const int row0 = of_tile * C::kRows, n = min(C::kRows, x.m * a.shared - row0), step0 = row0 / a.shared;
      constexpr int kLines = G * 2 / T;   // of 128 bytes, a row
      for (int i = lane; i < n * kLines; i += 32) {
        const char* at = static_cast<const char*>(a.q) + q_from(x, of_head, step0, row0 - step0 * a.shared, i / kLines) * (T == 2 ? 4 : 2) + i % kLines * 128;
        if (i % kLines * (T == 2 ? 32 : 64) < s.head_dim) asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
      }
    };
    if (mine > 0) {
      if (C::kRows > kRowsAtOnce) prefetch(q, head, row_tile);
      const int row0 = row_tile * C::kRows, step0 = row0 / a.shared;
      fetch(q_from(q, head, step0, row0 - step0 * a.shared, my_row), my_row < min(C::kRows, q.m * a.shared - row0));
    }

    // ---- its tiles come through a ring; lane (N j + i) % 32 knows where tile i of unit j lies
    int look_seq = seq;
    long long look_base = base;
    const unsigned char* where = nullptr;
    unsigned bad_even = 0u, bad_odd = 0u;   // tiles without a page, of batches of 32
    auto look_up = [&](int batch) {
      const long long u = u0 + batch * (32 / N) + lane / N;
      bool wrong = false;
      where = nullptr;
      if (u < u1) {
        Seq x = load(look_seq);
        for (long long n; u >= look_base + (n = x.all(s));) {
          look_base += n;
          x = load(++look_seq);
        }
        const long long local = u - look_base, segment = quotient(local, x.units);
        const int at = (int)(local - segment * x.units) * N + lane % N, of = (int)quotient(segment, x.n_row_tiles);
        if ((long long)at * kTile < x.len) {
          const int index = s.by_page_tiles.quotient(at);
          const int page = index < s.max_pages ? a.table[(long long)look_seq * s.max_pages + index] : -1;
          wrong = (unsigned)page >= (unsigned)s.n_pages;
          if (!wrong) where = a.pages + tile_at(s, page, of, at - index * s.page_tiles);
        }
      }
      const unsigned mask = __ballot_sync(0xffffffffu, wrong);
      if (batch & 1) bad_odd = mask;
      else bad_even = mask;
    };
    int stage = 0;
    uint32_t phase = 0;
    bool gave_up = false;    // a copy did not arrive

    // what of the columns' operands is of tile i: the columns of the others are zero
    uint32_t only[kSet];
    uint32_t q_at[kSet];
#pragma unroll
    for (int i = 0; i < kSet; ++i) {
      const bool of = gr / (2 * L) == i;
      only[i] = of ? ~0u : 0u;
      q_at[i] = s32(s_q) + ((kSet == 1 || of ? gr % (2 * L) : 2 * L) * 4 + t4) * 16;
    }
    const int my_tile = t4 / L;   // the one of a set whose scores this lane has
    const uint32_t ring_at = s32(ring), start_at = s32(s_start), sum_at = s32(s_sum);
    const uint32_t my_pair = my_tile * C::kStride + kCodeBytes + gr * 8, my_codes = lane * 16;
    const uint32_t my_slot = ring_at + lane % N * C::kStride, my_bar = s32(bars);   // where its copies go, and their barriers
    const uint64_t policy = L == 4 ? as_usual() : first_out();   // (many rows: other units read the same tiles)
    auto row_of = [&](int n, int r) { return T == 2 ? n * L + t4 % L : n * 2 * L + t4 % L * 2 + r; };

    // unit j, if there is one, to its stage (its K or its V, where they come apart)
    auto issue = [&](int j, int stage, bool of_v) {
      if (j < mine && lane / N == j % (32 / N)) {
        const uint32_t bar = my_bar + (stage + of_v) * 8;
        if (where) {
          asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(C::kStride) : "memory");
          copy_tile(my_slot + (C::kSplit ? of_v * C::kToV : stage * N * C::kStride), where + of_v * C::kHalf, C::kStride, bar, policy);
        } else {
          asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
        }
      }
    };
    if (mine > 0) look_up(0);
#pragma unroll 1
    for (int i = 0; i < C::kBars / 8; ++i) issue(C::kSplit ? 0 : i, C::kSplit ? 0 : i, C::kSplit && i);

    // ---- segments of the share
    for (int j = 0; j < mine && !gave_up;) {
      const int n_units = min(q.units - unit, mine - j), begun = j, end = j + n_units;   // of this segment
      const int row0 = row_tile * C::kRows, n_rows = min(C::kRows, q.m * a.shared - row0);
      // row r of the tile: row of the step, q head; its tokens
      const int step0 = row0 / a.shared, in0 = row0 - step0 * a.shared;
      auto step_row = [&](int r) { return step0 + step_of(in0, r); };
      auto q_head = [&](int r) { return head * a.shared + row0 + r - step_row(r) * a.shared; };
      auto sees = [&](int r) { return q.seen + step_row(min(r, n_rows - 1)) + 1; };

      // the rows as B operand.  (Columns of rows that are not there hold what they held.)
      for (int r0 = 0; r0 < n_rows; r0 += kRowsAtOnce) {
        const int r = r0 + my_row;
        if (j && r0 == 0) fetch(q_from(q, head, step0, in0, r), r < n_rows);
        float v[8], top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = channel(i);
          top = fmaxf(top, fabsf(v[i]));
        }
        if (r0 + kRowsAtOnce < n_rows) fetch(q_from(q, head, step0, in0, r + kRowsAtOnce), r + kRowsAtOnce < n_rows);
#pragma unroll
        for (int o = kRowLanes / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        // 2^k takes the largest to below 2^11 (2^14), as a product of two; a row of zeros, or with an infinity, stays as it is
        int k = (T == 2 ? 137 : 140) - (int)(__float_as_uint(top) >> 23);
        if (top == 0.f || top > 3.402823466e38f) k = 0;
        const float k0 = __uint_as_float((uint32_t)(127 + k / 2) << 23), k1 = __uint_as_float((uint32_t)(127 + k - k / 2) << 23);
        float lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = v[i] * k0 * k1, odd = (i & 1) ? 0.0625f : 1.f;   // (codes of odd channels enter as 16 code)
          v[i] = T == 2 ? rintf(x) : x;
          lo[i] = T == 2 ? rintf((x - v[i]) * kLow) * odd : 0.f;
          v[i] *= odd;
        }
        if (r < n_rows && my_word < 8 * G) {
          // channels i and i + 4 of word h of lane t: of its two steps, registers b0 and b1
          const int col = T == 2 ? r % L * 2 : r % (2 * L), nt = T == 2 ? r / L : r / (2 * L);
          uint4* to = reinterpret_cast<uint4*>(s_q + ((nt * G + my_word / 8) * 2 + my_word % 2) * 512 + (col * 4 + my_word % 8 / 2) * 16);
          to[0] = make_uint4(pack_half2(v[0], v[4]), pack_half2(v[1], v[5]), pack_half2(v[2], v[6]), pack_half2(v[3], v[7]));
          if constexpr (T == 2)   // the next column
            to[4] = make_uint4(pack_half2(lo[0], lo[4]), pack_half2(lo[1], lo[5]), pack_half2(lo[2], lo[6]), pack_half2(lo[3], lo[7]));
          // (powers of two: 2^(24 - k) in two steps)
          const float back0 = __uint_as_float((uint32_t)(127 - k / 2) << 23), back1 = __uint_as_float((uint32_t)(151 - k + k / 2) << 23);
          if (my_word == 0) s_factor[r] = fminf(fmaxf(a.scale * back0 * back1, -0x1p100f), 0x1p100f);
        }
      }
      __syncwarp();
      // Per block, what the scores' sums begin with, -8 times the sum of the column's q (the sums are then those of
      // code - 8), as the sums for codes that are all -8; and the sum of the row's q.
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 bq = lds128(s32(s_q) + ((n * G + g) * 2 + h) * 512 + (gr % (2 * L) * 4 + t4) * 16);
            mma_f16(acc, 0x80088008u, 0x80088008u, 0x80808080u, 0x80808080u, bq.x, bq.y);
            mma_f16(acc, 0x80088008u, 0x80088008u, 0x80808080u, 0x80808080u, bq.z, bq.w);
          }
          if (gr == 0 && t4 < L) {
            if constexpr (T == 2) {
              const int r = g * C::kRows + row_of(n, 0);
              s_start[2 * r] = acc[0];
              s_start[2 * r + 1] = acc[1];
              s_sum[r] = fmaf(acc[1], 1.f / kLow, acc[0]) * -0.125f;
            } else {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                s_start[2 * (g * C::kRows + row_of(n, e))] = acc[e];
                s_sum[g * C::kRows + row_of(n, e)] = acc[e] * -0.125f;
              }
            }
          }
        }
      __syncwarp();
      if (j + n_units < mine) {   // the rows of the segment behind
        Seq x = q;
        int x_seq = seq, x_head = head, x_tile = row_tile + 1;
        if (x_tile == x.n_row_tiles) {
          x_tile = 0;
          if (++x_head == s.n_heads) {
            x_head = 0;
            do x = load(++x_seq);
            while (x.n_row_tiles == 0);
          }
        }
        prefetch(x, x_head, x_tile);
      }

      // sums and maxima, of each tile of a unit its own until the segment ends
      float O[NT][G][4][4], z[NT][kLR][G], m[NT][kLR], l[NT][kLR], factor[NT][kLR];
      float unit_of[NT][kLR][G];   // of p s in O: kOne / (a power of two not below any p s so far); 0 before the first
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
          m[n][r] = kNone;
          l[n][r] = 0.f;
          factor[n][r] = s_factor[row_of(n, r)];
#pragma unroll
          for (int g = 0; g < G; ++g) z[n][r][g] = unit_of[n][r][g] = 0.f;
        }
      }
      const int least = sees(0), most = sees(n_rows - 1);

      // A unit from token `first_pos` on; masked: where some row does not see all of it, or a page is missing (a bit for each tile)
      auto pass = [&](auto is_masked, int first_pos, unsigned missing, int next) {
        constexpr bool kMasked = decltype(is_masked)::value;
        const int pos = first_pos + my_tile * kTile + gr;   // of the first set
        bool wrong[kSets];
        float S[kSets][NT][kLR][2], p[kSets][NT][kLR][2];
        const uint32_t k_at = ring_at + stage * N * C::kStride, v_at = k_at + C::kToV;
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
          wrong[u] = kMasked && (missing >> (u * kSet + my_tile) & 1u);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const uint2 pw = lds64(k_at + my_pair + (u * kSet * C::kStride + g * kBlockBytes));
            float acc[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              // -8 times the sum of the column's q: the sums are those of code - 8
              if constexpr (T == 2) {
                const float2 v = lds_float2(start_at + (g * C::kRows + row_of(n, 0)) * 8);
                acc[n][0] = acc[n][2] = v.x;
                acc[n][1] = acc[n][3] = v.y;
              } else {
                acc[n][0] = acc[n][2] = lds_float(start_at + (g * C::kRows + row_of(n, 0)) * 8);
                acc[n][1] = acc[n][3] = lds_float(start_at + (g * C::kRows + row_of(n, 1)) * 8);
              }
            }
#pragma unroll
            for (int i = 0; i < kSet; ++i) {
              const uint4 w = lds128(k_at + my_codes + ((u * kSet + i) * C::kStride + g * kBlockBytes));
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t x = h ? w.y : w.x, y = h ? w.w : w.z;
                const uint32_t x8 = x >> 8, y8 = y >> 8;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  const uint4 bq = lds128(q_at[i] + ((n * G + g) * 2 + h) * 512);
                  mma_f16(acc[n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, bq.x, bq.y);
                  mma_f16(acc[n], x8 & 0x000F000Fu, y8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x00F000F0u, bq.z, bq.w);
                }
              }
            }
            const float2 p0 = unpack_half2(pw.x), p1 = unpack_half2(pw.y);   // (s, mid) of tokens gr and gr + 8
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int r = 0; r < kLR; ++r) {
                const float qs = lds_float(sum_at + (g * C::kRows + row_of(n, r)) * 4);
                const float a0 = T == 2 ? fmaf(acc[n][1], 1.f / kLow, acc[n][0]) : acc[n][r];
                const float a1 = T == 2 ? fmaf(acc[n][3], 1.f / kLow, acc[n][2]) : acc[n][2 + r];
                S[u][n][r][0] = fmaf(p0.x, a0, g ? fmaf(p0.y, qs, S[u][n][r][0]) : p0.y * qs);
                S[u][n][r][1] = fmaf(p1.x, a1, g ? fmaf(p1.y, qs, S[u][n][r][1]) : p1.y * qs);
              }
          }
        }
        if constexpr (C::kSplit) {
          __syncwarp();
          issue(next, 0, false);
          if (__any_sync(0xffffffffu, !mbar_wait(bars + 1, phase))) {
            gave_up = true;
            return;
          }
        }
        uint2 pv[kSets][G];   // pairs of V
#pragma unroll
        for (int u = 0; u < kSets; ++u)
#pragma unroll
          for (int g = 0; g < G; ++g) pv[u][g] = lds64(v_at + my_pair + (u * kSet * C::kStride + g * kBlockBytes));
        // p s of token e; 0 for one that the row does not see (behind the last token lies anything)
        auto weight_of = [&](int u, int n, int r, int g, int e) {
          if (kMasked && sees(row_of(n, r)) - pos - u * kSet * kTile <= 8 * e) return 0.f;
          return p[u][n][r][e] * __low2float(*reinterpret_cast<const __half2*>(e ? &pv[u][g].y : &pv[u][g].x));
        };
        float top = 0.f;   // the largest p s, as it enters
        bool move = false;
#pragma unroll
        for (int u = 0; u < kSets; ++u)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < kLR; ++r) {
              if constexpr (kMasked) {   // (scaled here: a factor of 0, or below, would make something else of infinity)
                const int vis = sees(row_of(n, r)) - pos - u * kSet * kTile;
                S[u][n][r][0] = vis <= 0 ? -INFINITY : wrong[u] ? NAN : S[u][n][r][0] * factor[n][r];
                S[u][n][r][1] = vis <= 8 ? -INFINITY : wrong[u] ? NAN : S[u][n][r][1] * factor[n][r];
              }
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                p[u][n][r][e] = fmaf(S[u][n][r][e], kMasked ? 1.f : factor[n][r], -m[n][r]);
                move = move || p[u][n][r][e] > kLazy;
                p[u][n][r][e] = exp2_fast(p[u][n][r][e]);
              }
#pragma unroll
              for (int g = 0; g < G; ++g)
                top = fmaxf(top, fmaxf(weight_of(u, n, r, g, 0), weight_of(u, n, r, g, 1)) * unit_of[n][r][g]);
            }
        if (__any_sync(0xffffffffu, move || top > kTop)) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < kLR; ++r) {
              const float f = kMasked ? 1.f : factor[n][r];
              float now = m[n][r];
#pragma unroll
              for (int u = 0; u < kSets; ++u) now = fmaxf(now, fmaxf(S[u][n][r][0] * f, S[u][n][r][1] * f));
#pragma unroll
              for (int o = 4; o < 32; o <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
              const bool moved = now - m[n][r] > kLazy;
              if (!moved) now = m[n][r];   // (another row's: this one's sums stay as they are)
              const float keep = exp2_fast(m[n][r] - now);
              m[n][r] = now;
              l[n][r] *= keep;
#pragma unroll
              for (int u = 0; u < kSets; ++u)
#pragma unroll
                for (int e = 0; e < 2; ++e) p[u][n][r][e] = exp2_fast(fmaf(S[u][n][r][e], f, -now));
#pragma unroll
              for (int g = 0; g < G; ++g) {
                z[n][r][g] *= keep;
                float largest = 0.f;
#pragma unroll
                for (int u = 0; u < kSets; ++u)
#pragma unroll
                  for (int e = 0; e < 2; ++e) largest = fmaxf(largest, weight_of(u, n, r, g, e));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
                float all = keep;   // what O is multiplied by
                if (moved || largest * unit_of[n][r][g] > kTop) {
                  const float was = unit_of[n][r][g] > 0.f ? over_power(unit_of[n][r][g]) : 0.f;
                  const float next = __uint_as_float((__float_as_uint(fmaxf(fmaxf(was * keep, largest), kLeast)) + 0x7FFFFFu) & 0x7F800000u);
                  all *= was * inverse_power(next);
                  unit_of[n][r][g] = over_power(next);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (kLR == 1 || (e & 1) == r) O[n][g][i][e] *= all;
              }
            }
        }
#pragma unroll
        for (int u = 0; u < kSets; ++u) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < kLR; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) l[n][r] += p[u][n][r][e];
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float mid0 = unpack_half2(pv[u][g].x).y, mid1 = unpack_half2(pv[u][g].y).y;
            uint32_t b0[NT][kTerms], b1[NT][kTerms];   // of tokens gr, of tokens gr + 8
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              float x[kLR][2];   // p s as it enters
#pragma unroll
              for (int r = 0; r < kLR; ++r) {
                x[r][0] = weight_of(u, n, r, g, 0) * unit_of[n][r][g];
                x[r][1] = weight_of(u, n, r, g, 1) * unit_of[n][r][g];
                if constexpr (kMasked) {   // (a token that this row does not see need not be a number)
                  const int vis = sees(row_of(n, r)) - pos - u * kSet * kTile;
                  if (vis > 0) z[n][r][g] = fmaf(p[u][n][r][0], mid0, z[n][r][g]);
                  if (vis > 8) z[n][r][g] = fmaf(p[u][n][r][1], mid1, z[n][r][g]);
                } else {
                  z[n][r][g] = fmaf(p[u][n][r][1], mid1, fmaf(p[u][n][r][0], mid0, z[n][r][g]));
                }
              }
              if constexpr (T == 2) {   // its upper eleven bits and the rest, side by side in the row's two columns
                const float x0 = x[0][0], x1 = x[0][1];
                const float h0 = __uint_as_float(__float_as_uint(x0) & 0xFFFFE000u), h1 = __uint_as_float(__float_as_uint(x1) & 0xFFFFE000u);
                b0[n][0] = pack_half2(h0, x0 - h0);
                b1[n][0] = pack_half2(h1, x1 - h1);
              } else {
                auto term = [&](int e, uint32_t& first, uint32_t& second) {   // to nearest, and what is left
                  first = pack_half2(x[0][e], x[kLR - 1][e]);
                  const float2 high = unpack_half2(first);
                  if (kTerms == 2) second = pack_half2(x[0][e] - high.x, x[kLR - 1][e] - high.y);
                };
                term(0, b0[n][0], b0[n][kTerms - 1]);
                term(1, b1[n][0], b1[n][kTerms - 1]);
              }
#pragma unroll
              for (int y = 0; y < kTerms; ++y) {
                b0[n][y] = transpose8x8(b0[n][y]);
                b1[n][y] = transpose8x8(b1[n][y]);
              }
            }
#pragma unroll
            for (int i = 0; i < kSet; ++i) {
              const uint4 w = lds128(v_at + my_codes + ((u * kSet + i) * C::kStride + g * kBlockBytes));
              const uint32_t x8 = w.x >> 8, y8 = w.y >> 8, z8 = w.z >> 8, w8 = w.w >> 8;
              const uint32_t A[4][4] = {{centred<false>(w.x), centred<false>(w.y), centred<false>(w.z), centred<false>(w.w)},
                                        {centred<true>(w.x), centred<true>(w.y), centred<true>(w.z), centred<true>(w.w)},
                                        {centred<false>(x8), centred<false>(y8), centred<false>(z8), centred<false>(w8)},
                                        {centred<true>(x8), centred<true>(y8), centred<true>(z8), centred<true>(w8)}};
#pragma unroll
              for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int y = 0; y < kTerms; ++y) {
                  const uint32_t c0 = kSet == 1 ? b0[n][y] : b0[n][y] & only[i], c1 = kSet == 1 ? b1[n][y] : b1[n][y] & only[i];
#pragma unroll
                  for (int k = 0; k < 4; ++k) mma_f16(O[n][g][k], A[k][0], A[k][1], A[k][2], A[k][3], c0, c1);
                }
              }
            }
          }
        }
      };

      // the warp's part of a segment that it shares (or that it has to sum in pieces): channels 8 gr .. + 7 of a block
      const bool tail = unit == 0;
      float* part = a.parts + (2ll * share + tail) * C::kPart;
      auto flush_row = [&](int n, int r) { return (n * 4 + t4) * kLR + r; };   // (the one that the row's sums go to in the end, where the lane has it)
      auto maximum_at = [&](int n, int r) { return part + C::kPartRows * (C::kDim + 2) + flush_row(n, r); };   // that they were flushed at
      auto lane_sums = [&](int n, int g, int r, float (&v)[8]) {
        const float f = unit_of[n][r][g] > 0.f ? inverse_power(unit_of[n][r][g]) : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = (T == 2 ? O[n][g][i][0] + O[n][g][i][1] : O[n][g][i][r]) * f;
          v[i + 4] = (T == 2 ? O[n][g][i][2] + O[n][g][i][3] : O[n][g][i][2 + r]) * f;
        }
        if ((j - begun) * kSets > C::kFlush) {   // (not the first)
          const float keep = exp2_fast(__ldcg(maximum_at(n, r)) - m[n][r]);
          const float4* from = reinterpret_cast<const float4*>(part + flush_row(n, r) * C::kDim + g * kGroup + gr * 8);
          const float4 x = __ldcg(from), y = __ldcg(from + 1);
          v[0] = fmaf(x.x, keep, v[0]), v[1] = fmaf(x.y, keep, v[1]), v[2] = fmaf(x.z, keep, v[2]), v[3] = fmaf(x.w, keep, v[3]);
          v[4] = fmaf(y.x, keep, v[4]), v[5] = fmaf(y.y, keep, v[5]), v[6] = fmaf(y.z, keep, v[6]), v[7] = fmaf(y.w, keep, v[7]);
        }
      };
      auto to_part = [&](int row, int g, const float (&v)[8]) {
        float4* to = reinterpret_cast<float4*>(part + row * C::kDim + g * kGroup + gr * 8);
        __stcg(to, make_float4(v[0], v[1], v[2], v[3]));
        __stcg(to + 1, make_float4(v[4], v[5], v[6], v[7]));
      };

      for (int pos = unit * N * kTile; j < end; pos += N * kTile) {
        if (__any_sync(0xffffffffu, !mbar_wait(bars + stage, phase))) gave_up = true;
        if (gave_up) break;
        if ((j + C::kStages) % (32 / N) == 0 && j + C::kStages < mine) look_up((j + C::kStages) / (32 / N));
        const unsigned missing = ((j & 32 / N) ? bad_odd : bad_even) >> j % (32 / N) * N & ((1u << N) - 1);   // tiles that have no page
        if (missing && lane == 0) ctl->status = GSI_ERR_INVALID_ARG;
        if (least - pos >= N * kTile && !missing) {
          pass(std::false_type{}, pos, 0u, j + C::kStages);
        } else if (pos < most) {
          pass(std::true_type{}, pos, missing, j + C::kStages);
        } else if constexpr (C::kSplit) {
          issue(j + 1, 0, false);
          if (__any_sync(0xffffffffu, !mbar_wait(bars + 1, phase))) gave_up = true;
        }
        if (C::kSplit && gave_up) break;
        __syncwarp();
        issue(j + C::kStages, stage, C::kSplit);
        if (++stage == C::kStages) {
          stage = 0;
          phase ^= 1u;
        }
        ++j;
        if ((j - begun) * kSets % C::kFlush == 0 && j < end) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
              for (int r = 0; r < kLR; ++r) {
                float v[8];
                lane_sums(n, g, r, v);
                to_part(flush_row(n, r), g, v);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[n][g][i][e] = 0.f;
            }
            __syncwarp();   // (the eight lanes of a row share the word: all have read the one before)
#pragma unroll
            for (int r = 0; r < kLR; ++r) __stcg(maximum_at(n, r), m[n][r]);
          }
        }
      }
      if (gave_up) {
        if (lane == 0) ctl->status = GSI_ERR_TIMEOUT;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < kLR; ++r) l[n][r] = NAN;
      }

      // ---- the segment's sums: over the lanes and the tiles of a unit; out, where they are the whole of it
      const bool whole = tail && n_units == q.units;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < kLR; ++r) {
          float top = m[n][r];
#pragma unroll
          for (int o = L; o < 4; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          const float share_of = exp2_fast(m[n][r] - top);
          l[n][r] *= share_of;
#pragma unroll
          for (int o = L; o < 32; o <<= 1) l[n][r] += __shfl_xor_sync(0xffffffffu, l[n][r], o);
          const int row = row_of(n, r);
          const bool writes = t4 < L && row < n_rows;
          const long long to = (long long)(q.q0 + step_row(row)) * a.out_token + q_head(row) * a.out_head;
          const float over = l[n][r] == 0.f ? 0.f : 1.f / l[n][r];   // (no token seen: 0)
#pragma unroll
          for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) z[n][r][g] += __shfl_xor_sync(0xffffffffu, z[n][r][g], o);
            float v[8];
            lane_sums(n, g, r, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              v[i] = (v[i] + z[n][r][g]) * share_of;
#pragma unroll
              for (int o = L; o < 4; o <<= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
            }
            if (!writes) continue;
            if (whole) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int c = g * kGroup + gr * 8 + i;
                if (c < s.head_dim) store_from_float(a.out, kType, to + c, v[i] * over);
              }
            } else {
              to_part(row, g, v);
            }
          }
          if (!whole && writes && gr == 0) __stcg(reinterpret_cast<float2*>(part + C::kPartRows * C::kDim) + row, make_float2(top, l[n][r]));
        }
      if (!whole) {
        // the boundaries between shares that lie within the segment: shares first .. first + n_parts - 1 have a part
        const long long begin = u0 + (end - n_units) - unit + C::kCost * (segment + 1);   // with what the segments count as
        const long long b1 = quotient((begin + C::kSnap) * shares + weight - 1, weight);
        const long long b2 = quotient((begin + q.units - C::kSnap + 1) * shares + weight - 1, weight) - 1;
        const int first = (int)b1 - 1, n_parts = (int)(b2 - b1) + 2;
        __threadfence();
        __syncwarp();
        bool last = false;
        if (lane == 0) {
          last = atomicAdd(a.tickets + first, 1u) == (unsigned)n_parts - 1;
          if (last) {
            a.tickets[first] = 0u;
            __threadfence();
          }
        }
        last = __any_sync(0xffffffffu, last);
        if (last && n_parts <= kFew) {
#pragma unroll 1
          for (int i = lane; i < n_rows * (C::kDim / 4); i += 32) {
            const int r = i / (C::kDim / 4), c4 = i % (C::kDim / 4);
            float2 ml[kFew];
            float4 px[kFew];
            float top = kNone;
#pragma unroll
            for (int y = 0; y < kFew; ++y) {
              const float* from = a.parts + (2ll * (first + min(y, n_parts - 1)) + (y == 0)) * C::kPart;
              ml[y] = __ldcg(reinterpret_cast<const float2*>(from + C::kPartRows * C::kDim) + r);
              px[y] = __ldcg(reinterpret_cast<const float4*>(from + r * C::kDim) + c4);
            }
#pragma unroll
            for (int y = 0; y < kFew; ++y)
              if (y < n_parts) top = fmaxf(top, ml[y].x);
            float all = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < kFew; ++y) {
              if (y >= n_parts) continue;
              const float f = exp2_fast(ml[y].x - top);
              all += ml[y].y * f;
              v[0] += px[y].x * f, v[1] += px[y].y * f, v[2] += px[y].z * f, v[3] += px[y].w * f;
            }
            const long long to = (long long)(q.q0 + step_row(r)) * a.out_token + q_head(r) * a.out_head + c4 * 4;
            for (int e = 0; e < 4; ++e)
              if (c4 * 4 + e < s.head_dim) store_from_float(a.out, kType, to + e, all == 0.f ? 0.f : v[e] / all);
          }
        } else if (last && lane == 0) {
          Pending& x = s_pending[atomicAdd(&s_n_pending, 1)];
          x.first = first;
          x.parts = n_parts;
          x.rows = n_rows;
          for (int r = 0; r < n_rows; ++r) x.out[r] = (long long)(q.q0 + step_row(r)) * a.out_token + q_head(r) * a.out_head;
        }
      }
      // the next segment
      unit += n_units;
      if (unit == q.units) {
        unit = 0;
        ++segment;
        if (++row_tile == q.n_row_tiles) {
          row_tile = 0;
          if (++head == s.n_heads) {
            head = 0;
            if (end < mine) do q = load(++seq);
              while (q.n_row_tiles == 0);
          }
        }
      }
    }
    if (gave_up) {
      // (copies in flight land before the block's memory is another's)
      for (int i = 0; i < C::kStages; ++i) {
        mbar_wait(bars + stage, phase);
        if (C::kSplit) mbar_wait(bars + 1, phase);
        if (++stage == C::kStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
  }

  // ---- segments that many warps share, by the block of the last of them: its threads take four channels each,
  // of every part or, few rows, of one part in `sets`;
  __syncthreads();
  // as many rows at a time as their weights have room for.
  constexpr int kLanes = C::kDim / 4, kWeights = 8192;
  static_assert(kWeights * 8 + kThreads * 16 + kMaxRows * 4 <= C::kSmem && kWeights >= kMaxShares, "the rings' memory is free by now");
  float2* s_ml = reinterpret_cast<float2*>(smem);                                     // [rows][parts]: maximum and sum, then the weight
  float4* s_v = reinterpret_cast<float4*>(smem + kWeights * 8);                       // [sets][rows][kLanes]
  float* s_all = reinterpret_cast<float*>(smem + kWeights * 8 + kThreads * 16);       // [rows]
  const int n_pending = s_n_pending;
  for (int i = 0; i < n_pending; ++i) {
    const Pending& x = s_pending[i];
    auto part_of = [&](int y) { return a.parts + (2ll * (x.first + y) + (y == 0)) * C::kPart; };
    const int at_once = min(x.rows, max(1, kWeights / x.parts));
    for (int r0 = 0; r0 < x.rows; r0 += at_once) {
      const int rows = min(at_once, x.rows - r0), n = rows * kLanes, sets = max(1, kThreads / n);
      for (int e = tid; e < rows * x.parts; e += kThreads) {
        const int r = e / x.parts, y = e - r * x.parts;
        s_ml[e] = __ldcg(reinterpret_cast<const float2*>(part_of(y) + C::kPartRows * C::kDim) + r0 + r);
      }
      __syncthreads();
      for (int r = warp; r < rows; r += kWarps) {
        float top = kNone, all = 0.f;
        for (int y = lane; y < x.parts; y += 32) top = fmaxf(top, s_ml[r * x.parts + y].x);
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        for (int y = lane; y < x.parts; y += 32) {
          float2& ml = s_ml[r * x.parts + y];
          ml.x = exp2_fast(ml.x - top);
          all += ml.y * ml.x;
        }
        all = warp_sum(all);
        if (lane == 0) s_all[r] = all;
      }
      __syncthreads();
      for (int e0 = 0; e0 < n; e0 += kThreads) {   // (once, but where a set is more than the block's threads)
        const int set = n >= kThreads ? 0 : tid / n, e = e0 + tid - set * n, r = e / kLanes, c4 = e - r * kLanes;
        const bool mine = set < sets && e < n;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine) {
#pragma unroll 16
          for (int y = set; y < x.parts; y += sets) {
            const float4 w = __ldcg(reinterpret_cast<const float4*>(part_of(y) + (r0 + r) * C::kDim) + c4);
            const float f = s_ml[r * x.parts + y].x;
            v.x += w.x * f, v.y += w.y * f, v.z += w.z * f, v.w += w.w * f;
          }
        }
        if (sets > 1) {
          if (mine) s_v[set * n + e] = v;
          __syncthreads();
          if (mine && set == 0)
            for (int y = 1; y < sets; ++y) {
              const float4 w = s_v[y * n + e];
              v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
            }
        }
        if (mine && set == 0) {
          const float all = s_all[r], sums[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c4 * 4 + k < s.head_dim) store_from_float(a.out, kType, x.out[r0 + r] + c4 * 4 + k, all == 0.f ? 0.f : sums[k] / all);
        }
      }
      __syncthreads();
    }
  }
}

template <int G, gsi_dtype_t kType, int L, int NT>
cudaError_t launch(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  using C = Cfg<G, kColumns<kType>, L, NT>;
  static_assert(C::kSmem + 6144 <= 232448, "with what else a block holds in shared memory");
  static_assert(C::kRows <= C::kPartRows && 4 * NT * C::kLaneRows <= C::kPartRows && C::kHalf % 16 == 0 && C::kStages >= 1, "layout");
  if (!a.q) return cudaFuncSetAttribute(k_kv_attend<G, kType, L, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
  return launch_pdl(k_kv_attend<G, kType, L, NT>, dim3(kGrid), dim3(C::kThreads), C::kSmem, stream, s, a, ctl);
}

// `rows`: of a unit, in column pairs (1, 2, 4, or 8 in two column tiles)
template <int G, gsi_dtype_t kType>
cudaError_t launch_rows(int rows, const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  if constexpr (G <= 2) {
    if (rows == 1) return launch<G, kType, 1, 1>(s, a, ctl, stream);
    if (rows == 8) return launch<G, kType, 4, 2>(s, a, ctl, stream);
  }
  if (rows <= 2) return launch<G, kType, 2, 1>(s, a, ctl, stream);
  return launch<G, kType, 4, 1>(s, a, ctl, stream);
}
template <gsi_dtype_t kType>
cudaError_t launch_groups(int rows, const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  switch (s.groups) {
    case 1: return launch_rows<1, kType>(rows, s, a, ctl, stream);
    case 2: return launch_rows<2, kType>(rows, s, a, ctl, stream);
    case 3: return launch_rows<3, kType>(rows, s, a, ctl, stream);
    default: return launch_rows<4, kType>(rows, s, a, ctl, stream);
  }
}
cudaError_t launch_any(gsi_dtype_t type, int rows, const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  return type == GSI_F32 ? launch_groups<GSI_F32>(rows, s, a, ctl, stream) : type == GSI_BF16 ? launch_groups<GSI_BF16>(rows, s, a, ctl, stream)
                                                                                           : launch_groups<GSI_F16>(rows, s, a, ctl, stream);
}

}  // namespace

cudaError_t prepare_attend(const Shape& s) {
  for (const gsi_dtype_t type : {GSI_F32, GSI_BF16, GSI_F16})
    for (int rows = 1; rows <= 8; rows *= 2) {
      const cudaError_t e = launch_any(type, rows, s, AttendArgs{}, nullptr, nullptr);
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  // The smallest unit that holds the rows of a sequence on average (half a row left over may go to a second tile of rows:
  // batches are padded); requests as in the last plan, though all are looked at.
  const double mean = (double)a.n_rows * a.shared / a.likely - 0.5;
  int rows = 1;
  while (rows < 8 && rows * (a.dtype == GSI_F32 ? 1 : 2) < mean) rows *= 2;
  return launch_any(a.dtype, rows, s, a, ctl, stream);
}

}  // namespace kv
}  // namespace gsi

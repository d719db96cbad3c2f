// A cache of keys and values in 4 bits: handles and argument checks, tables and slot maps from the requests'
// lengths, new rows into the pages and back.  The attention over them is gsi_kv_attend.cu.
#include <climits>
#include <cmath>
#include <new>
#include <type_traits>

#include "gsi_kv.cuh"

namespace gsi {
namespace kv {

namespace {

constexpr int kPlanThreads = 512;
constexpr int kLongRun = 8;   // slots of a thread in one round, where they are many
constexpr int kPlanGrid = 296;

__device__ __forceinline__ int clamp_int(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }
// (up to 2^31 - 4096 tokens)
__device__ __forceinline__ int pages_of(int tokens, const Shape& s) { return s.by_page.quotient(tokens + s.page_tokens - 1); }

// The last index s with first[s] <= i (first[0] <= i, ascending).
__device__ __forceinline__ int last_at_most(const int* first, int n, int i) {
  int lo = 0, hi = n;   // first[lo] <= i < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The block that has read the state last; the state may be written by it alone.
__device__ __forceinline__ bool read_last(Control* ctl, int* s_last) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    *s_last = atomicAdd(&ctl->plan_ticket, 1u) == gridDim.x - 1;
    if (*s_last) ctl->plan_ticket = 0u;
  }
  __syncthreads();
  return *s_last;
}

// Every block works the requests' sums out for itself (2048 requests: 16 KB from the L2), so that no block waits for
// another; the sequences' first rows and first pages stay in shared memory, where each run of tokens and each page of the
// block looks up its own.  The block that is last to have read the state moves it on.
// Bound by the launch and three dependent reads (one token or 64: 3.0-3.4 us a call); prompts of 512 requests, 2.05 million tokens,
// take 13 us, 3 of them the slots' and positions' bytes: after the scan 1.7 trips a thread, each a search, a page's lookup and a store in turn.
template <int kRun>
__global__ void __launch_bounds__(kPlanThreads) k_kv_plan(Shape s, PlanArgs a, Control* ctl) {
  extern __shared__ int sm[];
  int* s_row = sm;                    // first row of a sequence
  int* s_page = s_row + a.n_seqs;     // pages that those before it ask for
  int* s_len = s_page + a.n_seqs;     // its tokens so far; -1: refused
  __shared__ Scan2 s_warp[kPlanThreads / 32];
  __shared__ int s_last, s_took, s_refused;
  const int threads = blockDim.x;
  if (threadIdx.x == 0) s_took = s_refused = 0;
  pdl_launch_dependents();
  pdl_wait();
  const int n_free = min(max(*a.n_free, 0), s.n_pages);
  const int per = (a.n_seqs + threads - 1) / threads, first = threadIdx.x * per, last = min(first + per, a.n_seqs);
  const long long room = (long long)s.max_pages * s.page_tokens;
  auto need_of = [&](int len, int add) { return pages_of(len + add, s) - pages_of(len, s); };
  auto fits = [&](int len, int add) { return add >= 0 && len >= 0 && (long long)len + add <= room; };
  Scan2 sum{0, 0}, total;
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = a.n_new[i];
    sum.a += max(add, 0);
    if (fits(len, add)) sum.b += need_of(len, add);
  }
  Scan2 at = block_scan(sum, &total, s_warp);
  const long long n_rows = total.a;
  if (n_rows > s.max_tokens) {   // (those whose rows end behind the slots ask for nothing)
    long long row = at.a;
    sum.b = 0;
    for (int i = first; i < last; ++i) {
      const int len = a.lens[i], add = a.n_new[i];
      row += max(add, 0);
      if (fits(len, add) && row <= s.max_tokens) sum.b += need_of(len, add);
    }
    at.b = block_scan(sum, &total, s_warp).b;
  }
  int took = 0, refused = 0;
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = a.n_new[i];
    s_row[i] = clamp_int(at.a);
    s_page[i] = clamp_int(at.b);
    at.a += max(add, 0);
    bool ok = fits(len, add) && at.a <= s.max_tokens;
    if (ok) {
      const int need = need_of(len, add);
      at.b += need;
      ok = need == 0 || at.b <= n_free;
      if (ok && need) took = (int)at.b;
    }
    refused += !ok;
    s_len[i] = ok ? len : -1;
    if (blockIdx.x == 0) {
      a.q_start[i] = s_row[i];
      a.kv_len[i] = ok ? len + add : 0;
    }
  }
  if (took) atomicMax(&s_took, took);   // (the largest that is served: one result in any order)
  if (refused) atomicAdd(&s_refused, refused);
  if (blockIdx.x == 0)   // (requests that the plan is not about have no rows)
    for (int i = a.n_seqs + threadIdx.x; i <= a.upto; i += threads) {
      a.q_start[i] = clamp_int(n_rows);
      if (i < a.upto) a.kv_len[i] = 0;
    }
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.counts[0] = clamp_int(n_rows);
    a.counts[1] = s_took;
    a.counts[2] = n_free - s_took;
    a.counts[3] = s_refused;
  }
  // slots and positions, a run of tokens a thread: its sequence and the pages it may touch are looked up once
  const bool vec = ((reinterpret_cast<uintptr_t>(a.slots) | reinterpret_cast<uintptr_t>(a.positions)) & 15) == 0;
  auto page_of = [&](int q, int len, int index) {   // the page's first slot less its first position; INT_MIN if there is no such page
    const int held = pages_of(len, s);
    const int page = index < held ? a.table[(long long)q * s.max_pages + index] : a.free_pages[n_free - 1 - (s_page[q] + index - held)];
    if ((unsigned)page < (unsigned)s.n_pages) return (page - index) * s.page_tokens;
    ctl->status = GSI_ERR_INVALID_ARG;
    return INT_MIN;
  };
  for (long long i0 = ((long long)blockIdx.x * threads + threadIdx.x) * kRun; i0 < s.max_tokens; i0 += (long long)gridDim.x * threads * kRun) {
    int slot[kRun], pos[kRun];
#pragma unroll
    for (int u = 0; u < kRun; ++u) slot[u] = pos[u] = -1;
    if (i0 < n_rows) {
      int q = last_at_most(s_row, a.n_seqs, (int)i0);
      auto behind_of = [&](int x) { return x + 1 < a.n_seqs ? s_row[x + 1] : clamp_int(n_rows); };
      int behind = behind_of(q) - (int)i0;   // tokens of the sequence that are left
      if (behind >= kRun) {
        const int len = s_len[q], p = len + (int)i0 - s_row[q];
        if (len >= 0) {
          const int index = s.by_page.quotient(p), left = (index + 1) * s.page_tokens - p;   // (two pages at most)
          const int base = page_of(q, len, index), next = left < kRun ? page_of(q, len, index + 1) : base;
#pragma unroll
          for (int u = 0; u < kRun; ++u) {
            const int from = u < left ? base : next;
            pos[u] = from == INT_MIN ? -1 : p + u;
            slot[u] = from == INT_MIN ? -1 : from + p + u;
          }
        }
      } else {
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
          if (i0 + u >= n_rows) continue;
          while (behind == 0) {
            ++q;
            behind = behind_of(q) - s_row[q];
          }
          const int len = s_len[q], p = len + (int)(i0 + u) - s_row[q];
          --behind;
          if (len < 0) continue;
          const int from = page_of(q, len, s.by_page.quotient(p));
          pos[u] = from == INT_MIN ? -1 : p;
          slot[u] = from == INT_MIN ? -1 : from + p;
        }
      }
    }
    if (kRun % 4 == 0 && vec && i0 + kRun <= s.max_tokens) {
#pragma unroll
      for (int u = 0; u + 3 < kRun; u += 4) {
        *reinterpret_cast<int4*>(a.slots + i0 + u) = make_int4(slot[u], slot[u + 1], slot[u + 2], slot[u + 3]);
        *reinterpret_cast<int4*>(a.positions + i0 + u) = make_int4(pos[u], pos[u + 1], pos[u + 2], pos[u + 3]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kRun; ++u)
        if (i0 + u < s.max_tokens) {
          a.slots[i0 + u] = slot[u];
          a.positions[i0 + u] = pos[u];
        }
    }
  }
  // the new pages
  for (int j = blockIdx.x * threads + threadIdx.x; j < s_took; j += gridDim.x * threads) {
    const int q = last_at_most(s_page, a.n_seqs, j);
    a.table[(long long)q * s.max_pages + pages_of(s_len[q], s) + j - s_page[q]] = a.free_pages[n_free - 1 - j];
  }
  if (!a.commit) return;
  if (!read_last(ctl, &s_last)) return;
  for (int i = first; i < last; ++i)
    if (s_len[i] >= 0) a.lens[i] = s_len[i] + a.n_new[i];
  if (threadIdx.x == 0) *a.n_free = n_free - s_took;
}

// Pages back, in the reverse of the order in which a plan for empty sequences would take them.  In a graph: 3.2 us where none of 64 requests
// has ended; a plan for 64 prompts of 2048 tokens and their release 13.8 us together, 512 of 4000 tokens 22.5.
__global__ void __launch_bounds__(kPlanThreads) k_kv_release(Shape s, ReleaseArgs a, Control* ctl) {
  extern __shared__ int sm[];
  int* s_page = sm;   // pages that the sequences before give back
  __shared__ Scan2 s_warp[kPlanThreads / 32];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait();
  const int n_free = min(max(*a.n_free, 0), s.n_pages);
  const int per = (a.n_seqs + kPlanThreads - 1) / kPlanThreads, first = threadIdx.x * per, last = min(first + per, a.n_seqs);
  auto held = [&](int i) { return a.done[i] ? min(pages_of(min(max(a.lens[i], 0), 1 << 30), s), s.max_pages) : 0; };
  Scan2 sum{0, 0}, total;
  for (int i = first; i < last; ++i) sum.a += held(i);
  Scan2 at = block_scan(sum, &total, s_warp);
  for (int i = first; i < last; ++i) {
    s_page[i] = clamp_int(at.a);
    at.a += held(i);
  }
  __syncthreads();
  // (more pages than the pool has: not a state that plans and releases leave)
  const bool fits = total.a <= s.n_pages - n_free;
  const int n = fits ? (int)total.a : 0;
  if (!fits && blockIdx.x == 0 && threadIdx.x == 0) ctl->status = GSI_ERR_INVALID_ARG;
  for (int j = blockIdx.x * kPlanThreads + threadIdx.x; j < n; j += gridDim.x * kPlanThreads) {
    const int q = last_at_most(s_page, a.n_seqs, j);
    int* entry = a.table + (long long)q * s.max_pages + (j - s_page[q]);
    a.free_pages[n_free + n - 1 - j] = *entry;
    *entry = -1;
  }
  if (!read_last(ctl, &s_last) || !fits) return;
  for (int i = first; i < last; ++i)
    if (a.done[i]) a.lens[i] = 0;
  if (threadIdx.x == 0) *a.n_free = n_free + n;
}

__device__ __forceinline__ float min_nan(float a, float b) {   // (NaN where one is)
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Channels 4 t + 16 i .. + 3 of 64, i = 0..3, of a row as they lie in memory: what lane quarter t takes (four lanes read 64
// or 32 bytes in one go).  Of channels from n on, channel 0 again, which changes neither bound.
template <gsi_dtype_t kType>
struct Quarters {
  static constexpr int kWords = kType == GSI_F32 ? 16 : 8;
  uint32_t w[kWords];

  template <bool kVec>
  __device__ __forceinline__ void load(const void* base, long long at, int t, int n) {
    if (kVec && n >= kGroup) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kType == GSI_F32) {
          const uint4 v = *(reinterpret_cast<const uint4*>(static_cast<const float*>(base) + at) + 4 * i + t);
          w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        } else {
          const uint2 v = *(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at) + 4 * i + t);
          w[2 * i] = v.x, w[2 * i + 1] = v.y;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = i / 4 * 16 + t * 4 + i % 4;
        if constexpr (kType == GSI_F32) {
          w[i] = *(static_cast<const uint32_t*>(base) + at + (c < n ? c : 0));
        } else {
          const uint32_t v = *(static_cast<const uint16_t*>(base) + at + (c < n ? c : 0));
          w[i / 2] = (i & 1) ? w[i / 2] | v << 16 : v;
        }
      }
    }
  }
  __device__ __forceinline__ float channel(int i) const {
    if constexpr (kType == GSI_F32) return __uint_as_float(w[i]);
    else if constexpr (kType == GSI_BF16) return __uint_as_float((i & 1) ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    else return (i & 1) ? __high2float(*reinterpret_cast<const __half2*>(&w[i / 2])) : __low2float(*reinterpret_cast<const __half2*>(&w[i / 2]));
  }
  // NaN where one is.
  __device__ __forceinline__ void bounds(float* lo, float* hi) const {
    if constexpr (kType == GSI_F32) {
      *lo = *hi = channel(0);
#pragma unroll
      for (int i = 1; i < 16; ++i) {
        *lo = min_nan(*lo, channel(i));
        *hi = max_nan(*hi, channel(i));
      }
    } else {
      using Pair = typename std::conditional<kType == GSI_BF16, __nv_bfloat162, __half2>::type;
      Pair a = *reinterpret_cast<const Pair*>(&w[0]), b = a;
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        a = __hmin2_nan(a, *reinterpret_cast<const Pair*>(&w[i]));
        b = __hmax2_nan(b, *reinterpret_cast<const Pair*>(&w[i]));
      }
      *lo = min_nan(__low2float(a), __high2float(a));
      *hi = max_nan(__low2float(b), __high2float(b));
    }
  }
};

// The pair (s, mid) of 64 channels, and what takes their codes.
struct Scale {
  __half2 pair;
  float step, mid, inverse;
  bool finite, plain;   // plain: no code has to be clamped
};
__device__ __forceinline__ Scale scale_of(float lo, float hi) {
  Scale z;
  z.finite = lo >= -3.402823466e38f && hi <= 3.402823466e38f;   // (false for NaN)
  const __half s = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f), 65504.f));
  z.step = __half2float(s);
  const __half mid = __float2half_rn(fminf(fmaxf(__fadd_rn(lo, 8.f * z.step), -65504.f), 65504.f));
  z.mid = __half2float(mid);
  z.inverse = z.step > 0.f ? __fdividef(1.f, z.step) : 0.f;   // (no step: code 8)
  z.pair = z.finite ? __halves2half2(s, mid) : __half2half2(__ushort_as_half(0x7FFF));
  z.plain = z.finite && (lo - z.mid) * z.inverse > -8.499f && (hi - z.mid) * z.inverse < 7.499f;
  return z;
}
__device__ __noinline__ uint32_t exact_codes(float4 x, float mid, float step, bool finite) {
  uint32_t got = 0u;
  const float channel[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float code = __fadd_rn(rintf(__fdiv_rn(__fsub_rn(channel[k], mid), step)), 8.f);
    got |= (uint32_t)fminf(fmaxf(code, 0.f), 15.f) << 4 * k;
  }
  return finite ? got : 0u;
}
constexpr float kWhole = 12582912.f;   // 1.5 x 2^23: a sum with it is a whole number of its last digit

// Codes of a lane's sixteen channels, four to 16 bits.  code - 8 = rint((x - mid) / s), where the product with 1 / s serves for
// the quotient, a single fp32 division: it is off by 8.5 (2^-22 + 2^-24) at most, which only matters next to a border (where
// 16-bit rows lie once in a thousand channels: their differences from mid often are a whole number and a half of steps).
template <gsi_dtype_t kType>
__device__ __forceinline__ void codes_of(const Quarters<kType>& q, const Scale& z, uint32_t (&got)[4]) {
  float far = 0.f;
  auto exact = [&](int i) {
    got[i] = exact_codes(make_float4(q.channel(4 * i), q.channel(4 * i + 1), q.channel(4 * i + 2), q.channel(4 * i + 3)), z.mid, z.step, z.finite);
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float v = 0.f;
    if (kType != GSI_F32) far = 0.f;
#pragma unroll
    for (int k = 3; k >= 0; --k) {
      const float r = __fsub_rn(q.channel(4 * i + k), z.mid) * z.inverse, whole = __fsub_rn(__fadd_rn(r, kWhole), kWhole);
      far = fmaxf(far, fabsf(r - whole));
      v = fmaf(v, 16.f, whole);
    }
    got[i] = __float_as_uint(v + (8388608.f + 0x8888)) & 0xFFFFu;   // (the sum of code 16^k, as a whole number)
    if (kType != GSI_F32 && !(z.plain && far < 0.49999f)) exact(i);
  }
  if (kType == GSI_F32 && !(z.plain && far < 0.49999f)) {   // (seldom: one look for all)
#pragma unroll
    for (int i = 0; i < 4; ++i) exact(i);
  }
}

// Of four lanes (quarters t of a row), each with four 16-bit pieces h[i] of piece group i: lane t gets group t's four, in
// lane order.
__device__ __forceinline__ uint2 transpose4(uint32_t h0, uint32_t h1, uint32_t h2, uint32_t h3, int t) {
  const uint32_t low = h0 | h1 << 16, high = h2 | h3 << 16;
  const uint32_t far = __shfl_xor_sync(0xffffffffu, (t & 2) ? low : high, 2);
  const uint32_t a = (t & 2) ? far : low, b = (t & 2) ? high : far;    // groups (t & 2) + 0, 1 of lanes t & 1 and (t & 1) + 2
  const uint32_t send = (t & 1) ? __byte_perm(a, b, 0x5410) : __byte_perm(a, b, 0x7632);
  const uint32_t keep = (t & 1) ? __byte_perm(a, b, 0x7632) : __byte_perm(a, b, 0x5410);
  const uint32_t got = __shfl_xor_sync(0xffffffffu, send, 1);
  const uint32_t first = (t & 1) ? got : keep, second = (t & 1) ? keep : got;   // of lanes 0 and 2, of lanes 1 and 3
  return make_uint2(__byte_perm(first, second, 0x5410), __byte_perm(first, second, 0x7632));
}

// A warp takes eight tokens of one head, 64 channels of K and of V (of one of them, where rows are few: grid.z = 2): four
// lanes a token, sixteen channels a lane.  Blocks of the same tokens are neighbours: heads, or (head, channels) where rows are few.
constexpr int kRowWarps = 4;
struct Item {
  int row, head, group;
};
__device__ __forceinline__ Item item_of(const Shape& s, long long octet, int head, int group) {
  return {(int)(octet * 8) + (int)(threadIdx.x & 31) / 4, head, group};
}
#define FOR_OCTETS(octet, n) \
  for (long long octet = (long long)blockIdx.y * kRowWarps + (threadIdx.x >> 5); octet * 8 < (n); octet += (long long)gridDim.y * kRowWarps)

// The block of K of a slot's tile (that of V is as many blocks on as a head has); t: the token within the tile.
__device__ __forceinline__ unsigned char* block_of(const Shape& s, unsigned char* pages, int slot, const Item& it, int* t) {
  const int page = s.by_page.quotient(slot), in = slot - page * s.page_tokens;
  *t = in % kTile;
  return pages + tile_at(s, page, it.head, in / kTile) + it.group * kBlockBytes;
}

// K and V of a row are under way together.  Bound by issue for long prompts (slots 75 % busy when all sixteen channels were divided): 16001 rows of 32 heads
// of 128 take 106 us in bf16 (3.2 TB/s), 8000 in fp32 64 us (4.7 TB/s).
template <gsi_dtype_t kType, bool kVec>
__global__ void __launch_bounds__(kRowWarps * 32, kType == GSI_F32 ? 7 : 8) k_kv_append(Shape s, RowsArgs a, Control* ctl) {
  const int quarter = threadIdx.x & 3;
  pdl_launch_dependents();
  pdl_wait();
  const int v0 = blockIdx.z, v1 = gridDim.z == 2 ? v0 + 1 : 2;
  const bool whole = gridDim.x == s.n_heads;   // all channels of a head
  const int head = whole ? blockIdx.x : blockIdx.x / s.groups, g0 = whole ? 0 : blockIdx.x - head * s.groups, g1 = whole ? s.groups : g0 + 1;
  FOR_OCTETS(octet, a.n) {
    Item it = item_of(s, octet, head, g0);
    int slot = it.row < a.n ? a.slots[it.row] : -1;
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    const int from = min(it.row, a.n - 1);   // (a row that goes nowhere is read all the same)
    const int other = __shfl_xor_sync(0xffffffffu, slot, 4);
    int t = 0;
    unsigned char* first = slot >= 0 ? block_of(s, a.pages, slot, it, &t) : nullptr;
    const long long k_at = from * a.k_token + head * a.k_head, v_at = from * a.v_token + head * a.v_head;
    for (; it.group < g1; ++it.group) {
      Quarters<kType> rows[2];
      if (v0 == 0) rows[0].template load<kVec>(a.k, k_at + it.group * kGroup, quarter, s.head_dim - it.group * kGroup);
      if (v1 == 2) rows[1].template load<kVec>(a.v, v_at + it.group * kGroup, quarter, s.head_dim - it.group * kGroup);
      unsigned char* block = first + (it.group - g0) * kBlockBytes;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        if (v < v0 || v >= v1) continue;
        float lo, hi;
        rows[v].bounds(&lo, &hi);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
          hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        }
        const Scale z = scale_of(lo, hi);
        uint32_t codes[4];
        codes_of(rows[v], z, codes);
        const uint2 code = transpose4(codes[0], codes[1], codes[2], codes[3], quarter);
        unsigned char* to = block + v * s.groups * kBlockBytes;
        if (first && quarter == 0) *reinterpret_cast<__half2*>(to + pair_byte(t)) = z.pair;
        if (!v) {
          if (first) *reinterpret_cast<uint2*>(to + k_byte(t, quarter * 16)) = code;
          continue;
        }
        // V: a word is four channels of a pair of tokens; where the neighbouring lanes hold the other token of the pair,
        // each writes one of their two octets of channels whole
        const uint2 far = make_uint2(__shfl_xor_sync(0xffffffffu, code.x, 4), __shfl_xor_sync(0xffffffffu, code.y, 4));
        if (!first) continue;
        if (other >= 0 && other == (slot ^ 1)) {
          const int odd = t & 1;
          const uint32_t mine = odd ? code.y : code.x, theirs = odd ? far.y : far.x;
          const uint32_t even_token = odd ? theirs : mine, odd_token = odd ? mine : theirs;
          *reinterpret_cast<uint2*>(to + v_byte(t & ~1, quarter * 16 + odd * 8)) =
              make_uint2(__byte_perm(even_token, odd_token, 0x5410), __byte_perm(even_token, odd_token, 0x7632));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint16_t*>(to + v_byte(t, quarter * 16 + i * 4)) = (uint16_t)((i < 2 ? code.x : code.y) >> 16 * (i & 1));
        }
      }
    }
  }
}

// A lane quarter takes channels 4 t + 16 i .. + 3, so that four lanes write 64 (32) bytes in one go: 16001 rows of 32 heads of 128 to
// fp32 in 102 us, 5.8 TB/s.
template <gsi_dtype_t kType, bool kVec>
__global__ void __launch_bounds__(kRowWarps * 32) k_kv_read(Shape s, RowsArgs a, Control* ctl) {
  const int quarter = threadIdx.x & 3;
  pdl_launch_dependents();
  pdl_wait();
  const int v0 = blockIdx.z, v1 = gridDim.z == 2 ? v0 + 1 : 2;
  const int head = blockIdx.x / s.groups, group = blockIdx.x - head * s.groups;
  FOR_OCTETS(octet, a.n) {
    const Item it = item_of(s, octet, head, group);
    if (it.row >= a.n) continue;
    int slot = a.slots[it.row];
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    uint32_t codes[2][4];
    __half2 pairs[2];
    if (slot >= 0) {
      int t;
      const unsigned char* block = block_of(s, a.pages, slot, it, &t);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        if (v < v0 || v >= v1) continue;
        const unsigned char* from = block + v * s.groups * kBlockBytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = i * 16 + quarter * 4;
          codes[v][i] = *reinterpret_cast<const uint16_t*>(from + (v ? v_byte(t, c) : k_byte(t, c)));
        }
        pairs[v] = *reinterpret_cast<const __half2*>(from + pair_byte(t));
      }
    }
    const long long at = it.row * a.k_token + it.head * a.k_head + it.group * kGroup;
    const int n = s.head_dim - it.group * kGroup;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if (v < v0 || v >= v1) continue;
      void* to = v ? a.v : a.k;
      const float2 pair = __half22float2(pairs[v]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = i * 16 + quarter * 4;
        float x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          x[k] = slot >= 0 ? __fmaf_rn(pair.x, (float)((int)(codes[v][i] >> 4 * k & 15u) - 8), pair.y) : 0.f;   // (the product is exact)
        if (kVec && c + 4 <= n) {
          if constexpr (kType == GSI_F32) {
            __stcs(reinterpret_cast<float4*>(static_cast<float*>(to) + at + c), make_float4(x[0], x[1], x[2], x[3]));
          } else {
            uint2 y;
            if constexpr (kType == GSI_BF16) {
              const __nv_bfloat162 p = __floats2bfloat162_rn(x[0], x[1]), q = __floats2bfloat162_rn(x[2], x[3]);
              y = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
            } else {
              const __half2 p = __floats2half2_rn(x[0], x[1]), q = __floats2half2_rn(x[2], x[3]);
              y = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
            }
            __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(to) + at + c), y);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k < n) store_from_float(to, kType, at + c + k, x[k]);
        }
      }
    }
  }
}

dim3 rows_grid(const Shape& s, int n, bool whole_heads) {
  const long long octet_blocks = ((long long)n + 8 * kRowWarps - 1) / (8 * kRowWarps);
  // K and V of a row, and the blocks of a head, apart where there are warps for it (64 rows at 16 heads of 256: 7.3 us in and
  // back against 10.5)
  const bool few = (long long)s.n_heads * s.groups * octet_blocks <= 148 * 4;
  const long long wide = few || !whole_heads ? (long long)s.n_heads * s.groups : s.n_heads, most = 65535;
  return dim3((unsigned)wide, (unsigned)(octet_blocks < most ? octet_blocks : most), few ? 2 : 1);
}

}  // namespace

cudaError_t launch_plan(const Shape& s, const PlanArgs& a, Control* ctl, cudaStream_t stream) {
  // A token a thread for decode steps (64 requests: 3.3 us a call against 5.2), runs of them for prompts.
  const bool one = s.max_tokens <= kPlanThreads * 4;
  const int threads = a.n_seqs <= 128 && s.max_tokens <= 128 ? 128 : kPlanThreads, run = one ? 1 : kLongRun;
  const long long blocks = ((long long)s.max_tokens + threads * run - 1) / (threads * run);
  return launch_pdl(one ? k_kv_plan<1> : k_kv_plan<kLongRun>, dim3((unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid)), dim3(threads), (size_t)a.n_seqs * 12,
                    stream, s, a, ctl);
}
cudaError_t launch_release(const Shape& s, const ReleaseArgs& a, Control* ctl, cudaStream_t stream) {
  const long long most = (long long)a.n_seqs * s.max_pages, blocks = ((most < s.n_pages ? most : s.n_pages) + kPlanThreads * kLongRun - 1) / (kPlanThreads * kLongRun);
  return launch_pdl(k_kv_release, dim3((unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid)), dim3(kPlanThreads), (size_t)a.n_seqs * 4, stream, s, a, ctl);
}
template <gsi_dtype_t kType>
static cudaError_t append_of(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  constexpr long long size = kType == GSI_F32 ? 4 : 2, mask = 4 * size - 1;   // four channels at a time
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & mask) == 0 &&
                   ((a.k_token | a.k_head | a.v_token | a.v_head) * size & mask) == 0;
  const dim3 grid = rows_grid(s, a.n, true);
  return vec ? launch_pdl(k_kv_append<kType, true>, grid, dim3(kRowWarps * 32), 0, stream, s, a, ctl) : launch_pdl(k_kv_append<kType, false>, grid, dim3(kRowWarps * 32), 0, stream, s, a, ctl);
}
template <gsi_dtype_t kType>
static cudaError_t read_of(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  const uintptr_t mask = kType == GSI_F32 ? 15 : 7;
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & mask) == 0 && s.head_dim % 4 == 0;
  const dim3 grid = rows_grid(s, a.n, false);
  return vec ? launch_pdl(k_kv_read<kType, true>, grid, dim3(kRowWarps * 32), 0, stream, s, a, ctl) : launch_pdl(k_kv_read<kType, false>, grid, dim3(kRowWarps * 32), 0, stream, s, a, ctl);
}
cudaError_t launch_append(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  return a.dtype == GSI_F32 ? append_of<GSI_F32>(s, a, ctl, stream) : a.dtype == GSI_BF16 ? append_of<GSI_BF16>(s, a, ctl, stream)
                                                                                        : append_of<GSI_F16>(s, a, ctl, stream);
}
cudaError_t launch_read(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  return a.dtype == GSI_F32 ? read_of<GSI_F32>(s, a, ctl, stream) : a.dtype == GSI_BF16 ? read_of<GSI_BF16>(s, a, ctl, stream)
                                                                                      : read_of<GSI_F16>(s, a, ctl, stream);
}

}  // namespace kv
}  // namespace gsi

using namespace gsi;

struct gsi_kv {
  kv::Shape shape;
  kv::Control* ctl;
  float* parts;
  unsigned* tickets;
  int device;
  int planned;   // requests of the last plan
  cudaStream_t last_stream;
};

namespace {

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t parts_bytes(const kv::Shape& s) { return (size_t)kv::kMaxShares * 2 * kv::kPartFloats(s.groups) * 4; }

gsi_status_t make_shape(const gsi_kv_desc_t* d, kv::Shape* s) {
  if (!d) return GSI_ERR_INVALID_ARG;
  if (d->n_heads <= 0 || d->head_dim <= 0 || d->page_tokens <= 0 || d->n_pages <= 0 || d->max_seqs <= 0 || d->max_pages <= 0 || d->max_tokens <= 0)
    return GSI_ERR_INVALID_ARG;
  if (d->head_dim > GSI_KV_MAX_DIM || d->n_heads > GSI_KV_MAX_HEADS || d->page_tokens % kv::kTile || d->page_tokens > 4096 || d->max_seqs > GSI_KV_MAX_SEQS ||
      (long long)d->n_pages * d->page_tokens >= 1ll << 31 || (long long)d->max_pages * d->page_tokens > 1ll << 30)
    return GSI_ERR_UNSUPPORTED;
  s->n_heads = d->n_heads;
  s->head_dim = d->head_dim;
  s->groups = (d->head_dim + kv::kGroup - 1) / kv::kGroup;
  s->page_tokens = d->page_tokens;
  s->page_tiles = d->page_tokens / kv::kTile;
  s->n_pages = d->n_pages;
  s->max_seqs = d->max_seqs;
  s->max_pages = d->max_pages;
  s->max_tokens = d->max_tokens;
  s->by_page = kv::Divisor::of(s->page_tokens);
  s->by_page_tiles = kv::Divisor::of(s->page_tiles);
  s->tile_bytes = 2ll * s->groups * kv::kBlockBytes;
  s->head_bytes = s->page_tiles * s->tile_bytes;
  s->page_bytes = s->n_heads * s->head_bytes;
  return GSI_OK;
}

inline bool is_type(gsi_dtype_t t) { return t == GSI_BF16 || t == GSI_F32 || t == GSI_F16; }
inline bool aligned(const void* p, unsigned n) { return p && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline unsigned size_of(gsi_dtype_t t) { return t == GSI_F32 ? 4 : 2; }
gsi_status_t on_device(gsi_kv_t h) {
  int now = -1;
  if (cudaGetDevice(&now) != cudaSuccess) return GSI_ERR_CUDA;
  return now == h->device ? GSI_OK : GSI_ERR_INVALID_ARG;
}
gsi_status_t launched(gsi_kv_t h, cudaStream_t stream, cudaError_t e) {
  h->last_stream = stream;
  return e == cudaSuccess ? GSI_OK : GSI_ERR_CUDA;
}
gsi_status_t attend(gsi_kv_t h, const void* q, gsi_dtype_t dtype, int64_t q_token_stride, int64_t q_head_stride, int n_rows, int n_q_heads, float scale,
                    const int* q_start, const int* kv_len, const int* table, int n_seqs, const void* pages, void* out, int64_t out_token_stride,
                    int64_t out_head_stride, bool clear, gsi_stream_t stream) {
  if (!h || !is_type(dtype) || n_rows < 0 || n_q_heads <= 0 || n_q_heads % h->shape.n_heads || n_seqs <= 0 || n_seqs > h->shape.max_seqs ||
      !std::isfinite(scale))
    return GSI_ERR_INVALID_ARG;
  if ((long long)n_rows * n_q_heads >= 1ll << 31 || n_q_heads / h->shape.n_heads > kv::kMaxShared) return GSI_ERR_UNSUPPORTED;
  if (n_rows == 0) return GSI_OK;
  if (!aligned(q, size_of(dtype)) || !aligned(out, size_of(dtype)) || !aligned(pages, 16)) return GSI_ERR_INVALID_ARG;
  for (const int* p : {q_start, kv_len, table})
    if (!aligned(p, 4)) return GSI_ERR_INVALID_ARG;
  if (q_token_stride < 0 || q_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const kv::AttendArgs a{q, out, dtype, q_token_stride, q_head_stride, out_token_stride, out_head_stride, n_rows, n_q_heads,
                         n_q_heads / h->shape.n_heads, 1.f / (n_q_heads / h->shape.n_heads), aligned(q, 16) && ((q_token_stride | q_head_stride) * size_of(dtype) & 15) == 0,
                         (float)(scale * 1.4426950408889634), q_start, kv_len, table, n_seqs, h->planned && h->planned < n_seqs ? h->planned : n_seqs, static_cast<const unsigned char*>(pages),
                         clear, h->parts, h->tickets};
  return launched(h, stream, kv::launch_attend(h->shape, a, h->ctl, stream));
}

}  // namespace

extern "C" {

size_t gsi_kv_page_bytes(const gsi_kv_desc_t* desc) {
  kv::Shape s;
  return make_shape(desc, &s) == GSI_OK ? (size_t)s.page_bytes : 0;
}

size_t gsi_kv_workspace_bytes(const gsi_kv_desc_t* desc) {
  kv::Shape s;
  return make_shape(desc, &s) == GSI_OK ? up256(sizeof(kv::Control)) + up256(kv::kMaxShares * 4) + up256(parts_bytes(s)) : 0;
}

gsi_status_t gsi_kv_locate(const gsi_kv_desc_t* desc, int slot, int head, int channel, int is_v, size_t* code_byte_out,
                           size_t* pair_byte_out) {
  kv::Shape s;
  const gsi_status_t st = make_shape(desc, &s);
  if (st != GSI_OK) return st;
  if (!code_byte_out || !pair_byte_out || slot < 0 || slot >= s.n_pages * s.page_tokens || head < 0 || head >= s.n_heads || channel < 0 ||
      channel >= s.head_dim || (is_v != 0 && is_v != 1))
    return GSI_ERR_INVALID_ARG;
  const int in = slot % s.page_tokens, t = in % kv::kTile, c = channel % kv::kGroup;
  const size_t block = (size_t)kv::tile_at(s, slot / s.page_tokens, head, in / kv::kTile) +
                       (size_t)(is_v * s.groups + channel / kv::kGroup) * kv::kBlockBytes;
  *code_byte_out = block + (is_v ? kv::v_byte(t, c) : kv::k_byte(t, c));
  *pair_byte_out = block + kv::pair_byte(t);
  return GSI_OK;
}

gsi_status_t gsi_kv_create(const gsi_kv_desc_t* desc, void* workspace, size_t workspace_bytes, gsi_stream_t stream, gsi_kv_t* out) {
  kv::Shape s;
  if (!out) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = make_shape(desc, &s);
  if (st != GSI_OK) return st;
  if (!aligned(workspace, 256)) return GSI_ERR_INVALID_ARG;
  if (workspace_bytes < gsi_kv_workspace_bytes(desc)) return GSI_ERR_WORKSPACE;
  gsi_kv* h = new (std::nothrow) gsi_kv;
  if (!h) return GSI_ERR_ALLOC;
  char* ws = static_cast<char*>(workspace);
  h->shape = s;
  h->ctl = reinterpret_cast<kv::Control*>(ws);
  h->tickets = reinterpret_cast<unsigned*>(ws + up256(sizeof(kv::Control)));
  h->parts = reinterpret_cast<float*>(ws + up256(sizeof(kv::Control)) + up256(kv::kMaxShares * 4));
  h->planned = 0;
  h->last_stream = stream;
  if (cudaGetDevice(&h->device) != cudaSuccess || kv::prepare_attend(s) != cudaSuccess ||
      cudaMemsetAsync(ws, 0, up256(sizeof(kv::Control)) + up256(kv::kMaxShares * 4), stream) != cudaSuccess ||
      cudaStreamSynchronize(stream) != cudaSuccess) {
    delete h;
    return GSI_ERR_CUDA;
  }
  *out = h;
  return GSI_OK;
}

gsi_status_t gsi_kv_plan(gsi_kv_t h, const int* n_new, int n_seqs, int commit, int* lens, int* n_free, const int* free_pages, int* table,
                         int* q_start, int* kv_len, int* slots, int* positions, int* counts, gsi_stream_t stream) {
  if (!h || n_seqs <= 0 || n_seqs > h->shape.max_seqs || (commit & ~(GSI_KV_COMMIT | GSI_KV_ALL_SEQS))) return GSI_ERR_INVALID_ARG;
  for (const void* p : {(const void*)n_new, (const void*)lens, (const void*)n_free, (const void*)free_pages, (const void*)table,
                        (const void*)q_start, (const void*)kv_len, (const void*)slots, (const void*)positions, (const void*)counts})
    if (!aligned(p, 4)) return GSI_ERR_INVALID_ARG;
  if (kv_len == lens || n_new == kv_len || n_new == lens) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const kv::PlanArgs a{n_new, n_seqs, commit & GSI_KV_ALL_SEQS ? h->shape.max_seqs : n_seqs, commit & GSI_KV_COMMIT, lens, n_free, free_pages, table, q_start, kv_len, slots, positions, counts};
  h->planned = n_seqs;
  return launched(h, stream, kv::launch_plan(h->shape, a, h->ctl, stream));
}

gsi_status_t gsi_kv_release(gsi_kv_t h, const unsigned char* done, int n_seqs, int* lens, int* n_free, int* free_pages, int* table,
                            gsi_stream_t stream) {
  if (!h || n_seqs <= 0 || n_seqs > h->shape.max_seqs || !done) return GSI_ERR_INVALID_ARG;
  for (const void* p : {(const void*)lens, (const void*)n_free, (const void*)free_pages, (const void*)table})
    if (!aligned(p, 4)) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const kv::ReleaseArgs a{done, n_seqs, lens, n_free, free_pages, table};
  return launched(h, stream, kv::launch_release(h->shape, a, h->ctl, stream));
}

gsi_status_t gsi_kv_append(gsi_kv_t h, const void* k, const void* v, gsi_dtype_t dtype, int64_t k_token_stride, int64_t k_head_stride,
                           int64_t v_token_stride, int64_t v_head_stride, const int* slots, int n_tokens, void* pages, gsi_stream_t stream) {
  if (!h || n_tokens < 0 || !is_type(dtype)) return GSI_ERR_INVALID_ARG;
  if (n_tokens == 0) return GSI_OK;
  if (!aligned(k, size_of(dtype)) || !aligned(v, size_of(dtype)) || !aligned(slots, 4) || !aligned(pages, 16)) return GSI_ERR_INVALID_ARG;
  if (k_token_stride < 0 || k_head_stride < 0 || v_token_stride < 0 || v_head_stride < 0) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const kv::RowsArgs a{const_cast<void*>(k), const_cast<void*>(v), dtype, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
                       slots, n_tokens, static_cast<unsigned char*>(pages)};
  return launched(h, stream, kv::launch_append(h->shape, a, h->ctl, stream));
}

gsi_status_t gsi_kv_read(gsi_kv_t h, const void* pages, const int* slots, int n, gsi_dtype_t dtype, void* k_out, void* v_out,
                         gsi_stream_t stream) {
  if (!h || n < 0 || !is_type(dtype)) return GSI_ERR_INVALID_ARG;
  if (n == 0) return GSI_OK;
  if (!aligned(k_out, size_of(dtype)) || !aligned(v_out, size_of(dtype)) || !aligned(slots, 4) || !aligned(pages, 16)) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const long long head = h->shape.head_dim, token = head * h->shape.n_heads;
  const kv::RowsArgs a{k_out, v_out, dtype, token, head, token, head, slots, n, static_cast<unsigned char*>(const_cast<void*>(pages))};
  return launched(h, stream, kv::launch_read(h->shape, a, h->ctl, stream));
}

gsi_status_t gsi_kv_attend(gsi_kv_t h, const void* q, gsi_dtype_t dtype, int64_t q_token_stride, int64_t q_head_stride, int n_rows,
                           int n_q_heads, float scale, const int* q_start, const int* kv_len, const int* table, int n_seqs,
                           const void* pages, void* out, int64_t out_token_stride, int64_t out_head_stride, gsi_stream_t stream) {
  return attend(h, q, dtype, q_token_stride, q_head_stride, n_rows, n_q_heads, scale, q_start, kv_len, table, n_seqs, pages, out, out_token_stride,
                out_head_stride, false, stream);
}

gsi_status_t gsi_kv_attend_all(gsi_kv_t h, const void* q, gsi_dtype_t dtype, int64_t q_token_stride, int64_t q_head_stride, int n_rows,
                               int n_q_heads, float scale, const int* q_start, const int* kv_len, const int* table, int n_seqs,
                               const void* pages, void* out, int64_t out_token_stride, int64_t out_head_stride, gsi_stream_t stream) {
  return attend(h, q, dtype, q_token_stride, q_head_stride, n_rows, n_q_heads, scale, q_start, kv_len, table, n_seqs, pages, out, out_token_stride,
                out_head_stride, true, stream);
}

gsi_status_t gsi_kv_get_status(gsi_kv_t h, int* device_status) {
  if (!h || !device_status) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  if (cudaStreamSynchronize(h->last_stream) != cudaSuccess) return GSI_ERR_CUDA;
  int v = 0;
  if (cudaMemcpy(&v, &h->ctl->status, sizeof v, cudaMemcpyDeviceToHost) != cudaSuccess) return GSI_ERR_CUDA;
  *device_status = v;
  return GSI_OK;
}

gsi_status_t gsi_kv_destroy(gsi_kv_t h) {
  if (!h) return GSI_ERR_INVALID_ARG;
  delete h;
  return GSI_OK;
}

}  // extern "C"

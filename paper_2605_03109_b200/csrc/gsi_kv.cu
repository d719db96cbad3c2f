// A cache of keys and values in 4 bits: handles and argument checks, tables and slot maps from the requests'
// lengths, new rows into the pages and back.  The attention over them is gsi_kv_attend.cu.
#include <climits>
#include <cmath>
#include <new>

#include "gsi_kv.cuh"

namespace gsi {
namespace kv {

namespace {

constexpr int kPlanThreads = 512;
constexpr int kRun = 8;   // slots of a thread in one round
constexpr int kPlanGrid = 444;

__device__ __forceinline__ int clamp_int(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }
// (up to 2^31 tokens and a page)
__device__ __forceinline__ int pages_of(long long tokens, int page_tokens) { return (int)(((unsigned)tokens + page_tokens - 1) / (unsigned)page_tokens); }

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
// Bound by the launch and three dependent reads (one token: 4.1 us a call); for prompts by the writes of slots and positions.
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
  auto need_of = [&](int len, int add) { return pages_of((long long)len + add, s.page_tokens) - pages_of(len, s.page_tokens); };
  auto fits = [&](int len, int add) { return add >= 0 && len >= 0 && (long long)len + add <= room; };
  Scan2 sum{0, 0}, total;
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = __ldg(a.n_new + i);
    sum.a += max(add, 0);
    if (fits(len, add)) sum.b += need_of(len, add);
  }
  Scan2 at = block_scan(sum, &total, s_warp);
  const long long n_rows = total.a;
  if (n_rows > s.max_tokens) {   // (those whose rows end behind the slots ask for nothing)
    long long row = at.a;
    sum.b = 0;
    for (int i = first; i < last; ++i) {
      const int len = a.lens[i], add = __ldg(a.n_new + i);
      row += max(add, 0);
      if (fits(len, add) && row <= s.max_tokens) sum.b += need_of(len, add);
    }
    at.b = block_scan(sum, &total, s_warp).b;
  }
  int took = 0, refused = 0;
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = __ldg(a.n_new + i);
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
  __syncthreads();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.q_start[a.n_seqs] = clamp_int(n_rows);
    a.counts[0] = clamp_int(n_rows);
    a.counts[1] = s_took;
    a.counts[2] = n_free - s_took;
    a.counts[3] = s_refused;
  }
  // slots and positions, a run of tokens a thread: its sequence is looked up once, a page where it changes
  const bool vec = ((reinterpret_cast<uintptr_t>(a.slots) | reinterpret_cast<uintptr_t>(a.positions)) & 15) == 0;
  for (long long i0 = ((long long)blockIdx.x * threads + threadIdx.x) * kRun; i0 < s.max_tokens; i0 += (long long)gridDim.x * threads * kRun) {
    int slot[kRun], pos[kRun];
    int q = 0, len = -1, p = 0, behind = 0, base = 0, left = 0;   // tokens of the sequence, of the page, that are left
    if (i0 < n_rows) {
      q = last_at_most(s_row, a.n_seqs, (int)i0);
      behind = (q + 1 < a.n_seqs ? s_row[q + 1] : clamp_int(n_rows)) - (int)i0;
      len = s_len[q];
      p = len + (int)i0 - s_row[q];
    }
#pragma unroll
    for (int u = 0; u < kRun; ++u) {
      slot[u] = pos[u] = -1;
      if (i0 + u >= n_rows) continue;
      if (behind == 0) {
        do {
          ++q;
          behind = (q + 1 < a.n_seqs ? s_row[q + 1] : clamp_int(n_rows)) - s_row[q];
        } while (behind == 0);
        len = p = s_len[q];
        left = 0;
      }
      --behind;
      if (len < 0) continue;
      if (left == 0) {
        const int index = p / s.page_tokens, held = pages_of(len, s.page_tokens);
        const int page = index < held ? a.table[(long long)q * s.max_pages + index] : __ldg(a.free_pages + (n_free - 1 - (s_page[q] + index - held)));
        base = (unsigned)page < (unsigned)s.n_pages ? (page - index) * s.page_tokens : INT_MIN;
        left = (index + 1) * s.page_tokens - p;
        if (base == INT_MIN) ctl->status = GSI_ERR_INVALID_ARG;
      }
      if (base != INT_MIN) {
        pos[u] = p;
        slot[u] = base + p;
      }
      ++p;
      --left;
    }
    if (vec && i0 + kRun <= s.max_tokens) {
#pragma unroll
      for (int u = 0; u < kRun; u += 4) {
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
    a.table[(long long)q * s.max_pages + pages_of(s_len[q], s.page_tokens) + j - s_page[q]] = __ldg(a.free_pages + (n_free - 1 - j));
  }
  if (!a.commit) return;
  if (!read_last(ctl, &s_last)) return;
  for (int i = first; i < last; ++i)
    if (s_len[i] >= 0) a.lens[i] = s_len[i] + __ldg(a.n_new + i);
  if (threadIdx.x == 0) *a.n_free = n_free - s_took;
}

// Pages back, in the reverse of the order in which a plan for empty sequences would take them.
__global__ void __launch_bounds__(kPlanThreads) k_kv_release(Shape s, ReleaseArgs a, Control* ctl) {
  extern __shared__ int sm[];
  int* s_page = sm;   // pages that the sequences before give back
  __shared__ Scan2 s_warp[kPlanThreads / 32];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait();
  const int n_free = min(max(*a.n_free, 0), s.n_pages);
  const int per = (a.n_seqs + kPlanThreads - 1) / kPlanThreads, first = threadIdx.x * per, last = min(first + per, a.n_seqs);
  auto held = [&](int i) { return a.done[i] ? min(pages_of(max(a.lens[i], 0), s.page_tokens), s.max_pages) : 0; };
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
// Two 16-bit values of a word.
template <gsi_dtype_t kType>
__device__ __forceinline__ float2 pair_of(uint32_t w) {
  if constexpr (kType == GSI_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Channels 4 t + 16 i .. + 3 of a row, i = 0..3, as lane quarter t takes them (four lanes read 64 or 32 bytes in one go); those
// from n on repeat channel 0 of `at`, which changes neither bound.
template <gsi_dtype_t kType, bool kVec>
__device__ __forceinline__ void load_quarters(const void* base, long long at, int t, int n, float (&x)[16]) {
  if (kVec && n >= kGroup) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kType == GSI_F32) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(base) + at) + 4 * i + t);
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
      } else {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at) + 4 * i + t);
        const float2 a = pair_of<kType>(v.x), b = pair_of<kType>(v.y);
        x[4 * i] = a.x, x[4 * i + 1] = a.y, x[4 * i + 2] = b.x, x[4 * i + 3] = b.y;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = i / 4 * 16 + t * 4 + i % 4;
      x[i] = load_as_float(base, kType, at + (c < n ? c : 0));
    }
  }
}

// rint((x - mid) / step) of the four channels c .. c + 3 as signed nibbles.  The quotient, a single fp32 division, is only
// taken where the product with 1 / step, which is off by 2^-22 of it at most, lies near a border.
__device__ __forceinline__ uint32_t nibbles4(const float* x, float mid, float step, float inverse) {
  uint32_t got = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float d = __fsub_rn(x[i], mid);
    float r = fminf(fmaxf(d * inverse, -8.f), 7.f);
    float k = __fadd_rn(r, 12582912.f);   // 1.5 x 2^23: its last bits are the whole number
    if (fabsf(r - __fsub_rn(k, 12582912.f)) > 0.4999f) k = __fadd_rn(fminf(fmaxf(__fdiv_rn(d, step), -8.f), 7.f), 12582912.f);
    got |= (__float_as_uint(k) & 15u) << 4 * i;
  }
  return got;
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

// A warp takes eight tokens of one head, K or V, 64 channels: four lanes a token, sixteen channels a lane.
struct Item {
  int row, head, group, is_v;
};
__device__ __forceinline__ Item item_of(const Shape& s, int n, long long w) {
  Item it;
  it.group = (int)(w % s.groups);
  w /= s.groups;
  it.is_v = (int)(w & 1);
  w >>= 1;
  it.head = (int)(w % s.n_heads);
  it.row = (int)(w / s.n_heads) * 8 + ((threadIdx.x & 31) >> 2);
  return it;
}
__host__ __device__ __forceinline__ long long items(const Shape& s, int n) { return ((long long)n + 7) / 8 * s.n_heads * 2 * s.groups; }

// The block of a slot's tile, or null; t: the token within the tile.
__device__ __forceinline__ unsigned char* block_of(const Shape& s, unsigned char* pages, int slot, const Item& it, int* t) {
  const int page = slot / s.page_tokens, in = slot - page * s.page_tokens;
  *t = in % kTile;
  return pages + tile_at(s, page, it.head, in / kTile) + (it.is_v * s.groups + it.group) * kBlockBytes;
}

// Bound by the rows' bytes for long prompts, where 64 channels of a token cost four lanes about 70 instructions each.
template <gsi_dtype_t kType, bool kVec>
__global__ void __launch_bounds__(256) k_kv_append(Shape s, RowsArgs a, Control* ctl) {
  const int quarter = threadIdx.x & 3;
  pdl_launch_dependents();
  pdl_wait();
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < items(s, a.n); w += (long long)gridDim.x * 8) {
    const Item it = item_of(s, a.n, w);
    int slot = it.row < a.n ? __ldg(a.slots + it.row) : -1;
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (slot >= 0)
      load_quarters<kType, kVec>(it.is_v ? a.v : a.k, it.row * (it.is_v ? a.v_token : a.k_token) + it.head * (it.is_v ? a.v_head : a.k_head) + it.group * kGroup,
                                 quarter, s.head_dim - it.group * kGroup, x);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) {
      lo = min_nan(lo, x[i]);
      hi = max_nan(hi, x[i]);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const bool finite = lo >= -3.402823466e38f && hi <= 3.402823466e38f;   // (false for NaN)
    const __half s16 = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f), 65504.f));
    const float step = __half2float(s16);
    const __half m16 = __float2half_rn(fminf(fmaxf(__fadd_rn(lo, 8.f * step), -65504.f), 65504.f));
    const float mid = __half2float(m16), inverse = step == 0.f ? 0.f : __fdividef(1.f, step);
    uint2 code = transpose4(nibbles4(x, mid, step, inverse), nibbles4(x + 4, mid, step, inverse), nibbles4(x + 8, mid, step, inverse),
                            nibbles4(x + 12, mid, step, inverse), quarter);
    code.x = step == 0.f ? 0x88888888u : code.x ^ 0x88888888u;   // (8 where there is no step)
    code.y = step == 0.f ? 0x88888888u : code.y ^ 0x88888888u;
    if (!finite) code = make_uint2(0u, 0u);
    int t = 0;
    unsigned char* block = slot >= 0 ? block_of(s, a.pages, slot, it, &t) : nullptr;
    // V: a word is four channels of a pair of tokens; where the neighbouring lanes hold the other token of the pair,
    // each writes one of their two octets of channels whole
    const int other = __shfl_xor_sync(0xffffffffu, slot, 4);
    const uint2 far = make_uint2(__shfl_xor_sync(0xffffffffu, code.x, 4), __shfl_xor_sync(0xffffffffu, code.y, 4));
    if (!block) continue;
    if (quarter == 0) {
      const __half2 pair = finite ? __halves2half2(s16, m16) : __half2half2(__ushort_as_half(0x7FFF));
      *reinterpret_cast<__half2*>(block + pair_byte(t)) = pair;
    }
    if (!it.is_v) {
      *reinterpret_cast<uint2*>(block + k_byte(t, quarter * 16)) = code;
    } else if (other >= 0 && other == (slot ^ 1)) {
      const int odd = t & 1;
      const uint32_t mine = odd ? code.y : code.x, theirs = odd ? far.y : far.x;
      const uint32_t even_token = odd ? theirs : mine, odd_token = odd ? mine : theirs;
      *reinterpret_cast<uint2*>(block + v_byte(t & ~1, quarter * 16 + odd * 8)) =
          make_uint2(__byte_perm(even_token, odd_token, 0x5410), __byte_perm(even_token, odd_token, 0x7632));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint16_t*>(block + v_byte(t, quarter * 16 + i * 4)) = (uint16_t)((i < 2 ? code.x : code.y) >> 16 * (i & 1));
    }
  }
}

// A lane quarter takes channels 4 t + 16 i .. + 3, so that four lanes write 64 (32) bytes in one go.
template <gsi_dtype_t kType, bool kVec>
__global__ void __launch_bounds__(256) k_kv_read(Shape s, RowsArgs a, Control* ctl) {
  const int quarter = threadIdx.x & 3;
  pdl_launch_dependents();
  pdl_wait();
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < items(s, a.n); w += (long long)gridDim.x * 8) {
    const Item it = item_of(s, a.n, w);
    if (it.row >= a.n) continue;
    int slot = __ldg(a.slots + it.row);
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    int t = 0;
    const unsigned char* block = slot >= 0 ? block_of(s, a.pages, slot, it, &t) : nullptr;
    uint32_t codes[4] = {0u, 0u, 0u, 0u};
    float2 pair = make_float2(0.f, 0.f);
    if (block) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = i * 16 + quarter * 4;
        codes[i] = *reinterpret_cast<const uint16_t*>(block + (it.is_v ? v_byte(t, c) : k_byte(t, c)));
      }
      pair = __half22float2(*reinterpret_cast<const __half2*>(block + pair_byte(t)));
    }
    void* to = it.is_v ? a.v : a.k;
    const long long at = it.row * a.k_token + it.head * a.k_head + it.group * kGroup;
    const int n = s.head_dim - it.group * kGroup;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = i * 16 + quarter * 4;
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] = block ? __fmaf_rn(pair.x, (float)((int)(codes[i] >> 4 * k & 15u) - 8), pair.y) : 0.f;   // (the product is exact)
      if (kVec && c + 4 <= n) {
        if constexpr (kType == GSI_F32) {
          __stcs(reinterpret_cast<float4*>(static_cast<float*>(to) + at + c), make_float4(x[0], x[1], x[2], x[3]));
        } else {
          uint2 v;
          if constexpr (kType == GSI_BF16) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(x[0], x[1]), q = __floats2bfloat162_rn(x[2], x[3]);
            v = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
          } else {
            const __half2 p = __floats2half2_rn(x[0], x[1]), q = __floats2half2_rn(x[2], x[3]);
            v = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
          }
          __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(to) + at + c), v);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < n) store_from_float(to, kType, at + c + k, x[k]);
      }
    }
  }
}

int rows_grid(const Shape& s, int n) {
  const long long blocks = (items(s, n) + 7) / 8;
  return (int)(blocks < 148 * 8 ? blocks : 148 * 8);
}

}  // namespace

cudaError_t launch_plan(const Shape& s, const PlanArgs& a, Control* ctl, cudaStream_t stream) {
  const int threads = a.n_seqs <= 128 && s.max_tokens <= 128 * kRun ? 128 : kPlanThreads;
  const long long blocks = ((long long)s.max_tokens + threads * kRun - 1) / (threads * kRun);
  return launch_pdl(k_kv_plan, dim3((unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid)), dim3(threads), (size_t)a.n_seqs * 12, stream, s, a, ctl);
}
cudaError_t launch_release(const Shape& s, const ReleaseArgs& a, Control* ctl, cudaStream_t stream) {
  const long long most = (long long)a.n_seqs * s.max_pages, blocks = ((most < s.n_pages ? most : s.n_pages) + kPlanThreads * kRun - 1) / (kPlanThreads * kRun);
  return launch_pdl(k_kv_release, dim3((unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid)), dim3(kPlanThreads), (size_t)a.n_seqs * 4, stream, s, a, ctl);
}
template <gsi_dtype_t kType>
static cudaError_t append_of(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  constexpr long long size = kType == GSI_F32 ? 4 : 2, mask = 4 * size - 1;   // four channels at a time
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & mask) == 0 &&
                   ((a.k_token | a.k_head | a.v_token | a.v_head) * size & mask) == 0;
  const dim3 grid(rows_grid(s, a.n));
  return vec ? launch_pdl(k_kv_append<kType, true>, grid, dim3(256), 0, stream, s, a, ctl) : launch_pdl(k_kv_append<kType, false>, grid, dim3(256), 0, stream, s, a, ctl);
}
template <gsi_dtype_t kType>
static cudaError_t read_of(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  const uintptr_t mask = kType == GSI_F32 ? 15 : 7;
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & mask) == 0 && s.head_dim % 4 == 0;
  const dim3 grid(rows_grid(s, a.n));
  return vec ? launch_pdl(k_kv_read<kType, true>, grid, dim3(256), 0, stream, s, a, ctl) : launch_pdl(k_kv_read<kType, false>, grid, dim3(256), 0, stream, s, a, ctl);
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
  cudaStream_t last_stream;
};

namespace {

size_t up256(size_t v) { return (v + 255) / 256 * 256; }
size_t parts_bytes(const kv::Shape& s) { return (size_t)kv::kMaxShares * 2 * kv::kPartFloats(s.groups) * 4; }

gsi_status_t make_shape(const gsi_kv_desc_t* d, kv::Shape* s) {
  if (!d) return GSI_ERR_INVALID_ARG;
  if (d->n_heads <= 0 || d->head_dim <= 0 || d->page_tokens <= 0 || d->n_pages <= 0 || d->max_seqs <= 0 || d->max_pages <= 0 || d->max_tokens <= 0)
    return GSI_ERR_INVALID_ARG;
  if (d->head_dim > GSI_KV_MAX_DIM || d->n_heads > 65536 || d->page_tokens % kv::kTile || d->page_tokens > 4096 || d->max_seqs > GSI_KV_MAX_SEQS ||
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
  if (!h || n_seqs <= 0 || n_seqs > h->shape.max_seqs || (commit != 0 && commit != 1)) return GSI_ERR_INVALID_ARG;
  for (const void* p : {(const void*)n_new, (const void*)lens, (const void*)n_free, (const void*)free_pages, (const void*)table,
                        (const void*)q_start, (const void*)kv_len, (const void*)slots, (const void*)positions, (const void*)counts})
    if (!aligned(p, 4)) return GSI_ERR_INVALID_ARG;
  if (kv_len == lens || n_new == kv_len || n_new == lens) return GSI_ERR_INVALID_ARG;
  const gsi_status_t st = on_device(h);
  if (st != GSI_OK) return st;
  const kv::PlanArgs a{n_new, n_seqs, commit, lens, n_free, free_pages, table, q_start, kv_len, slots, positions, counts};
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
                         n_q_heads / h->shape.n_heads, 1.f / (n_q_heads / h->shape.n_heads), (float)(scale * 1.4426950408889634), q_start, kv_len, table, n_seqs, static_cast<const unsigned char*>(pages),
                         h->parts, h->tickets};
  return launched(h, stream, kv::launch_attend(h->shape, a, h->ctl, stream));
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

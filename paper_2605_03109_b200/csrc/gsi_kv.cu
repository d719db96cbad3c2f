// A cache of keys and values in 4 bits: handles and argument checks, tables and slot maps from the requests'
// lengths, new rows into the pages and back.  The attention over them is gsi_kv_attend.cu.
#include <cmath>
#include <new>

#include "gsi_kv.cuh"

namespace gsi {
namespace kv {

namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanTokens = 4 * kPlanThreads;   // slots of a block in one round
constexpr int kPlanGrid = 296;

__device__ __forceinline__ int clamp_int(long long v) { return v > 0x7fffffffll ? 0x7fffffff : (int)v; }
__device__ __forceinline__ int pages_of(long long tokens, int page_tokens) { return (int)((tokens + page_tokens - 1) / page_tokens); }

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
// another; the sequences' first rows and first pages stay in shared memory, where each token and page of the block
// looks up its own.  The block that is last to have read the state moves it on.
// Bound by the launch and three dependent reads; by the writes of slots and positions for prompts.
__global__ void __launch_bounds__(kPlanThreads) k_kv_plan(Shape s, PlanArgs a, Control* ctl) {
  extern __shared__ int sm[];
  int* s_row = sm;                    // first row of a sequence
  int* s_page = s_row + a.n_seqs;     // pages that those before it ask for
  int* s_len = s_page + a.n_seqs;     // its tokens so far; -1: refused
  __shared__ Scan2 s_warp[kPlanThreads / 32];
  __shared__ int s_last, s_took, s_refused;
  if (threadIdx.x == 0) s_took = s_refused = 0;
  const int n_free = min(max(*a.n_free, 0), s.n_pages);
  const int per = (a.n_seqs + kPlanThreads - 1) / kPlanThreads, first = threadIdx.x * per, last = min(first + per, a.n_seqs);
  const long long room = (long long)s.max_pages * s.page_tokens;
  // (rows of a sequence come first, whether it can be longer follows from where they end)
  Scan2 sum{0, 0}, total;
  for (int i = first; i < last; ++i) sum.a += max(__ldg(a.n_new + i), 0);
  Scan2 at = block_scan(sum, &total, s_warp);
  const long long n_rows = total.a;
  long long row = at.a;
  auto fits = [&](int len, int add, long long end) {
    return add >= 0 && len >= 0 && (long long)len + add <= room && end <= s.max_tokens;
  };
  sum = {0, 0};
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = __ldg(a.n_new + i);
    row += max(add, 0);
    if (fits(len, add, row)) sum.b += pages_of((long long)len + add, s.page_tokens) - pages_of(len, s.page_tokens);
  }
  Scan2 got = block_scan(sum, &total, s_warp);
  row = at.a;
  long long asked = got.b;
  int took = 0, refused = 0;
  for (int i = first; i < last; ++i) {
    const int len = a.lens[i], add = __ldg(a.n_new + i);
    s_row[i] = clamp_int(row);
    s_page[i] = clamp_int(asked);
    row += max(add, 0);
    bool ok = fits(len, add, row);
    if (ok) {
      const int need = pages_of((long long)len + add, s.page_tokens) - pages_of(len, s.page_tokens);
      asked += need;
      ok = need == 0 || asked <= n_free;
      if (ok && need) took = (int)asked;
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
  // slots and positions, four tokens a thread
  for (long long i0 = (long long)blockIdx.x * kPlanTokens + threadIdx.x * 4; i0 < s.max_tokens; i0 += (long long)gridDim.x * kPlanTokens) {
    int slot[4], pos[4];
    int q = i0 < n_rows ? last_at_most(s_row, a.n_seqs, (int)i0) : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      slot[u] = pos[u] = -1;
      const long long i = i0 + u;
      if (i >= n_rows || i >= s.max_tokens) continue;
      while (q + 1 < a.n_seqs && s_row[q + 1] <= i) ++q;
      const int len = s_len[q];
      if (len < 0) continue;
      const int p = len + (int)(i - s_row[q]), index = p / s.page_tokens, held = pages_of(len, s.page_tokens);
      const int page = index < held ? a.table[(long long)q * s.max_pages + index] : __ldg(a.free_pages + (n_free - 1 - (s_page[q] + index - held)));
      if ((unsigned)page >= (unsigned)s.n_pages) {
        ctl->status = GSI_ERR_INVALID_ARG;
        continue;
      }
      pos[u] = p;
      slot[u] = page * s.page_tokens + (p - index * s.page_tokens);
    }
    if (i0 + 4 <= s.max_tokens && (reinterpret_cast<uintptr_t>(a.slots) & 15) == 0 && (reinterpret_cast<uintptr_t>(a.positions) & 15) == 0) {
      *reinterpret_cast<int4*>(a.slots + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      *reinterpret_cast<int4*>(a.positions + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
      for (int u = 0; u < 4 && i0 + u < s.max_tokens; ++u) {
        a.slots[i0 + u] = slot[u];
        a.positions[i0 + u] = pos[u];
      }
    }
  }
  // the new pages
  for (int j = blockIdx.x * kPlanThreads + threadIdx.x; j < s_took; j += gridDim.x * kPlanThreads) {
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

// Sixteen channels of a row from `channel` on; those from head_dim on are 0.
template <bool kVec>
__device__ __forceinline__ void load16(const void* base, gsi_dtype_t dtype, long long at, int n, float (&x)[16]) {
  if (kVec && n >= 16) {
    if (dtype == GSI_F32) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 v = __ldg(p + i);
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
      }
    } else {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 v = __ldg(p + i);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (dtype == GSI_BF16) {
            x[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
            x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
          } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
            x[8 * i + 2 * j] = f.x;
            x[8 * i + 2 * j + 1] = f.y;
          }
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i < n ? load_as_float(base, dtype, at + i) : 0.f;
  }
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

template <bool kVec>
__global__ void __launch_bounds__(256) k_kv_append(Shape s, RowsArgs a, Control* ctl) {
  const int lane = threadIdx.x & 31, quarter = lane & 3;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < items(s, a.n); w += (long long)gridDim.x * 8) {
    const Item it = item_of(s, a.n, w);
    int slot = it.row < a.n ? __ldg(a.slots + it.row) : -1;
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    const int c = it.group * kGroup + quarter * 16, n = min(s.head_dim - c, 16);   // (n <= 0: no channel of this lane)
    float x[16];
    float lo = INFINITY, hi = -INFINITY;
    bool finite = true;
    if (slot >= 0 && n > 0)
      load16<kVec>(it.is_v ? a.v : a.k, a.dtype, it.row * (it.is_v ? a.v_token : a.k_token) + it.head * (it.is_v ? a.v_head : a.k_head) + c, n, x);
    else
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        finite = finite && fabsf(x[i]) <= 3.402823466e38f;
      }
    int all = finite;
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      all &= __shfl_xor_sync(0xffffffffu, all, o);
    }
    const __half s16 = __float2half_rn(fminf(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f), 65504.f));
    const float step = __half2float(s16);
    const __half m16 = __float2half_rn(fminf(fmaxf(__fadd_rn(lo, 8.f * step), -65504.f), 65504.f));
    const float mid = __half2float(m16);
    uint32_t code[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = step == 0.f ? 8.f : __fadd_rn(rintf(__fdiv_rn(__fsub_rn(x[i], mid), step)), 8.f);
      v = fminf(fmaxf(v, 0.f), 15.f);
      code[i >> 3] |= (all && i < n ? (uint32_t)v : 0u) << 4 * (i & 7);
    }
    int t = 0;
    unsigned char* block = slot >= 0 ? block_of(s, a.pages, slot, it, &t) : nullptr;
    // V: a word is four channels of a pair of tokens; where the neighbouring lanes hold the other token of the pair,
    // each writes one of their two octets of channels whole
    const int other = __shfl_xor_sync(0xffffffffu, slot, 4);
    const uint32_t far[2] = {__shfl_xor_sync(0xffffffffu, code[0], 4), __shfl_xor_sync(0xffffffffu, code[1], 4)};
    if (!block) continue;
    if (quarter == 0) {
      const __half2 pair = all ? __halves2half2(s16, m16) : __half2half2(__ushort_as_half(0x7FFF));
      *reinterpret_cast<__half2*>(block + pair_byte(t)) = pair;
    }
    if (!it.is_v) {
      *reinterpret_cast<uint2*>(block + k_byte(t, quarter * 16)) = make_uint2(code[0], code[1]);
    } else if (other >= 0 && other == (slot ^ 1)) {
      const int odd = t & 1;
      const uint32_t mine = odd ? code[1] : code[0], theirs = odd ? far[1] : far[0];
      const uint32_t even_token = odd ? theirs : mine, odd_token = odd ? mine : theirs;
      *reinterpret_cast<uint2*>(block + v_byte(t & ~1, quarter * 16 + odd * 8)) =
          make_uint2((even_token & 0xFFFFu) | odd_token << 16, even_token >> 16 | (odd_token & 0xFFFF0000u));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint16_t*>(block + v_byte(t, quarter * 16 + i * 4)) = (uint16_t)(code[i >> 1] >> 16 * (i & 1));
    }
  }
}

template <bool kVec>
__global__ void __launch_bounds__(256) k_kv_read(Shape s, RowsArgs a, Control* ctl) {
  const int lane = threadIdx.x & 31, quarter = lane & 3;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < items(s, a.n); w += (long long)gridDim.x * 8) {
    const Item it = item_of(s, a.n, w);
    const int c = it.group * kGroup + quarter * 16, n = min(s.head_dim - c, 16);
    if (it.row >= a.n || n <= 0) continue;
    int slot = __ldg(a.slots + it.row);
    if (slot >= s.n_pages * s.page_tokens) {
      ctl->status = GSI_ERR_INVALID_ARG;
      slot = -1;
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (slot >= 0) {
      int t;
      const unsigned char* block = block_of(s, a.pages, slot, it, &t);
      uint32_t code[2];
      if (!it.is_v) {
        const uint2 v = *reinterpret_cast<const uint2*>(block + k_byte(t, quarter * 16));
        code[0] = v.x;
        code[1] = v.y;
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // (a word of v: four channels of this token and of the other of its pair)
          const uint2 v = *reinterpret_cast<const uint2*>(block + v_byte(t & ~1, quarter * 16 + i * 8));
          code[i] = (t & 1) ? v.x >> 16 | (v.y & 0xFFFF0000u) : (v.x & 0xFFFFu) | v.y << 16;
        }
      }
      const float2 pair = __half22float2(*reinterpret_cast<const __half2*>(block + pair_byte(t)));
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[i] = __fmaf_rn(pair.x, (float)((int)(code[i >> 3] >> 4 * (i & 7) & 15u) - 8), pair.y);   // (the product is exact)
    }
    void* to = it.is_v ? a.v : a.k;
    const long long at = it.row * a.k_token + it.head * a.k_head + c;
    if (kVec && n == 16 && a.dtype == GSI_F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<float4*>(static_cast<float*>(to) + at)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) store_from_float(to, a.dtype, at + i, x[i]);
    }
  }
}

int rows_grid(const Shape& s, int n) {
  const long long blocks = (items(s, n) + 7) / 8;
  return (int)(blocks < 148 * 8 ? blocks : 148 * 8);
}

}  // namespace

cudaError_t launch_plan(const Shape& s, const PlanArgs& a, Control* ctl, cudaStream_t stream) {
  const long long blocks = ((long long)s.max_tokens + kPlanTokens - 1) / kPlanTokens;
  k_kv_plan<<<(unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid), kPlanThreads, (size_t)a.n_seqs * 12, stream>>>(s, a, ctl);
  return cudaGetLastError();
}
cudaError_t launch_release(const Shape& s, const ReleaseArgs& a, Control* ctl, cudaStream_t stream) {
  const long long most = (long long)a.n_seqs * s.max_pages, blocks = ((most < s.n_pages ? most : s.n_pages) + kPlanTokens - 1) / kPlanTokens;
  k_kv_release<<<(unsigned)(blocks < kPlanGrid ? blocks : kPlanGrid), kPlanThreads, (size_t)a.n_seqs * 4, stream>>>(s, a, ctl);
  return cudaGetLastError();
}
cudaError_t launch_append(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  const long long size = a.dtype == GSI_F32 ? 4 : 2;
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0 &&
                   ((a.k_token | a.k_head | a.v_token | a.v_head) * size & 15) == 0;
  const dim3 grid(rows_grid(s, a.n));
  if (vec) k_kv_append<true><<<grid, 256, 0, stream>>>(s, a, ctl);
  else k_kv_append<false><<<grid, 256, 0, stream>>>(s, a, ctl);
  return cudaGetLastError();
}
cudaError_t launch_read(const Shape& s, const RowsArgs& a, Control* ctl, cudaStream_t stream) {
  const bool vec = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 15) == 0 && s.head_dim % 4 == 0;
  const dim3 grid(rows_grid(s, a.n));
  if (vec) k_kv_read<true><<<grid, 256, 0, stream>>>(s, a, ctl);
  else k_kv_read<false><<<grid, 256, 0, stream>>>(s, a, ctl);
  return cudaGetLastError();
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

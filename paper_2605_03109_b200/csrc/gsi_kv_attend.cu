// Attention over keys and values in 4 bits.
#include "gsi_kv.cuh"

namespace gsi {
namespace kv {

namespace {

constexpr int kThreads = 128;

// A block per row and q head, in passes of kThreads tokens: a thread takes the dot product of a token, then of the
// output's channels.  One running maximum and sum per block.
__global__ void __launch_bounds__(kThreads) k_kv_attend(Shape s, AttendArgs a, Control* ctl) {
  __shared__ float s_q[GSI_KV_MAX_DIM], s_p[kThreads], s_red[kThreads / 32];
  __shared__ const unsigned char* s_tile[kThreads / kTile];
  const int row = blockIdx.x, head = blockIdx.y / a.shared, tid = threadIdx.x;
  // the sequence of the row
  int lo = 0, hi = a.n_seqs;
  if (row < a.q_start[0] || row >= a.q_start[a.n_seqs]) return;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.q_start[mid] <= row) lo = mid;
    else hi = mid;
  }
  const int seq = lo, kv_len = a.kv_len[seq];
  const int sees = kv_len - a.q_start[seq + 1] + row + 1;
  for (int c = tid; c < s.head_dim; c += kThreads)
    s_q[c] = load_as_float(a.q, a.dtype, row * a.q_token + blockIdx.y * a.q_head + c) * a.scale;
  float o[2] = {0.f, 0.f}, top = -INFINITY, sum = 0.f;
  for (int p0 = 0; p0 < sees; p0 += kThreads) {
    __syncthreads();
    if (tid < kThreads / kTile) {
      const int tile = p0 / kTile + tid, index = tile / s.page_tiles;
      const int page = tile * kTile < sees && index < s.max_pages ? a.table[(long long)seq * s.max_pages + index] : -1;
      s_tile[tid] = (unsigned)page < (unsigned)s.n_pages ? a.pages + tile_at(s, page, head, tile % s.page_tiles) : nullptr;
      if (tile * kTile < sees && !s_tile[tid]) ctl->status = GSI_ERR_INVALID_ARG;
    }
    __syncthreads();
    const unsigned char* tile = s_tile[tid / kTile];
    const int t = tid % kTile;
    float score = -INFINITY;
    if (p0 + tid < sees) {
      score = tile ? 0.f : NAN;
      for (int g = 0; tile && g < s.groups; ++g) {
        const unsigned char* block = tile + g * kBlockBytes;
        const float2 pair = __half22float2(*reinterpret_cast<const __half2*>(block + pair_byte(t)));
        const int n = min(kGroup, s.head_dim - g * kGroup);
        for (int c = 0; c < n; ++c) {
          const int code = block[k_byte(t, c)] >> 4 * (c & 1) & 15;
          score += s_q[g * kGroup + c] * __fmaf_rn(pair.x, (float)(code - 8), pair.y);
        }
      }
    }
    float m = score;
#pragma unroll
    for (int off = 16; off; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    if ((tid & 31) == 0) s_red[tid >> 5] = m;
    __syncthreads();
    const float next = fmaxf(top, fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3])));
    const float base = next == -INFINITY ? 0.f : next, keep = expf(top - base);
    top = next;
    s_p[tid] = p0 + tid < sees ? expf(score - base) : 0.f;
    __syncthreads();
    sum *= keep;
    o[0] *= keep;
    o[1] *= keep;
    const int n = min(kThreads, sees - p0);
    for (int i = 0; i < n; ++i) {
      const float p = s_p[i];
      const unsigned char* from = s_tile[i / kTile];
      sum += p;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int c = tid + u * kThreads;
        if (c >= s.head_dim) continue;
        if (!from) {
          o[u] = NAN;
          continue;
        }
        const unsigned char* block = from + (s.groups + c / kGroup) * kBlockBytes;
        const float2 pair = __half22float2(*reinterpret_cast<const __half2*>(block + pair_byte(i % kTile)));
        const int code = block[v_byte(i % kTile, c % kGroup)] >> 4 * (c & 1) & 15;
        o[u] += p * __fmaf_rn(pair.x, (float)(code - 8), pair.y);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int c = tid + u * kThreads;
    if (c < s.head_dim) store_from_float(a.out, a.dtype, row * a.out_token + blockIdx.y * a.out_head + c, sees > 0 ? o[u] / sum : 0.f);
  }
}

}  // namespace

cudaError_t launch_attend(const Shape& s, const AttendArgs& a, Control* ctl, cudaStream_t stream) {
  k_kv_attend<<<dim3(a.n_rows, a.n_q_heads), kThreads, 0, stream>>>(s, a, ctl);
  return cudaGetLastError();
}

}  // namespace kv
}  // namespace gsi

// Attention of drafted tokens over the paged cache (include/hstu.h): every node
// of a user's forest sees the cached tokens, the nodes on its way to its root
// and itself.
#include "kernels.h"

namespace hstu {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float cached(const void* p, int64_t i, int kind) {
  if (kind == kCacheBf16) return bf16_bits_to_f32(((const uint16_t*)p)[i]);
  if (kind == kCacheInt8) return (float)((const int8_t*)p)[i];
  return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)p)[i], 0);
}

// One workgroup for each row and head.
__global__ __launch_bounds__(kThreads) void attn_tree_kernel(const TreeArgs a, int kind) {
  __shared__ int way[kMaxDraft];
  __shared__ int count;
  __shared__ float p[kThreads];
  __shared__ float qs[128];
  __shared__ float sum[kThreads];
  const int64_t t = blockIdx.x;
  const int head = blockIdx.y, tid = threadIdx.x, H = a.ja.num_heads;
  const int b = find_seq(a.ja.seq_offsets, a.ja.num_seqs, t);
  const int64_t o = a.ja.seq_offsets[b];
  const int64_t i = t - o;
  if (i < 0 || i >= a.max_draft || t >= a.ja.seq_offsets[b + 1]) return;
  if (tid == 0) {
    int n = 0;
    int64_t x = i;
    while (true) {
      way[n++] = (int)x;
      const int64_t up = a.parents ? a.parents[o + x] : -1;
      if (up < 0 || up >= x) break;
      x = up;
    }
    count = n;
  }
  for (int c = tid; c < a.d_qk; c += kThreads)
    qs[c] = bf16_bits_to_f32(((const uint16_t*)a.t.q)[t * a.t.q_stride + head * a.d_qk + c]);
  __syncthreads();
  const int N = a.ja.max_seq_len;
  const int64_t cap = (int64_t)a.c.max_pages << a.c.lg_page;
  const int64_t n_b = max((int64_t)0, min(a.c.lengths[b], cap));
  const int64_t pi = n_b + count - 1;
  const int64_t ti = a.ja.timestamps[t];
  auto weight = [&](float s, int64_t pj, int64_t tj) {
    const int64_t at = max((int64_t)0, (N - 1) + pj - pi);
    s += a.ja.rab_pos[at] + a.ja.rab_time[time_bucket64(ti - tj, a.ja.num_buckets)];
    return s * sigmoid_fast(s);
  };
  const int c = tid % a.d_v, part = tid / a.d_v, parts = kThreads / a.d_v;
  float acc = 0.0f;
  for (int64_t j0 = 0; j0 < n_b; j0 += kThreads) {
    const int64_t j = j0 + tid;
    float w = 0.0f;
    if (j < n_b) {
      const int64_t page = a.c.page_table[(int64_t)b * a.c.max_pages + (j >> a.c.lg_page)];
      if (page >= 0 && page < a.c.num_pages) {
        const int place = (int)j & ((1 << a.c.lg_page) - 1);
        const int64_t row = ((page * H + head) << a.c.lg_page) + place;
        float s = 0.0f;
        for (int e = 0; e < a.d_qk; e++) s += qs[e] * cached(a.c.kc, row * a.d_qk + e, kind);
        if (kind != kCacheBf16) s *= a.c.k_scale[row];
        w = weight(s, j, a.c.tc[(page << a.c.lg_page) + place]);
      }
    }
    p[tid] = w;
    __syncthreads();
    for (int m = part; m < kThreads && j0 + m < n_b; m += parts) {
      const int64_t j = j0 + m;
      const int64_t page = a.c.page_table[(int64_t)b * a.c.max_pages + (j >> a.c.lg_page)];
      if (page < 0 || page >= a.c.num_pages) continue;
      const int place = (int)j & ((1 << a.c.lg_page) - 1);
      const int64_t ph = page * H + head;
      float v = cached(a.c.vc, ((ph * a.d_v + c) << a.c.lg_page) + place, kind);
      if (kind != kCacheBf16) v *= a.c.v_scale[(ph << a.c.lg_page) + place];
      acc += p[m] * v;
    }
    __syncthreads();
  }
  for (int j0 = 0; j0 < count; j0 += kThreads) {
    const int m = j0 + tid;
    if (m < count) {
      const int64_t r = o + way[m];
      const uint16_t* k = (const uint16_t*)a.t.k + r * a.t.k_stride + head * a.d_qk;
      float s = 0.0f;
      for (int e = 0; e < a.d_qk; e++) s += qs[e] * bf16_bits_to_f32(k[e]);
      p[tid] = weight(s, pi - m, a.ja.timestamps[r]);
    }
    __syncthreads();
    for (int x = part; x < kThreads && j0 + x < count; x += parts)
      acc += p[x] * bf16_bits_to_f32(((const uint16_t*)a.t.v)[(o + way[j0 + x]) * a.t.v_stride +
                                                              head * a.d_v + c]);
    __syncthreads();
  }
  sum[tid] = acc;
  __syncthreads();
  if (part == 0) {
    for (int x = 1; x < parts; x++) acc += sum[x * a.d_v + c];
    ((uint16_t*)a.out)[(t * H + head) * a.d_v + c] = f32_to_bf16_bits(acc / (float)N);
  }
}

// Depths of a forest by halving the ways to the roots: a node knows how many
// steps lie between it and a node on its way, and takes over that one's.
__global__ __launch_bounds__(kThreads) void tree_positions_kernel(int64_t total, int max_draft,
                                                                  const int64_t* offs,
                                                                  const int64_t* parents,
                                                                  const int64_t* base,
                                                                  int64_t* positions) {
  constexpr int M = kMaxDraft / kThreads;
  __shared__ short2 node[kMaxDraft];  // (a node on the way or -1, steps to it)
  const int b = blockIdx.x, tid = threadIdx.x;
  const int64_t o = offs[b];
  const int n = (int)max((int64_t)0, min(min(offs[b + 1], total) - o, (int64_t)max_draft));
  if (o < 0) return;
  short2 x[M];
  bool more = false;
#pragma unroll
  for (int m = 0; m < M; m++) {
    const int i = tid + m * kThreads;
    x[m] = short2{-1, 0};
    if (i < n && parents) {
      const int64_t up = parents[o + i];
      if (up >= 0 && up < i) x[m] = short2{(short)up, 1};
    }
    if (i < n) node[i] = x[m];
    more |= x[m].x >= 0;
  }
  while (__syncthreads_or(more)) {
    more = false;
#pragma unroll
    for (int m = 0; m < M; m++)
      if (x[m].x >= 0) {
        const short2 up = node[x[m].x];
        x[m] = short2{up.x, (short)(x[m].y + up.y)};
        more |= up.x >= 0;
      }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; m++) {
      const int i = tid + m * kThreads;
      if (i < n) node[i] = x[m];
    }
  }
  const int64_t p0 = base ? base[b] : 0;
#pragma unroll
  for (int m = 0; m < M; m++) {
    const int i = tid + m * kThreads;
    if (i < n) positions[o + i] = p0 + x[m].y;
  }
}

}  // namespace

hipError_t launch_attn_tree(const TreeArgs& a, int kind, hipStream_t s) {
  hipLaunchKernelGGL(attn_tree_kernel, dim3((unsigned)a.ja.total_tokens, a.ja.num_heads),
                     dim3(kThreads), 0, s, a, kind);
  return hipGetLastError();
}

hipError_t launch_tree_positions(int32_t num_seqs, int64_t total_tokens, int32_t max_draft,
                                 const int64_t* seq_offsets, const int64_t* parents,
                                 const int64_t* base, int64_t* positions, hipStream_t s) {
  hipLaunchKernelGGL(tree_positions_kernel, dim3((unsigned)num_seqs), dim3(kThreads), 0, s,
                     total_tokens, max_draft, seq_offsets, parents, base, positions);
  return hipGetLastError();
}

}  // namespace hstu

// Attention of drafted tokens over the paged cache: how a call is cut up, the sum
// of its partial outputs, and the positions of the drafted tokens.  The kernel
// itself is in attn_tree.h.
#include <algorithm>

#include "attn_tree.h"

namespace hstu {
namespace {

using tree::kThreads;

// A forest that the rows' ways to the roots are found in: up(l, i) is the node 2^l
// steps above node i, or -1.  levels: how many of them are in use.

// All nodes are roots.
struct FlatForest {
  static constexpr int levels = 0;
  __device__ FlatForest(const TreeArgs&, int64_t, int, short*) {}
  __device__ int up(int, int) const { return -1; }
  __device__ int64_t time(const TreeArgs& a, int64_t o, int n) const {
    return a.ja.timestamps[o + n];
  }
};

// Up to 64 nodes, node l in lane l of every wave, without LDS and barriers.
struct LaneForest {
  static constexpr int kMost = 6;
  int levels = 0, ways[kMost];
  int64_t times;
  __device__ LaneForest(const TreeArgs& a, int64_t o, int n, short*) {
    const int lane = __lane_id();
    const int64_t p = lane < n ? a.parents[o + lane] : -1;
    times = lane < n ? a.ja.timestamps[o + lane] : 0;
    int x = p >= 0 && p < lane ? (int)p : -1;
#pragma unroll
    for (int l = 0; l < kMost; l++) {
      ways[l] = x;
      if (__ballot(x >= 0)) levels = l + 1;
      const int y = __shfl(x, x >= 0 ? x : lane, 64);
      x = x >= 0 ? y : -1;
    }
  }
  __device__ int up(int l, int n) const {
    int w = ways[0];
#pragma unroll
    for (int k = 1; k < kMost; k++) w = l == k ? ways[k] : w;
    return __shfl(w, n, 64);
  }
  __device__ int64_t time(const TreeArgs&, int64_t, int n) const { return __shfl(times, n, 64); }
};

// Any number of nodes, in LDS: [level][max_draft].
struct LdsForest {
  int levels = 0, ld;
  const short* ways;
  __device__ LdsForest(const TreeArgs& a, int64_t o, int n, short* space)
      : ld(a.max_draft), ways(space) {
    bool more = false;
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int64_t p = a.parents[o + i];
      const short x = p >= 0 && p < i ? (short)p : (short)-1;
      space[i] = x;
      more |= x >= 0;
    }
    // a way has at most n - 1 steps: no level with 2^l >= n is in use
    while (__syncthreads_or(more) && 1 << ++levels < n) {
      more = false;
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const short x = space[(levels - 1) * ld + i];
        const short y = x >= 0 ? space[(levels - 1) * ld + x] : (short)-1;
        space[levels * ld + i] = y;
        more |= y >= 0;
      }
    }
  }
  __device__ int up(int l, int n) const { return ways[l * ld + n]; }
  __device__ int64_t time(const TreeArgs& a, int64_t o, int n) const {
    return a.ja.timestamps[o + n];
  }
};

__device__ __forceinline__ void add8(float* x, u32x4 v, float w) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    x[2 * i] = fmaf(w, __uint_as_float(v[i] << 16), x[2 * i]);
    x[2 * i + 1] = fmaf(w, __uint_as_float(v[i] & 0xffff0000u), x[2 * i + 1]);
  }
}

// The drafted keys of a row and head (the row's own and those on its way to the
// root), added to the partial outputs of the cached ones, in order; out = the sum
// / N.  A wave takes a row and head: d / 8 lanes share a key or a partial output,
// so several of them are under way at once.  Latency-bound for few rows, then
// bound by the partial outputs' bytes: 5 us for 16 rows of 4 heads, 11.6 us for 830 rows
// of 4 heads with up to 8 partial outputs.  Where there are many chunks the four waves
// of a workgroup share a row and head (`waves` 4).
template <int DQK, int DV, typename Forest>
__global__ __launch_bounds__(kThreads) void tree_finish_kernel(const TreeArgs a,
                                                               const TreeSplit sp) {
  constexpr int LK = DQK / 8, LV = DV / 8;  // lanes of a K row, of a V row
  extern __shared__ short space[];
  __shared__ float score[kThreads / 64][64];
  __shared__ float rest[kThreads / 64 - 1][DV];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int H = a.ja.num_heads;
  const int per = sp.per, waves = sp.waves;
  const int blocks = (a.max_draft + per - 1) / per;
  const int b = blockIdx.x / blocks, r0 = blockIdx.x % blocks * per;
  const int64_t o = a.ja.seq_offsets[b];
  const int64_t o1 = min(a.ja.seq_offsets[b + 1], a.ja.total_tokens);
  const int64_t cap = (int64_t)a.c.max_pages << a.c.lg_page;
  const int64_t n_b = max((int64_t)0, min(a.c.lengths[b], cap));
  const int L = (int)max((int64_t)0, min(o1 - o, (int64_t)a.max_draft));
  if (o < 0 || r0 >= L) return;
  const int used = (int)((n_b + sp.chunk_len - 1) / sp.chunk_len);
  const int rows = min(per, L - r0);
  const Forest forest(a, o, r0 + rows, space);
  const int N = a.ja.max_seq_len;
  const int share = waves == 1 ? 0 : wave;  // of the chunks
  const int pairs = rows * (waves == 1 ? H : 1);
  for (int pair = waves == 1 ? wave : 0; pair < pairs; pair += waves == 1 ? kThreads / 64 : 1) {
    const int i = r0 + (waves == 1 ? pair / H : pair);
    const int head = waves == 1 ? pair % H : blockIdx.y;
    const int64_t t = o + i;
    const u32x4 q8 = *reinterpret_cast<const u32x4*>(
        (const uint16_t*)a.t.q + t * a.t.q_stride + head * DQK + 8 * (lane % LK));
    auto key = [&](int n) {
      return *reinterpret_cast<const u32x4*>((const uint16_t*)a.t.k + (o + n) * a.t.k_stride +
                                             head * DQK + 8 * (lane % LK));
    };
    auto value = [&](int n) {
      return *reinterpret_cast<const u32x4*>((const uint16_t*)a.t.v + (o + n) * a.t.v_stride +
                                             head * DV + 8 * (lane % LV));
    };
    int count = 1;  // nodes on the way, this one included
    for (int l = forest.levels - 1, n = i; l >= 0; l--) {
      const int m = forest.up(l, n);
      if (m >= 0) {
        count += 1 << l;
        n = m;
      }
    }
    auto above = [&](int steps) {
      int n = i;
      for (int l = 0; l < forest.levels; l++) {
        const int m = forest.up(l, n);
        if ((steps >> l) & 1) n = m;
      }
      return n;
    };
    // The first of the values, on its way while the weights are found.
    const int first = above(min(lane / LV, count - 1));
    const u32x4 v8 = value(first);
    float x[8] = {};
    {
      const int64_t slot = a.ja.total_tokens * H * DV;
      const float* src = sp.part + (t * H + head) * DV + 8 * (lane % LV);
      const int step = 64 / LV * waves;
#pragma unroll 4
      for (int c = share * (64 / LV) + lane / LV; c < used; c += step) {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(src + c * slot);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(src + c * slot + 4);
#pragma unroll
        for (int e = 0; e < 4; e++) {
          x[e] += lo[e];
          x[4 + e] += hi[e];
        }
      }
      // the weights' factor -log2(e) comes off
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] *= -0.6931471805599453f;
    }
    if (share == 0) {
      float q[8] = {};
      add8(q, q8, 1.0f);
      const int64_t time = forest.time(a, o, i);
      // 64 nodes of the way at a time: lane y knows node y, its bias and its weight,
      // so that the loops over keys and values wait for nothing but their loads.
      for (int w0 = 0; w0 < count; w0 += 64) {
        const int here = min(64, count - w0), mine = min(lane, here - 1);
        const int node = above(w0 + mine);
        const float bias =
            tree::entry(a.ja.rab_pos[max(0, N - 1 - (w0 + mine))]) +
            tree::entry(a.ja.rab_time[time_bucket64(time - forest.time(a, o, node),
                                                    a.ja.num_buckets)]);
#pragma unroll 4
        for (int y0 = 0; y0 < here; y0 += 64 / LK) {
          float k[8] = {};
          add8(k, key(__shfl(node, min(y0 + lane / LK, here - 1), 64)), 1.0f);
          float s = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; e++) s = fmaf(q[e], k[e], s);
#pragma unroll
          for (int m = 1; m < LK; m *= 2) s += __shfl_xor(s, m, 64);
          if (lane % LK == 0) score[wave][y0 + lane / LK] = s;
        }
        __builtin_amdgcn_wave_barrier();
        float p = score[wave][mine] + bias;
        p *= sigmoid_fast(p);
        __builtin_amdgcn_wave_barrier();
#pragma unroll 4
        for (int y0 = 0; y0 < here; y0 += 64 / LV) {
          const int y = min(y0 + lane / LV, here - 1);
          const int n = __shfl(node, y, 64);
          const float w = __shfl(p, y, 64);
          const u32x4 v = w0 + y0 == 0 ? v8 : value(n);
          if (y0 + lane / LV < here) add8(x, v, w);
        }
      }
    }
#pragma unroll
    for (int m = LV; m < 64; m *= 2)
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] += __shfl_xor(x[e], m, 64);
    if (waves > 1) {
      if (share > 0 && lane < LV)
#pragma unroll
        for (int e = 0; e < 8; e++) rest[share - 1][8 * lane + e] = x[e];
      __syncthreads();
      if (share == 0)
#pragma unroll
        for (int w = 0; w < kThreads / 64 - 1; w++)
#pragma unroll
          for (int e = 0; e < 8; e++) x[e] += rest[w][8 * (lane % LV) + e];
      __syncthreads();
      if (share > 0) continue;
    }
    if (lane < LV) {
#pragma unroll
      for (int e = 0; e < 8; e++) x[e] /= (float)N;
      *reinterpret_cast<u32x4*>((uint16_t*)a.out + (t * H + head) * DV + 8 * lane) =
          pack_bf16x8(x);
    }
  }
}

// positions = base + depth of every drafted token.
__global__ __launch_bounds__(kThreads) void tree_positions_kernel(int64_t total, int max_draft,
                                                                  const int64_t* offs,
                                                                  const int64_t* parents,
                                                                  const int64_t* base,
                                                                  int64_t* positions) {
  __shared__ short2 node[kMaxDraft];
  const int b = blockIdx.x;
  const int64_t o = offs[b];
  if (o < 0) return;
  const int n = (int)max((int64_t)0, min(min(offs[b + 1], total) - o, (int64_t)max_draft));
  tree::walk(parents ? parents + o : nullptr, n, node);
  const int64_t p0 = base ? base[b] : 0;
  for (int i = threadIdx.x; i < n; i += kThreads) positions[o + i] = p0 + node[i].y;
}

}  // namespace

TreeSplit tree_split(int32_t num_seqs, int64_t total_tokens, int32_t num_heads, int32_t max_seq_len,
                     int32_t max_draft, int64_t cap) {
  // Workgroups: two for each of the 256 compute units.  16 users of 64 rows and up to
  // 8000 keys: 67 us; 256 workgroups 92, 768 77, 1024 73 (their partial outputs cost
  // more than they level).
  constexpr int64_t kWanted = 512;
  TreeSplit sp{};
  sp.rows = max_draft <= 16 ? 16 : max_draft <= 32 ? 32 : max_draft <= 64 ? 64 : 128;
  sp.row_blocks = (max_draft + sp.rows - 1) / sp.rows;
  const int64_t blocks =
      std::min((int64_t)num_seqs * sp.row_blocks, total_tokens / sp.rows + num_seqs);
  const int64_t keys = std::min(cap, (int64_t)max_seq_len);
  const int64_t most = (keys + tree::kBlock - 1) / tree::kBlock;
  // Four waves: heads and shares of the keys, or rows of one head.  Four heads share
  // what a workgroup knows of its keys and add nothing up at the end, but fewer of
  // them leave more workgroups for a small batch.
  sp.hg = sp.rows > 32 ? 1 : 4;
  while (num_heads % sp.hg) sp.hg /= 2;
  while (sp.hg > 1 && blocks * (num_heads / sp.hg) * most < kWanted) sp.hg /= 2;
  const int64_t base = blocks * (num_heads / sp.hg);
  const int64_t chunks = std::max((int64_t)1, std::min(most, (kWanted + base / 2) / base));
  sp.chunk_len = (int32_t)((most + chunks - 1) / chunks * tree::kBlock);
  sp.chunks = (int32_t)((cap + sp.chunk_len - 1) / sp.chunk_len);
  // The finish: four waves for a row and head where there are many chunks, else a wave
  // each, and a workgroup takes one row while there are few of them.
  sp.waves = sp.chunks > 16 ? 4 : 1;
  sp.per = sp.waves == 4 || total_tokens < 4096 ? 1 : total_tokens < 8192 ? 2 : 4;
  return sp;
}

hipError_t launch_attn_tree(const TreeArgs& a, const TreeSplit& sp, int kind, hipStream_t s) {
  hipError_t e = kind == kCacheBf16   ? tree::launch_bf16(a, sp, s)
                 : kind == kCacheE4m3 ? tree::launch_e4m3(a, sp, s)
                                      : tree::launch_int8(a, sp, s);
  if (e != hipSuccess || sp.last) return e;
  const dim3 grid((unsigned)((int64_t)a.ja.num_seqs * ((a.max_draft + sp.per - 1) / sp.per)),
                  sp.waves == 4 ? (unsigned)a.ja.num_heads : 1u);
  size_t space = 0;
  if (a.parents && a.max_draft > 64)
    for (int l = 0; l == 0 || 1 << l < a.max_draft; l++)
      space += (size_t)a.max_draft * sizeof(short);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), space, s, a, sp);
    return hipGetLastError();
  };
#define HSTU_FINISH(DQK, DV)                                                        \
  return !a.parents          ? go(tree_finish_kernel<DQK, DV, FlatForest>)          \
         : a.max_draft <= 64 ? go(tree_finish_kernel<DQK, DV, LaneForest>)          \
                             : go(tree_finish_kernel<DQK, DV, LdsForest>);
#define HSTU_FINISH_DV(DQK)                 \
  if (a.d_v == 32) { HSTU_FINISH(DQK, 32) } \
  if (a.d_v == 64) { HSTU_FINISH(DQK, 64) } \
  HSTU_FINISH(DQK, 128)
  if (a.d_qk == 32) { HSTU_FINISH_DV(32) }
  if (a.d_qk == 64) { HSTU_FINISH_DV(64) }
  HSTU_FINISH_DV(128)
#undef HSTU_FINISH_DV
#undef HSTU_FINISH
}

hipError_t launch_tree_positions(int32_t num_seqs, int64_t total_tokens, int32_t max_draft,
                                 const int64_t* seq_offsets, const int64_t* parents,
                                 const int64_t* base, int64_t* positions, hipStream_t s) {
  hipLaunchKernelGGL(tree_positions_kernel, dim3((unsigned)num_seqs), dim3(kThreads), 0, s,
                     total_tokens, max_draft, seq_offsets, parents, base, positions);
  return hipGetLastError();
}

}  // namespace hstu

// Attention of drafted tokens over the paged cache: how a call is cut up, the sum
// of its partial outputs, and the positions of the drafted tokens.  The kernel
// itself is in attn_tree.h.
#include <algorithm>

#include "attn_tree.h"

namespace hstu {
namespace {

using tree::kThreads;

// out = (sum over a user's chunks, in order, and the drafted part) / N.  A wave
// takes 64 groups of 4 features of a row, four waves a quarter of the chunks each.
__global__ __launch_bounds__(kThreads) void tree_join_kernel(const TreeArgs a, const TreeSplit sp) {
  __shared__ f32x4 sums[3][64];
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int b = find_seq(a.ja.seq_offsets, a.ja.num_seqs, t);
  const int64_t o = a.ja.seq_offsets[b];
  if (t < o || t - o >= a.max_draft || t >= a.ja.seq_offsets[b + 1]) return;
  const int64_t cap = (int64_t)a.c.max_pages << a.c.lg_page;
  const int64_t n_b = max((int64_t)0, min(a.c.lengths[b], cap));
  const int used = (int)((n_b + sp.chunk_len - 1) / sp.chunk_len);
  const int width = a.ja.num_heads * a.d_v / 4, c = blockIdx.y * 64 + lane;
  const int64_t slot = a.ja.total_tokens * width;
  const f32x4* src = reinterpret_cast<const f32x4*>(sp.part) + t * width + c;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < width) {
    const int per = (used + 3) / 4;
    const int end = min(used, (wave + 1) * per);
#pragma unroll 8
    for (int i = wave * per; i < end; i++) sum += src[i * slot];
    if (wave == 3) sum += src[sp.chunks * slot];
  }
  if (wave) sums[wave - 1][lane] = sum;
  __syncthreads();
  if (wave || c >= width) return;
  sum = ((sum + sums[0][lane]) + sums[1][lane]) + sums[2][lane];
  sum *= 1.0f / (float)a.ja.max_seq_len;
  uint2 w;
  w.x = pack_bf16x2(sum[0], sum[1]);
  w.y = pack_bf16x2(sum[2], sum[3]);
  reinterpret_cast<uint2*>(a.out)[t * width + c] = w;
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
  tree::walk<false>(parents ? parents + o : nullptr, n, 0, node, nullptr);
  const int64_t p0 = base ? base[b] : 0;
  for (int i = threadIdx.x; i < n; i += kThreads) positions[o + i] = p0 + node[i].y;
}

}  // namespace

TreeSplit tree_split(int32_t num_seqs, int64_t total_tokens, int32_t num_heads, int32_t max_seq_len,
                     int32_t max_draft, int64_t cap) {
  constexpr int64_t kWanted = 768;  // workgroups
  TreeSplit sp{};
  sp.rows = max_draft <= 16 ? 16 : 32;
  sp.row_blocks = (max_draft + sp.rows - 1) / sp.rows;
  const int64_t blocks =
      std::min((int64_t)num_seqs * sp.row_blocks, total_tokens / sp.rows + num_seqs);
  const int64_t keys = std::min(cap, (int64_t)max_seq_len);
  const int64_t most = (keys + tree::kBlock - 1) / tree::kBlock;
  sp.hg = num_heads % 4 == 0 ? 4 : num_heads % 2 == 0 ? 2 : 1;
  while (sp.hg > 1 && blocks * (num_heads / sp.hg) * most < kWanted) sp.hg /= 2;
  const int64_t base = blocks * (num_heads / sp.hg);
  const int64_t chunks = std::max((int64_t)1, std::min(most, (kWanted + base - 1) / base));
  sp.chunk_len = (int32_t)((most + chunks - 1) / chunks * tree::kBlock);
  sp.chunks = (int32_t)((cap + sp.chunk_len - 1) / sp.chunk_len);
  return sp;
}

hipError_t launch_attn_tree(const TreeArgs& a, const TreeSplit& sp, int kind, hipStream_t s) {
  hipError_t e = kind == kCacheBf16   ? tree::launch_bf16(a, sp, s)
                 : kind == kCacheE4m3 ? tree::launch_e4m3(a, sp, s)
                                      : tree::launch_int8(a, sp, s);
  if (e != hipSuccess || !sp.part) return e;
  const dim3 grid((unsigned)a.ja.total_tokens,
                  (unsigned)((a.ja.num_heads * a.d_v / 4 + 63) / 64));
  hipLaunchKernelGGL(tree_join_kernel, grid, dim3(kThreads), 0, s, a, sp);
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

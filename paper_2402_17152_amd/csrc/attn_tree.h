// Attention of drafted tokens over the paged cache (include/hstu.h): the kernel of
// the cached keys, instantiated for one kind of cache in each of
// attn_tree_{bf16,e4m3,int8}.hip.  Weights are pointwise, so sums over parts of the
// keys simply add up: the kernel leaves fp32 partial outputs, and a second one
// (attn_tree.hip) adds them to the drafted keys' part.
//
// A workgroup of four waves takes some drafted rows of one user, a chunk of the
// cached keys and `hg` heads; a wave takes one head, 16 R of the rows and every
// ks_count-th tile of T keys.  Waves of other rows of the same head load the same
// cached rows at the same time, which then come from the vector cache.
//
//   S^T = K Q^T on 16x16x32 matrix instructions, keys in the rows: lane
//   (row r = l % 16, group g = l / 16) of K's operand t reads key T/4 (r/4) + 4t +
//   r%4, so that accumulator t leaves keys T/4 g + 4 t + 0..3 of query row l % 16
//   in lane l.  That is the layout of the weights as the left operand of O = P V,
//   whose contraction runs over keys T/4 g + 8 s + 0..7: no exchange between lanes.
//   The cache holds V transposed, so its operand (T/4 keys of a feature) is one
//   load.  Nothing passes through LDS but what all heads and rows share.
//
// Codes of 8 bits are exact in bf16; a key's scales multiply the score and the
// weight.  Everything is kept times -log2(e): y = -log2(e) s gives SiLU(s) =
// s / (1 + 2^y) with one exp2, one reciprocal and one product, and the factor comes
// off at the end.  For 256 keys at a time the workgroup holds in LDS the pages, the
// scales, the times and the window of rab_pos that its rows can reach; where the
// time bucket of a row is the same for all keys of a tile (most of a long history:
// buckets are powers of two) the time bias is one number.
#pragma once

#include "kernels.h"

namespace hstu {
namespace tree {

constexpr int kThreads = 256;
constexpr int kBlock = 256;       // keys whose scales, times and pages are held
constexpr int kWindow = 512;      // entries of rab_pos that are held
constexpr int kMaxRows = 128;     // drafted rows of a workgroup
constexpr float kNegLog2e = -kLog2e;

// What is known of the times of a tile's keys against a row's.
enum { kTimesAny = 0, kTimesNear = 1, kTimesOne = 2 };

// What the waves of a workgroup share.
struct Shared {
  float scales[2][4][kBlock];      // of the block's keys, k (times -log2(e)) and v, per head
  float window[4][kWindow + 8];    // part of rab_pos (times -log2(e)), four shifted copies
  int64_t time[kBlock];            // of the keys
  int64_t rows16[kBlock / 16];     // first cache row of 16 keys for head 0, or -1
  short2 node[kMaxDraft];          // depths (y) of the drafted tokens
  float rtime[256];                // rab_time, times -log2(e)
  int64_t row_time[kMaxRows];
  float uniform[4][kMaxRows];      // the rows' entry of rtime for 64 keys (kTimesOne)
  int times[4];                    // kTimes* of 64 keys
};

// Two words of codes (8 of them) as bf16.
template <int KIND>
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
  u32x4 o;
  if constexpr (KIND == kCacheE4m3) {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int w = (int)(i ? hi : lo);
      o[2 * i] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
      o[2 * i + 1] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint32_t w = i ? hi : lo;
      o[2 * i] = pack_bf16x2((float)(int8_t)w, (float)(int8_t)(w >> 8));
      o[2 * i + 1] = pack_bf16x2((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
    }
  }
  return as_bf16x8(o);
}

// First of the eight features that lane group g contributes to contraction
// step `step` of K Q^T: the order in which 16-byte pieces of a cached row come.
template <int KIND, int DQK>
__device__ __forceinline__ int feature(int step, int g) {
  if (KIND == kCacheBf16 || DQK == 32) return 32 * step + 8 * g;
  return 64 * (step / 2) + 16 * g + 8 * (step % 2);
}

// Depths (node[i].y) of the nodes below n, whose parents are at `up` (null: all
// are roots), by halving the ways: in every round a node takes over the node that
// its own on the way knows of and adds that one's count of steps.  For a whole
// workgroup; ends past a barrier.
__device__ __forceinline__ void walk(const int64_t* up, int n, short2* node) {
  constexpr int M = kMaxDraft / kThreads;
  short2 x[M];
  bool more = false;
#pragma unroll
  for (int e = 0; e < M; e++) {
    const int i = threadIdx.x + e * kThreads;
    x[e] = short2{-1, 0};
    if (i < n) {
      const int64_t p = up ? up[i] : -1;
      if (p >= 0 && p < i) x[e] = short2{(short)p, 1};
      node[i] = x[e];
    }
    more |= x[e].x >= 0;
  }
  while (__syncthreads_or(more)) {
    more = false;
#pragma unroll
    for (int e = 0; e < M; e++)
      if (x[e].x >= 0) {
        const short2 u = node[x[e].x];
        x[e] = short2{u.x, (short)(x[e].y + u.y)};
        more |= u.x >= 0;
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < M; e++) {
      const int i = threadIdx.x + e * kThreads;
      if (i < n) node[i] = x[e];
    }
  }
}

// The same for up to 64 nodes in one wave, node l in lane l: returns its depth.
__device__ __forceinline__ int walk64(int parent) {
  int p = parent, d = p >= 0;
  while (__ballot(p >= 0)) {
    const int from = p >= 0 ? p : (int)__lane_id();
    const int pp = __shfl(p, from, 64), pd = __shfl(d, from, 64);
    if (p >= 0) {
      d += pd;
      p = pp;
    }
  }
  return d;
}

// Reductions over a wave; the result is in every lane.
template <bool MAX>
__device__ __forceinline__ int wave_extreme(int v) {
  auto pick = [](int x, int y) { return MAX ? (x > y ? x : y) : (x < y ? x : y); };
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));  // row_shr:1
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));  // row_shr:2
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));  // row_shr:4
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));  // row_shr:8
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xa, 0xf, false));  // row_bcast:15
  v = pick(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xc, 0xf, false));  // row_bcast:31
  return __builtin_amdgcn_readlane(v, 63);
}

template <bool MAX>
__device__ __forceinline__ int64_t wave_extreme64(int64_t v) {
  const int hi = (int)(v >> 32);
  const int top = wave_extreme<MAX>(hi);
  // the low words compare as unsigned numbers
  const int none = MAX ? INT32_MIN : INT32_MAX;
  const int lo = wave_extreme<MAX>(hi == top ? (int)((uint32_t)v ^ 0x80000000u) : none);
  return (int64_t)top << 32 | (uint32_t)(lo ^ (int)0x80000000u);
}

template <int KIND, int DQK, int DV, int R>
__global__ __launch_bounds__(kThreads, 2) void attn_tree_kernel(const TreeArgs a,
                                                                const TreeSplit sp) {
  constexpr bool Q8 = KIND != kCacheBf16;     // quantised
  constexpr int CB = Q8 ? 1 : 2;              // bytes of a code
  constexpr int T = Q8 ? 64 : 32;             // keys of a tile: 16 bytes of a feature per lane
  constexpr int GK = T / 4;                   // of a lane group
  constexpr int NT = T / 16, NS = T / 32;     // operands of K, contraction steps of P V
  constexpr int KW = DQK * CB / 16;           // words of a K row a lane reads
  constexpr int KS = DQK / 32, NC = DV / 16;  // contraction steps of K Q^T, column tiles
  __shared__ __attribute__((aligned(16))) Shared sh;
  __shared__ float sums[2 * 16 * R * DV];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int H = a.ja.num_heads, lg = a.c.lg_page;
  // Workgroups go to the eight dies in turn: the row blocks of one chunk and
  // head group, which read the same keys, follow each other on one die.
  const int die = blockIdx.x % 8, turn = blockIdx.x / 8;
  const int rb = turn % sp.row_blocks;
  const int unit = turn / sp.row_blocks * 8 + die;
  const int hgs = H / sp.hg;
  const int item = unit / hgs % sp.chunks, b = unit / hgs / sp.chunks;
  if (b >= a.ja.num_seqs) return;
  const int head0 = unit % hgs * sp.hg;
  const int cap = a.c.max_pages << lg;
  const int from = item * sp.chunk_len;
  const int32_t* table = a.c.page_table + (int64_t)b * a.c.max_pages;

  // What thread tid knows of key k0 + tid, fetched a block ahead.
  int64_t key_page, key_time;
  float key_ks[4], key_vs[4];
  auto fetch_page = [&](int k0) { return k0 + tid < cap ? table[(k0 + tid) >> lg] : -1; };
  const int first_page = fetch_page(from);
  const int64_t o = a.ja.seq_offsets[b];
  const int64_t o1 = min(a.ja.seq_offsets[b + 1], a.ja.total_tokens);
  const int n_b = (int)max((int64_t)0, min(a.c.lengths[b], (int64_t)cap));
  const int L = (int)max((int64_t)0, min(o1 - o, (int64_t)a.max_draft));
  const int r0 = rb * sp.rows;
  const int to = min(n_b, from + sp.chunk_len);
  if (o < 0 || r0 >= L || from >= to) return;
  auto fetch = [&](int k0, int page) {
    const int place = (k0 + tid) & ((1 << lg) - 1);
    key_page = k0 + tid < to && page < a.c.num_pages ? page : -1;
    key_time = key_page >= 0 ? a.c.tc[(key_page << lg) + place] : 0;
    if constexpr (Q8)
#pragma unroll
      for (int x = 0; x < 4; x++) {
        const int64_t at = ((key_page * H + head0 + x) << lg) + place;
        const bool on = key_page >= 0 && x < sp.hg;
        key_ks[x] = on ? a.c.k_scale[at] : 0.0f;
        key_vs[x] = on ? a.c.v_scale[at] : 0.0f;
      }
  };
  fetch(from, first_page);

  const int rows = min(sp.rows, L - r0);       // of the workgroup
  const int nodes = r0 + rows;
  // A wave's head, rows and share of the keys.
  const int wr_count = sp.rows / (16 * R), ks_count = 4 / (sp.hg * wr_count);
  const int hh = wave % sp.hg, wr = wave / sp.hg % wr_count, ks = wave / (sp.hg * wr_count);
  const int head = head0 + hh;
  const int w0 = wr * 16 * R;                  // its first row within the workgroup's
  const bool idle = w0 >= rows;
  const int r = lane % 16, g = lane / 16;
  const int N = a.ja.max_seq_len;

  // Q as the right operand: row r of each group, in the order of feature().
  bf16x8 q[R][KS];
#pragma unroll
  for (int m = 0; m < R; m++) {
    const int row = w0 + 16 * m + r;
    const uint16_t* src =
        (const uint16_t*)a.t.q + (o + r0 + row) * a.t.q_stride + (int64_t)head * DQK;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      u32x4 v = zero_u32x4();
      if (row < rows) v = *reinterpret_cast<const u32x4*>(src + feature<KIND, DQK>(s, g));
      q[m][s] = as_bf16x8(v);
    }
  }
  f32x4 acc[R][NC];
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int c = 0; c < NC; c++) acc[m][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int i = tid; i < a.ja.num_buckets; i += kThreads)
    sh.rtime[i] = a.ja.rab_time[i] * kNegLog2e;
  if (tid < kMaxRows) sh.row_time[tid] = tid < rows ? a.ja.timestamps[o + r0 + tid] : 0;
  // Depths of the rows (0 where there is none), and their extremes.
  const int64_t* parents = a.parents ? a.parents + o : nullptr;
  int depth[R], deep = 0, flat = 0;
#pragma unroll
  for (int m = 0; m < R; m++) depth[m] = 0;
  if (parents) {
    if (nodes <= 64) {
      const int64_t p = lane < nodes ? parents[lane] : -1;
      const int d = walk64(p >= 0 && p < lane ? (int)p : -1);
#pragma unroll
      for (int m = 0; m < R; m++) {
        const int x = __shfl(d, (r0 + w0 + 16 * m + r) & 63, 64);
        if (w0 + 16 * m + r < rows) depth[m] = x;
      }
      const bool own = lane >= r0 && lane < nodes;
      deep = wave_extreme<true>(own ? d : 0);
      flat = wave_extreme<false>(own ? d : kMaxDraft);
    } else {
      walk(parents, nodes, sh.node);
      flat = kMaxDraft;
      for (int i = r0 + lane; i < nodes; i += 64) {
        deep = max(deep, (int)sh.node[i].y);
        flat = min(flat, (int)sh.node[i].y);
      }
      deep = wave_extreme<true>(deep);
      flat = wave_extreme<false>(flat);
#pragma unroll
      for (int m = 0; m < R; m++)
        if (w0 + 16 * m + r < rows) depth[m] = sh.node[r0 + w0 + 16 * m + r].y;
    }
  }
  const bool windowed = deep - flat < kWindow - kBlock;
  // Where a row's window starts; a row that is not there takes the deepest's.
  int shift[R];
#pragma unroll
  for (int m = 0; m < R; m++) shift[m] = windowed ? max(0, min(deep - depth[m], deep - flat)) : 0;

  uint32_t kw[NT][KW];
  uint32_t vw[NC][4];
  for (int k0 = from; k0 < to; k0 += kBlock) {
    const int keys = min(kBlock, to - k0);
    __syncthreads();  // the block before is done with what follows
    const bool ok = key_page >= 0;
    if (tid % 16 == 0)
      sh.rows16[tid / 16] =
          ok ? ((key_page * H) << lg) + ((k0 + tid) & ((1 << lg) - 1)) : -1;
    const int next_page = fetch_page(k0 + kBlock);
    __syncthreads();
    // Cached row of key `at` of the block for head 0, or -1.
    auto row_of = [&](int at) {
      const int64_t x = sh.rows16[at / 16];
      return x < 0 ? x : x + at % 16;
    };
    auto load_k = [&](int t0, bool full) {
#pragma unroll
      for (int t = 0; t < NT; t++) {
        const int at = t0 + GK * (r / 4) + 4 * t + r % 4;
        const int64_t row = row_of(at);
        const char* src = (const char*)a.c.kc + (row + ((int64_t)head << lg)) * (DQK * CB);
        const bool on = full || (row >= 0 && at < keys);
        if constexpr (KW == 2) {
          uint2 v{0u, 0u};
          if (on) v = *reinterpret_cast<const uint2*>(src + 8 * g);
          kw[t][0] = v.x;
          kw[t][1] = v.y;
        } else {
#pragma unroll
          for (int u = 0; u < KW / 4; u++) {
            u32x4 v = zero_u32x4();
            if (on) v = *reinterpret_cast<const u32x4*>(src + 64 * u + 16 * g);
#pragma unroll
            for (int e = 0; e < 4; e++) kw[t][4 * u + e] = v[e];
          }
        }
      }
    };
    // How many of the keys of group g of a tile are there.
    auto left_of = [&](int t0) {
      const int at = t0 + GK * g;
      return sh.rows16[at / 16] < 0 ? 0 : max(0, min(GK, keys - at));
    };
    auto load_v = [&](int t0, bool full) {
      const int64_t row = row_of(t0 + GK * g);
      const int place = (int)(row & ((1 << lg) - 1));
      const int64_t ph = (row >> lg) + head;
      const int left = full ? GK : left_of(t0);
#pragma unroll
      for (int c = 0; c < NC; c++) {
        const char* src = (const char*)a.c.vc + (((ph * DV + 16 * c + r) << lg) + place) * CB;
        u32x4 v = zero_u32x4();
        if (full || left > 0) v = *reinterpret_cast<const u32x4*>(src);
        if (!full)
#pragma unroll
          for (int e = 0; e < 4; e++) {  // codes behind the last key count as zeros
            const int keep = (left * CB - 4 * e) * 8;  // bits
            v[e] = keep >= 32 ? v[e] : keep <= 0 ? 0u : v[e] & ((1u << keep) - 1u);
          }
#pragma unroll
        for (int e = 0; e < 4; e++) vw[c][e] = v[e];
      }
    };
    auto is_full = [&](int t0) {
      bool yes = t0 + T <= keys;
#pragma unroll
      for (int x = 0; x < T / 16; x++) yes = yes && sh.rows16[t0 / 16 + x] >= 0;
      return (bool)__builtin_amdgcn_readfirstlane(yes);
    };
    auto load = [&](int t0, auto part) {
      if (is_full(t0)) part(t0, true);
      else part(t0, false);
    };
    int t0 = ks * T;
    const bool work = !idle && t0 < keys;
    if (work) {
      load(t0, load_k);
      load(t0, load_v);
    }
    sh.time[tid] = key_time;
    if constexpr (Q8)
#pragma unroll
      for (int x = 0; x < 4; x++)
        if (x < sp.hg) {
          sh.scales[0][x][tid] = key_ks[x] * kNegLog2e;
          sh.scales[1][x][tid] = key_vs[x];
        }
    // The part of rab_pos that the block's pairs can reach: entry x belongs to
    // x = key - k0 + deep - depth; copy c starts c entries later, so that any
    // four in a row are one aligned read of some copy.
    if (windowed) {
      const int base = N - 1 + k0 - n_b - deep;
#pragma unroll
      for (int e = 0; e < kWindow / kThreads; e++) {
        const int x = tid + e * kThreads;
        if (x > kBlock + 2 + deep - flat) continue;
        const float v = a.ja.rab_pos[max(0, min(2 * N - 2, base + x))] * kNegLog2e;
#pragma unroll
        for (int c = 0; c < 4; c++)
          if (x >= c) sh.window[c][x - c] = v;
      }
    }
    // What the rows' times have in common with those of this wave's 64 keys:
    // |dt| is monotone in the key's time on either side of 0.
    {
      const int64_t lo = wave_extreme64<false>(ok ? key_time : INT64_MAX);
      const int64_t hi = wave_extreme64<true>(ok ? key_time : INT64_MIN);
      bool one = true, near = true;
      for (int i = lane; lo <= hi && i < rows; i += 64) {
        const int64_t x = sh.row_time[i] - lo, y = sh.row_time[i] - hi;
        const int bx = time_bucket64(x, a.ja.num_buckets);
        const int by = time_bucket64(y, a.ja.num_buckets);
        one &= bx == by && ((x >= 0) == (y >= 0) || bx == 0);
        near &= x == (int)x && y == (int)y && (int)x != INT32_MIN && (int)y != INT32_MIN;
        sh.uniform[wave][i] = sh.rtime[by];
      }
      const bool all_one = __ballot(!one) == 0, all_near = __ballot(!near) == 0;
      if (lane == 0) sh.times[wave] = all_one ? kTimesOne : all_near ? kTimesNear : kTimesAny;
    }
    __syncthreads();
    if (k0 + kBlock < to) fetch(k0 + kBlock, next_page);
    if (!work) continue;
    for (; t0 < keys; t0 += ks_count * T) {
      const int next = t0 + ks_count * T;
      const bool full = is_full(t0);
      const int times = __builtin_amdgcn_readfirstlane(sh.times[t0 / 64]);
#pragma unroll
      for (int s = 0; s < NS; s++) {
        f32x4 sc[R][2];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const int t = 2 * s + x;
#pragma unroll
          for (int m = 0; m < R; m++) sc[m][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int st = 0; st < KS; st++) {
            bf16x8 kf;
            if constexpr (Q8) kf = widen<KIND>(kw[t][2 * st], kw[t][2 * st + 1]);
            else kf = as_bf16x8(u32x4{kw[t][4 * st], kw[t][4 * st + 1], kw[t][4 * st + 2],
                                      kw[t][4 * st + 3]});
#pragma unroll
            for (int m = 0; m < R; m++) sc[m][x] = mfma16x16x32(kf, q[m][st], sc[m][x]);
          }
        }
        if (s == NS - 1 && next < keys) load(next, load_k);
        bf16x8 p[R];
#pragma unroll
        for (int m = 0; m < R; m++) {
          const int row = w0 + 16 * m + r;
          float w[8];
#pragma unroll
          for (int x = 0; x < 2; x++) {
            const int at = t0 + GK * g + 8 * s + 4 * x;
            // -log2(e) times the bias of four pairs
            f32x4 bv;
            if (windowed) {
              bv = *reinterpret_cast<const f32x4*>(
                  &sh.window[shift[m] & 3][(shift[m] & ~3) + at]);
            } else {
#pragma unroll
              for (int i = 0; i < 4; i++)
                bv[i] =
                    a.ja.rab_pos[max(0, N - 1 + k0 + at + i - n_b - depth[m])] * kNegLog2e;
            }
            if (times == kTimesOne) {
              bv += sh.uniform[t0 / 64][row];
            } else {
              const int64_t rt = sh.row_time[row];
#pragma unroll
              for (int i = 0; i < 4; i++) {
                int bucket;
                if (times == kTimesNear) {
                  const int dt = (int)rt - (int)sh.time[at + i];
                  bucket = min(31 - __clz(max(1, max(dt, -dt))), a.ja.num_buckets - 1);
                } else {
                  bucket = time_bucket64(rt - sh.time[at + i], a.ja.num_buckets);
                }
                bv[i] += sh.rtime[bucket];
              }
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
              float y;
              if constexpr (Q8) y = fmaf(sc[m][x][i], sh.scales[0][hh][at + i], bv[i]);
              else y = fmaf(sc[m][x][i], kNegLog2e, bv[i]);
              y *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y));
              if constexpr (Q8) y *= sh.scales[1][hh][at + i];
              w[4 * x + i] = y;
            }
          }
          if (!full) {
            const int left = left_of(t0) - 8 * s;
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = i < left ? w[i] : 0.0f;
          }
          p[m] = as_bf16x8(pack_bf16x8(w));
        }
#pragma unroll
        for (int c = 0; c < NC; c++) {
          bf16x8 vf;
          if constexpr (Q8) vf = widen<KIND>(vw[c][2 * s], vw[c][2 * s + 1]);
          else vf = as_bf16x8(u32x4{vw[c][0], vw[c][1], vw[c][2], vw[c][3]});
#pragma unroll
          for (int m = 0; m < R; m++) acc[m][c] = mfma16x16x32(p[m], vf, acc[m][c]);
        }
      }
      if (next < keys) load(next, load_v);
    }
  }

  // The waves of a head and rows add up, in order.
  for (int x = 1; x < ks_count; x++) {
    __syncthreads();
    float* space = sums + (wave % (4 / ks_count)) * (16 * R * DV);
    if (ks == x) {
#pragma unroll
      for (int m = 0; m < R; m++)
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            space[(16 * m + 4 * g + i) * DV + 16 * c + r] = acc[m][c][i];
    }
    __syncthreads();
    if (ks == 0) {
#pragma unroll
      for (int m = 0; m < R; m++)
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            acc[m][c][i] += space[(16 * m + 4 * g + i) * DV + 16 * c + r];
    }
  }
  if (ks != 0) return;
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int row = w0 + 16 * m + 4 * g + i;
      if (row >= rows) continue;
      float* dst = sp.part + (((int64_t)item * a.ja.total_tokens + o + r0 + row) * H + head) * DV + r;
#pragma unroll
      for (int c = 0; c < NC; c++) dst[16 * c] = acc[m][c][i];
    }
}

// The launch for one kind of cache.
template <int KIND>
hipError_t launch(const TreeArgs& a, const TreeSplit& sp, hipStream_t s) {
  const int64_t units = (int64_t)a.ja.num_seqs * sp.chunks * (a.ja.num_heads / sp.hg);
  const dim3 grid((unsigned)((units + 7) / 8 * 8 * sp.row_blocks));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, sp);
    return hipGetLastError();
  };
#define HSTU_TREE_R(DQK, DV)                                        \
  if (sp.rows == 16) return go(attn_tree_kernel<KIND, DQK, DV, 1>); \
  return go(attn_tree_kernel<KIND, DQK, DV, 2>);
#define HSTU_TREE_DV(DQK)                       \
  if (a.d_v == 32) { HSTU_TREE_R(DQK, 32) }     \
  if (a.d_v == 64) { HSTU_TREE_R(DQK, 64) }     \
  HSTU_TREE_R(DQK, 128)
  if (a.d_qk == 32) { HSTU_TREE_DV(32) }
  if (a.d_qk == 64) { HSTU_TREE_DV(64) }
  HSTU_TREE_DV(128)
#undef HSTU_TREE_DV
#undef HSTU_TREE_R
}

hipError_t launch_bf16(const TreeArgs& a, const TreeSplit& sp, hipStream_t s);
hipError_t launch_e4m3(const TreeArgs& a, const TreeSplit& sp, hipStream_t s);
hipError_t launch_int8(const TreeArgs& a, const TreeSplit& sp, hipStream_t s);

}  // namespace tree
}  // namespace hstu

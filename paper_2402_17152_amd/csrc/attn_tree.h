// Attention of drafted tokens over the paged cache (include/hstu.h): the kernels of
// the cached keys, instantiated for one kind of cache in each of
// attn_tree_{bf16,e4m3,int8}.hip.  Weights are pointwise, so sums over parts of the
// keys simply add up: the kernels leave fp32 partial outputs, and another one
// (attn_tree.hip) adds them to the drafted keys' part.
//
// A workgroup of four waves takes some drafted rows of one user and a chunk of the
// cached keys, in tiles of T keys.
//
//   S^T = K Q^T on 16x16x32 matrix instructions, keys in the rows: lane
//   (row r = l % 16, group g = l / 16) of K's operand t reads key T/4 (r/4) + 4t +
//   r%4, so that accumulator t leaves keys T/4 g + 4 t + 0..3 of query row l % 16
//   in lane l.  That is the layout of the weights as the left operand of O = P V,
//   whose contraction runs over keys T/4 g + 8 s + 0..7: no exchange between lanes.
//   The cache holds V transposed, so its operand (T/4 keys of a feature) is 16 bytes
//   in a row.  Column r of V's operand c is feature d_v / 16 r + c: a lane's outputs
//   of a row lie side by side.
//
// Codes of 8 bits are exact in bf16; a key's scales multiply the score and the
// weight.  Everything is kept times -log2(e): y = -log2(e) s gives SiLU(s) =
// s / (1 + 2^y) with one exp2, one reciprocal and one product, and the factor comes
// off at the end.  For 256 keys at a time the workgroup holds in LDS the pages, the
// scales, the times and the window of rab_pos that its rows can reach; where the
// time bucket of a row is the same for all keys of a tile (most of a long history:
// buckets are powers of two) the time bias is one number.
//
// Up to 32 rows, attn_tree_few_kernel: what counts is how fast the cache streams in.
// A wave takes a head (and a share of the keys) and loads the operands straight into
// registers, a tile ahead.  Lanes that are neighbours read different rows then, 16
// bytes each, and the vector cache takes one such access a clock: 9.8 TB/s, above
// the memory's rate but not by enough to load anything twice.
// More rows, attn_tree_many_kernel: the four waves take 16 R rows each of one head (R
// 1 up to 64 rows, so that a tree of 64 fills all four)
// and share its tiles through LDS, loaded in rows of 64 bytes and more (a fourth of
// the accesses; loaded by each wave for itself, 16 x 1024 rows over 1024-2048 keys
// spent 183 of 230 us on them).
//
// Measured, both kernels alone: 16 x 1 token over up to 1024 (bf16, 4 heads of 64) 9 us;
// 32 x 16 nodes over up to 4000 (e4m3, 8 heads of 64) 25 us, 3.7 TB/s; 1 x 7 nodes
// over 60001 (int8, 2 heads of 128) 17 us; 16 x 64 nodes over up to 8000 (e4m3, 4
// heads of 128) 52 us, a third of the time in vector instructions; 16 x 1000
// candidates over up to 2048 (bf16, 4 heads of 128) 115-122 us, 400 TFLOP/s.
#pragma once

#include <type_traits>

#include "kernels.h"

namespace hstu {
namespace tree {

constexpr int kThreads = 256;
constexpr int kBlock = 256;       // keys whose scales, times and pages are held
constexpr int kWindow = 512;      // entries of rab_pos that are held at most
constexpr float kNegLog2e = -kLog2e;

// An entry of the bias tables.  The lowest ones, the type's lowest value and -inf among
// them, are masks: held this far from the end of the range their sums and products
// stay finite, and SiLU is 0 there.
__device__ __forceinline__ float entry(float x) { return x < -6e37f ? -6e37f : x; }

// What is known of 64 keys: each row's time bucket is the same for all; the time
// differences fit 32 bits; all of the first, the second 32 keys are there.
enum { kOneBucket = 1, kNear = 2, kWhole = 4 };

// What the waves of a workgroup know of kBlock keys; HG: heads, ROWS: drafted rows,
// WIN: entries of rab_pos (kBlock and as many as the depths of the rows can differ).
template <int HG, int ROWS, int WIN>
struct Keys {
  static constexpr int spread = WIN - kBlock;
  float scales[2][HG][kBlock];     // k (times -log2(e)) and v
  float window[4][WIN + 4];        // part of rab_pos (times -log2(e)), four shifted copies
  int time[2][kBlock];             // low and high words
  int64_t rows16[kBlock / 16];     // first cache row of 16 keys for head 0
  int left16[kBlock / 16];         // how many of them are there; of none, row 0 is read
  float uniform[4][ROWS];          // the rows' entry of rtime for 64 keys (kOneBucket)
  int about[4];                    // what is known of 64 keys
};

// What they know of the drafted rows.
template <int ROWS>
struct Rows {
  float rtime[256];                // rab_time, times -log2(e)
  int64_t time[ROWS];
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

// The same for the 64-bit values of the lanes with `on`; those of all lanes often
// have the same high word.
template <bool MAX>
__device__ __forceinline__ int64_t wave_extreme64(int64_t v, bool on) {
  const int none = MAX ? INT32_MIN : INT32_MAX;
  const int hi = on ? (int)(v >> 32) : none;
  const uint64_t lanes = __ballot(on);
  int top = __builtin_amdgcn_readlane(hi, lanes ? __builtin_ctzll(lanes) : 0);
  if (__ballot(on && hi != top)) top = wave_extreme<MAX>(hi);
  // the low words compare as unsigned numbers
  const int lo = wave_extreme<MAX>(on && hi == top ? (int)((uint32_t)v ^ 0x80000000u) : none);
  return (int64_t)top << 32 | (uint32_t)(lo ^ (int)0x80000000u);
}

// A workgroup's part of the work.
struct Part {
  int b, head0, hg;        // user, first head, heads
  int from, to;            // cached keys
  int64_t o;               // first drafted token of the user
  int r0, rows;            // drafted rows: r0 .. r0 + rows - 1 of the user's
  int n_b, cap, lg;        // cached tokens, room for them, log2 of the page size
  int deep;                // the largest depth that the window is for
  bool windowed;           // Keys::window holds all that the rows reach
};

// The user, heads and chunk of a workgroup; false: there are none.
__device__ __forceinline__ bool find_place(const TreeArgs& a, const TreeSplit& sp, Part* w) {
  // Workgroups go to the eight dies in turn: the row blocks of one chunk and
  // head group, which read the same keys, follow each other on one die.
  const int die = blockIdx.x % 8, turn = blockIdx.x / 8;
  const int rb = turn % sp.row_blocks;
  const int unit = turn / sp.row_blocks * 8 + die;
  const int hgs = a.ja.num_heads / sp.hg;
  const int item = unit / hgs % sp.chunks;
  w->b = unit / hgs / sp.chunks;
  if (w->b >= a.ja.num_seqs) return false;
  w->hg = sp.hg;
  w->head0 = unit % hgs * sp.hg;
  w->lg = a.c.lg_page;
  w->cap = a.c.max_pages << w->lg;
  w->from = item * sp.chunk_len;
  w->r0 = rb * sp.rows;
  return true;
}

// Its rows and keys; false: there is nothing to do.
__device__ __forceinline__ bool find_part(const TreeArgs& a, const TreeSplit& sp, Part* w) {
  w->o = a.ja.seq_offsets[w->b];
  const int64_t o1 = min(a.ja.seq_offsets[w->b + 1], a.ja.total_tokens);
  w->n_b = (int)max((int64_t)0, min(a.c.lengths[w->b], (int64_t)w->cap));
  const int L = (int)max((int64_t)0, min(o1 - w->o, (int64_t)a.max_draft));
  w->to = min(w->n_b, w->from + sp.chunk_len);
  w->rows = min(sp.rows, L - w->r0);
  return w->o >= 0 && w->r0 < L && (w->from < w->to || (sp.last && w->from == 0));
}

// What a thread knows of key k0 + its number, before it is in LDS.
template <int HG>
struct Ahead {
  int64_t page, time;
  float ks[HG], vs[HG], pos[kWindow / kThreads];
};

__device__ __forceinline__ int fetch_page(const TreeArgs& a, const Part& w, int k0) {
  const int j = k0 + (int)threadIdx.x;
  return j < w.cap ? a.c.page_table[(int64_t)w.b * a.c.max_pages + (j >> w.lg)] : -1;
}

__device__ __forceinline__ int64_t valid_page(const TreeArgs& a, const Part& w, int k0, int page) {
  return k0 + (int)threadIdx.x < w.to && page < a.c.num_pages ? page : -1;
}

template <bool Q8, int HG>
__device__ __forceinline__ void fetch(const TreeArgs& a, const Part& w, int k0, int page,
                                      Ahead<HG>* h) {
  const int place = (k0 + (int)threadIdx.x) & ((1 << w.lg) - 1);
  h->page = valid_page(a, w, k0, page);
  h->time = h->page >= 0 ? a.c.tc[(h->page << w.lg) + place] : 0;
  if constexpr (Q8)
#pragma unroll
    for (int x = 0; x < HG; x++) {
      const int64_t at = ((h->page * a.ja.num_heads + w.head0 + x) << w.lg) + place;
      const bool on = h->page >= 0 && x < w.hg;
      h->ks[x] = on ? a.c.k_scale[at] : 0.0f;
      h->vs[x] = on ? a.c.v_scale[at] : 0.0f;
    }
}

// The part of rab_pos that the pairs of a block can reach: entry x belongs to
// x = key - k0 + deep - depth.
template <int HG>
__device__ __forceinline__ void fetch_pos(const TreeArgs& a, const Part& w, int k0, Ahead<HG>* h) {
  const int N = a.ja.max_seq_len, base = N - 1 + k0 - w.n_b - w.deep + (int)threadIdx.x;
  if (w.windowed)
#pragma unroll
    for (int e = 0; e < kWindow / kThreads; e++)
      h->pos[e] = a.ja.rab_pos[max(0, min(2 * N - 2, base + e * kThreads))];
}

// Where the rows of a block's keys are.
template <typename K>
__device__ __forceinline__ void put_rows(const TreeArgs& a, const Part& w, int k0, int64_t page,
                                         K* k) {
  const uint64_t there = __ballot(page >= 0);
  const int tid = threadIdx.x;
  if (tid % 16 == 0) {
    // keys of 16 lie on one page, the last ones may be missing
    k->rows16[tid / 16] =
        page >= 0 ? ((page * a.ja.num_heads) << w.lg) + ((k0 + tid) & ((1 << w.lg) - 1)) : 0;
    k->left16[tid / 16] = __popc((uint32_t)(there >> (tid % 64)) & 0xffffu);
  }
}

// The rest of what is known of them.
template <bool Q8, int HG, int ROWS, int WIN>
__device__ __forceinline__ void put_keys(const TreeArgs& a, const Part& w, const Rows<ROWS>& rows,
                                         const Ahead<HG>& h, Keys<HG, ROWS, WIN>* k) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  k->time[0][tid] = (int)h.time;
  k->time[1][tid] = (int)(h.time >> 32);
  if constexpr (Q8)
#pragma unroll
    for (int x = 0; x < HG; x++)
      if (x < w.hg) {
        k->scales[0][x][tid] = h.ks[x] * kNegLog2e;
        k->scales[1][x][tid] = h.vs[x];
      }
  // Copy c of the window starts c entries later: any four in a row are one
  // aligned read of some copy.
  if (w.windowed)
#pragma unroll
    for (int e = 0; e < kWindow / kThreads; e++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        const int x = tid + e * kThreads - c;
        if (x >= 0 && x < WIN) k->window[c][x] = entry(h.pos[e]) * kNegLog2e;
      }
  // What the rows' times have in common with those of this wave's 64 keys:
  // |dt| is monotone in the key's time on either side of 0.
  const bool ok = h.page >= 0;
  const uint64_t there = __ballot(ok);
  const int64_t lo = wave_extreme64<false>(h.time, ok);
  const int64_t hi = wave_extreme64<true>(h.time, ok);
  bool one = true, near = true;
  for (int i = lane; there && i < w.rows; i += 64) {
    const int64_t x = rows.time[i] - lo, y = rows.time[i] - hi;
    const int bx = time_bucket64(x, a.ja.num_buckets);
    const int by = time_bucket64(y, a.ja.num_buckets);
    one &= bx == by && ((x >= 0) == (y >= 0) || bx == 0);
    near &= x == (int)x && y == (int)y && (int)x != INT32_MIN && (int)y != INT32_MIN;
    k->uniform[wave][i] = rows.rtime[by];
  }
  const int all_one = __ballot(!one) == 0 ? kOneBucket : 0;
  const int all_near = __ballot(!near) == 0 ? kNear : 0;
  const int whole =
      ((uint32_t)there == ~0u ? kWhole : 0) | (there >> 32 == 0xffffffffu ? 2 * kWhole : 0);
  if (lane == 0) k->about[wave] = all_one | all_near | whole;
}

// The depths that the window covers, where max_draft says enough: it then does not
// wait for the depths themselves.
__device__ __forceinline__ bool bound_depths(const TreeArgs& a, Part* w) {
  w->windowed = a.max_draft <= kWindow - kBlock || !a.parents;
  w->deep = a.parents ? a.max_draft - 1 : 0;
  return w->windowed;
}

// Depths of this lane's rows w0 + 16 m + r (0 where there is none), and, where
// bound_depths() does not know them, the window's.  parent: of node `lane`.
// SMALL: max_draft is at most 64.
template <bool SMALL, int R>
__device__ __forceinline__ void find_depths(const TreeArgs& a, Part* w, int w0, int64_t parent,
                                            short2* node, int* depth) {
  const int lane = threadIdx.x % 64, r = lane % 16;
  const int nodes = w->r0 + w->rows;
#pragma unroll
  for (int m = 0; m < R; m++) depth[m] = 0;
  if (!a.parents) return;
  if (SMALL || nodes <= 64) {
    const int d = walk64(parent >= 0 && parent < lane ? (int)parent : -1);
#pragma unroll
    for (int m = 0; m < R; m++) {
      const int x = __shfl(d, (w->r0 + w0 + 16 * m + r) & 63, 64);
      if (w0 + 16 * m + r < w->rows) depth[m] = x;
    }
    if (!SMALL && !w->windowed) {  // depths below 64
      w->windowed = true;
      w->deep = 63;
    }
    return;
  }
  if constexpr (!SMALL) {
    walk(a.parents + w->o, nodes, node);
#pragma unroll
    for (int m = 0; m < R; m++)
      if (w0 + 16 * m + r < w->rows) depth[m] = node[w->r0 + w0 + 16 * m + r].y;
    if (!w->windowed) {
      int deep = 0, flat = kMaxDraft;
      for (int i = w->r0 + lane; i < nodes; i += 64) {
        deep = max(deep, (int)node[i].y);
        flat = min(flat, (int)node[i].y);
      }
      w->deep = wave_extreme<true>(deep);
      w->windowed = w->deep - wave_extreme<false>(flat) < kWindow - kBlock;
    }
  }
}

// Q as the right operand: rows w0 + 16 m + r, features in the order of feature().
template <int KIND, int DQK, int R>
__device__ __forceinline__ void load_q(const TreeArgs& a, const Part& w, int w0, int head,
                                       bf16x8 (&q)[R][DQK / 32]) {
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
#pragma unroll
  for (int m = 0; m < R; m++) {
    const int row = w0 + 16 * m + r;
    const uint16_t* src =
        (const uint16_t*)a.t.q + (w.o + w.r0 + row) * a.t.q_stride + (int64_t)head * DQK;
#pragma unroll
    for (int s = 0; s < DQK / 32; s++) {
      u32x4 v = zero_u32x4();
      if (row < w.rows) v = *reinterpret_cast<const u32x4*>(src + feature<KIND, DQK>(s, g));
      q[m][s] = as_bf16x8(v);
    }
  }
}

// -log2(e) times the bias of this lane's rows and the eight keys k0 + at ..
template <int R, int HG, int ROWS, int WIN>
__device__ __forceinline__ void find_bias(const TreeArgs& a, const Part& w, const Rows<ROWS>& rows,
                                          const Keys<HG, ROWS, WIN>& k, int about, int k0, int at, int w0,
                                          const int* depth, f32x4 (&bv)[R][2]) {
  const int r = threadIdx.x % 16;
  if (w.windowed && (about & kOneBucket)) {
#pragma unroll
    for (int m = 0; m < R; m++) {
      const float one = k.uniform[at / 64][w0 + 16 * m + r];
      const int shift = max(0, min(w.deep - depth[m], WIN - kBlock - 1));
      const float* win = &k.window[shift & 3][(shift & ~3) + at];
#pragma unroll
      for (int x = 0; x < 2; x++) bv[m][x] = *reinterpret_cast<const f32x4*>(win + 4 * x) + one;
    }
    return;
  }
  const int N = a.ja.max_seq_len;
#pragma unroll
  for (int m = 0; m < R; m++) {
    const int64_t rt = rows.time[w0 + 16 * m + r];
    const int shift = max(0, min(w.deep - depth[m], WIN - kBlock - 1));
    int bucket[8];
    if (about & kNear) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const int dt = (int)rt - k.time[0][at + i];
        bucket[i] = min(31 - __clz(max(1, max(dt, -dt))), a.ja.num_buckets - 1);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const int64_t kt = (int64_t)k.time[1][at + i] << 32 | (uint32_t)k.time[0][at + i];
        bucket[i] = time_bucket64(rt - kt, a.ja.num_buckets);
      }
    }
    float pos[8];
    if (w.windowed) {
#pragma unroll
      for (int x = 0; x < 2; x++) {
        const f32x4 v =
            *reinterpret_cast<const f32x4*>(&k.window[shift & 3][(shift & ~3) + at + 4 * x]);
#pragma unroll
        for (int i = 0; i < 4; i++) pos[4 * x + i] = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        pos[i] = entry(a.ja.rab_pos[max(0, N - 1 + k0 + at + i - w.n_b - depth[m])]) * kNegLog2e;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) bv[m][i / 4][i % 4] = pos[i] + rows.rtime[bucket[i]];
  }
}

// The weights (times -log2(e)) of a row and eight keys as the left operand of P V:
// scores sc, their bias, the keys' scales; keys from `left` on count nothing.
template <bool Q8>
__device__ __forceinline__ bf16x8 find_weights(const f32x4* sc, const f32x4* bv, const f32x4* kf,
                                               const f32x4* vf, bool whole, int left) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    float y;
    if constexpr (Q8) y = fmaf(sc[i / 4][i % 4], kf[i / 4][i % 4], bv[i / 4][i % 4]);
    else y = fmaf(sc[i / 4][i % 4], kNegLog2e, bv[i / 4][i % 4]);
    y *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y));
    if constexpr (Q8) y *= vf[i / 4][i % 4];
    w[i] = y;
  }
  if (!whole)
#pragma unroll
    for (int i = 0; i < 8; i++) w[i] = i < left ? w[i] : 0.0f;
  return as_bf16x8(pack_bf16x8(w));
}

// 16 bytes of codes with those behind the first `left` zeroed.
template <int CB>
__device__ __forceinline__ u32x4 cut(u32x4 v, int left) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int keep = (left * CB - 4 * e) * 8;  // bits
    v[e] = keep >= 32 ? v[e] : keep <= 0 ? 0u : v[e] & ((1u << keep) - 1u);
  }
  return v;
}

// Partial outputs of a wave's rows and head.
template <int DV, int R>
__device__ __forceinline__ void put_part(const TreeArgs& a, const TreeSplit& sp, const Part& w,
                                         int w0, int head, const f32x4 (&acc)[R][DV / 16]) {
  constexpr int NC = DV / 16;
  typedef float fv __attribute__((ext_vector_type(NC < 4 ? NC : 4)));
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int64_t item = w.from / sp.chunk_len;
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int row = w0 + 16 * m + 4 * g + i;
      if (row >= w.rows) continue;
      float* dst = sp.part + ((item * a.ja.total_tokens + w.o + w.r0 + row) * a.ja.num_heads +
                              head) * DV + NC * r;
#pragma unroll
      for (int c = 0; c < NC; c += 4) {
        fv x;
#pragma unroll
        for (int e = 0; e < NC && e < 4; e++) x[e] = acc[m][c + e][i];
        *reinterpret_cast<fv*>(dst + c) = x;
      }
    }
}

// The outputs themselves, where all of a row's cached keys are summed up and no node
// sees another one: with the row's own key.  The dot product is taken in the layout
// of load_q (32 features a lane), the value row by row.
template <int KIND, int DQK, int DV, int R>
__device__ __forceinline__ void put_out(const TreeArgs& a, const Part& w, int w0, int head,
                                        const bf16x8 (&q)[R][DQK / 32],
                                        const f32x4 (&acc)[R][DV / 16]) {
  constexpr int NC = DV / 16;
  typedef __bf16 bv __attribute__((ext_vector_type(NC)));
  const int lane = threadIdx.x % 64, r = lane % 16, g = lane / 16;
  const int N = a.ja.max_seq_len;
  const float bias = entry(a.ja.rab_pos[N - 1]) + entry(a.ja.rab_time[0]);  // of a token and itself
  const float inv = 1.0f / (float)N;
#pragma unroll
  for (int m = 0; m < R; m++) {
    const int own = min(w0 + 16 * m + r, w.rows - 1);
    const uint16_t* kr =
        (const uint16_t*)a.t.k + (w.o + w.r0 + own) * a.t.k_stride + (int64_t)head * DQK;
    bv v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int64_t t = w.o + w.r0 + min(w0 + 16 * m + 4 * g + i, w.rows - 1);
      v[i] = *reinterpret_cast<const bv*>((const uint16_t*)a.t.v + t * a.t.v_stride +
                                          (int64_t)head * DV + NC * r);
    }
    float s = 0.0f;
#pragma unroll
    for (int st = 0; st < DQK / 32; st++) {
      const bf16x8 k8 =
          as_bf16x8(*reinterpret_cast<const u32x4*>(kr + feature<KIND, DQK>(st, g)));
#pragma unroll
      for (int e = 0; e < 8; e++) s = fmaf((float)q[m][st][e], (float)k8[e], s);
    }
    s += __shfl_xor(s, 16, 64);
    s += __shfl_xor(s, 32, 64);
    s += bias;
    s *= sigmoid_fast(s);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float p = __shfl(s, 4 * g + i, 64);
      const int row = w0 + 16 * m + 4 * g + i;
      if (row >= w.rows) continue;
      bv x;
#pragma unroll
      for (int c = 0; c < NC; c++)  // the weights' factor -log2(e) comes off
        x[c] = (__bf16)(fmaf(p, (float)v[i][c], acc[m][c][i] * -0.6931471805599453f) * inv);
      *reinterpret_cast<bv*>((uint16_t*)a.out +
                             ((w.o + w.r0 + row) * a.ja.num_heads + head) * DV + NC * r) = x;
    }
  }
}

// H4: the four waves have a head each, else they share heads and keys as sp.hg says.
template <int KIND, int DQK, int DV, int R, bool H4>
__global__ __launch_bounds__(kThreads, 2) void attn_tree_few_kernel(const TreeArgs a,
                                                                    const TreeSplit sp) {
  constexpr bool Q8 = KIND != kCacheBf16;     // quantised
  constexpr int CB = Q8 ? 1 : 2;              // bytes of a code
  constexpr int T = Q8 ? 64 : 32;             // keys of a tile: 16 bytes of a feature per lane
  constexpr int GK = T / 4;                   // of a lane group
  constexpr int NT = T / 16, NS = T / 32;     // operands of K, contraction steps of P V
  constexpr int KW = DQK * CB / 16;           // words of a K row a lane reads
  constexpr int KS = DQK / 32, NC = DV / 16;  // contraction steps of K Q^T, column tiles
  // Tiles a wave has under way: the compute units' share of the memory's latency is
  // 43 KB; two tiles where the registers hold them.
  constexpr int P = H4 && R == 1 && DQK + DV <= 128 ? 2 : 1;
  using Kb = Keys<4, 16 * R, kBlock + 32>;
  __shared__ __attribute__((aligned(16))) union {
    Kb kb[2];
    float sums[2 * 16 * R * DV];
  } sh;
  __shared__ Rows<16 * R> rs;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  Part w;
  if (!find_place(a, sp, &w)) return;
  const int first_page = fetch_page(a, w, w.from);
  if (!find_part(a, sp, &w)) return;
  const int lg = w.lg;
  // A wave's head and share of the keys: tile j is tile j % turns of its share of
  // block j / turns.
  const int hg = H4 ? 4 : sp.hg, ks_count = 4 / hg, hh = wave % hg, ks = wave / hg;
  const int turns = kBlock / T / ks_count;
  const int head = w.head0 + hh;
  const int r = lane % 16, g = lane / 16;
  u32x4 kw[P][NT][(KW + 3) / 4];
  u32x4 vw[P][NC];
  // The loads of a tile: always the same number, of rows that exist, so that a
  // wait for one of them waits for nothing behind it.
  auto load_k = [&](int j, int set) {
    // operand t takes row at + 4 t + r % 4
    const int at = (j % turns * ks_count + ks) * T + GK * (r / 4);
    const char* src = (const char*)a.c.kc + (sh.kb[j / turns % 2].rows16[at / 16] +
                                             ((int64_t)head << lg) + at % 16 + r % 4) * (DQK * CB);
#pragma unroll
    for (int t = 0; t < NT; t++) {
      if constexpr (KW == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(src + 4 * t * DQK * CB + 8 * g);
        kw[set][t][0][0] = v.x;
        kw[set][t][0][1] = v.y;
      } else {
#pragma unroll
        for (int u = 0; u < KW / 4; u++)
          kw[set][t][u] =
              *reinterpret_cast<const u32x4*>(src + 4 * t * DQK * CB + 64 * u + 16 * g);
      }
    }
  };
  auto load_v = [&](int j, int set) {
    const int at = (j % turns * ks_count + ks) * T + GK * g;
    const int64_t row = sh.kb[j / turns % 2].rows16[at / 16];
    const int place = (int)(row & ((1 << lg) - 1)) + at % 16;
    const char* src =
        (const char*)a.c.vc + (((((row >> lg) + head) * DV + NC * r) << lg) + place) * CB;
#pragma unroll
    for (int c = 0; c < NC; c++)
      vw[set][c] = *reinterpret_cast<const u32x4*>(src + ((int64_t)(c * CB) << lg));
  };
  // What the workgroup needs once is asked for first, then the first tiles: loads
  // come back in order, and the few small ones should not wait for the many.
  Ahead<4> h;
  fetch<Q8>(a, w, w.from, first_page, &h);
  bound_depths(a, &w);  // there are at most 32 drafted tokens
  fetch_pos(a, w, w.from, &h);
  bf16x8 q[R][KS];
  load_q<KIND, DQK, R>(a, w, 0, head, q);
  const float bucket_bias = tid < a.ja.num_buckets ? a.ja.rab_time[tid] : 0.0f;
  const int64_t row_time = tid < w.rows ? a.ja.timestamps[w.o + w.r0 + tid] : 0;
  const int64_t parent = a.parents && lane < w.r0 + w.rows ? a.parents[w.o + lane] : -1;
  put_rows(a, w, w.from, h.page, &sh.kb[0]);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < P; j++) {
    load_k(j, j);
    load_v(j, j);
  }
  f32x4 acc[R][NC];
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int c = 0; c < NC; c++) acc[m][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  rs.rtime[tid] = entry(bucket_bias) * kNegLog2e;
  if (tid < 16 * R) rs.time[tid] = row_time;
  int depth[R];
  find_depths<true, R>(a, &w, 0, parent, nullptr, depth);
  __syncthreads();  // rs
  put_keys<Q8>(a, w, rs, h, &sh.kb[0]);
  if (w.from + kBlock < w.to) {
    fetch<Q8>(a, w, w.from + kBlock, fetch_page(a, w, w.from + kBlock), &h);
    fetch_pos(a, w, w.from + kBlock, &h);
  }
  __syncthreads();

  auto tile = [&](int j, int k0, auto set_) {
    constexpr int set = decltype(set_)::value;
    const Kb& kb = sh.kb[j / turns % 2];
    const int t0 = (j % turns * ks_count + ks) * T;
    const int about = __builtin_amdgcn_readfirstlane(kb.about[t0 / 64]);
    const int all = Q8 ? 3 * kWhole : kWhole << (t0 / 32 % 2);
    const bool whole = (about & all) == all;  // all keys are there
    // the last loads are of a block that has not been looked at: not used
    const int next = min(j + P, (w.to - w.from + kBlock - 1) / kBlock * turns - 1);
    int left = GK;                            // keys of this lane's group
    if (!whole) {
      const int at = t0 + GK * g;
      left = max(0, min(GK, kb.left16[at / 16] - at % 16));
#pragma unroll
      for (int c = 0; c < NC; c++) vw[set][c] = cut<CB>(vw[set][c], left);
    }
    f32x4 bias[NS][R][2];
#pragma unroll
    for (int s = 0; s < NS; s++)
      find_bias<R>(a, w, rs, kb, about, k0, t0 + GK * g + 8 * s, 0, depth, bias[s]);
#pragma unroll
    for (int s = 0; s < NS; s++) {
      const int at = t0 + GK * g + 8 * s;
      f32x4 sc[R][2];
#pragma unroll
      for (int x = 0; x < 2; x++) {
        const int t = 2 * s + x;
#pragma unroll
        for (int m = 0; m < R; m++) sc[m][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int st = 0; st < KS; st++) {
          bf16x8 kf;
          if constexpr (Q8)
            kf = widen<KIND>(kw[set][t][st / 2][st % 2 * 2], kw[set][t][st / 2][st % 2 * 2 + 1]);
          else
            kf = as_bf16x8(kw[set][t][st]);
#pragma unroll
          for (int m = 0; m < R; m++) sc[m][x] = mfma16x16x32(kf, q[m][st], sc[m][x]);
        }
      }
      if (s == NS - 1) load_k(next, set);
      f32x4 kf[2], vf[2];
      if constexpr (Q8)
#pragma unroll
        for (int x = 0; x < 2; x++) {
          kf[x] = *reinterpret_cast<const f32x4*>(&kb.scales[0][hh][at + 4 * x]);
          vf[x] = *reinterpret_cast<const f32x4*>(&kb.scales[1][hh][at + 4 * x]);
        }
      bf16x8 p[R];
#pragma unroll
      for (int m = 0; m < R; m++)
        p[m] = find_weights<Q8>(sc[m], bias[s][m], kf, vf, whole, left - 8 * s);
#pragma unroll
      for (int c = 0; c < NC; c++) {
        bf16x8 vf8;
        if constexpr (Q8) vf8 = widen<KIND>(vw[set][c][2 * s], vw[set][c][2 * s + 1]);
        else vf8 = as_bf16x8(vw[set][c]);
#pragma unroll
        for (int m = 0; m < R; m++) acc[m][c] = mfma16x16x32(p[m], vf8, acc[m][c]);
      }
    }
    load_v(next, set);
  };
  for (int n = 0, k0 = w.from; k0 < w.to; n++, k0 += kBlock) {
    const int keys = min(kBlock, w.to - k0), k1 = k0 + kBlock;
    for (int i = 0; i < turns; i += P) {
      if (i == turns - P && k1 < w.to) {
        // the next block, before the first loads of its tiles
        __syncthreads();  // the block before is done with
        put_rows(a, w, k1, h.page, &sh.kb[(n + 1) % 2]);
        put_keys<Q8>(a, w, rs, h, &sh.kb[(n + 1) % 2]);
        __syncthreads();
        if (k1 + kBlock < w.to) {
          fetch<Q8>(a, w, k1 + kBlock, fetch_page(a, w, k1 + kBlock), &h);
          fetch_pos(a, w, k1 + kBlock, &h);
        }
      }
      if ((i * ks_count + ks) * T >= keys) break;
      tile(n * turns + i, k0, std::integral_constant<int, 0>{});
      if constexpr (P == 2)
        if ((i + 1) * T < keys) tile(n * turns + i + 1, k0, std::integral_constant<int, 1>{});
    }
  }

  // The waves of a head add up: half of them to the other half, in order.
  for (int half = ks_count / 2; half; half /= 2) {
    __syncthreads();
    float* space = sh.sums + ((ks % half) * hg + hh) * (16 * R * DV);
    if (ks >= half && ks < 2 * half) {
#pragma unroll
      for (int m = 0; m < R; m++)
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            space[(16 * m + 4 * g + i) * DV + 16 * c + r] = acc[m][c][i];
    }
    __syncthreads();
    if (ks < half) {
#pragma unroll
      for (int m = 0; m < R; m++)
#pragma unroll
        for (int c = 0; c < NC; c++)
#pragma unroll
          for (int i = 0; i < 4; i++)
            acc[m][c][i] += space[(16 * m + 4 * g + i) * DV + 16 * c + r];
    }
  }
  if (ks) return;
  if (sp.last) put_out<KIND, DQK, DV, R>(a, w, 0, head, q, acc);
  else put_part<DV, R>(a, sp, w, 0, head, acc);
}

// A tile of one head in LDS.  K: rows of keys, V: rows of features, in 16-byte
// pieces; a row's pieces are permuted so that the 16 rows that a quarter of a wave
// reads one piece of lie in 16 different sixteenths of the banks.
template <int KIND, int DQK, int DV>
struct Tile {
  static constexpr int CB = KIND != kCacheBf16 ? 1 : 2;
  static constexpr int T = 64 / CB, GK = T / 4;
  static constexpr int KP = DQK * CB / 16;  // pieces of a K row: 2, 4, 8 or 16
  static constexpr int kPieces = T * KP, vPieces = DV * 4;
  char k[kPieces * 16];
  char v[vPieces * 16];

  __device__ static int k_at(int key, int piece) {
    // rows key % 4 + GK (0..3) are read together, 16 / KP of them side by side in
    // the banks
    const int low = KP == 16 ? key & 3 : KP == 8 ? key >> 1 & 1 : 0;
    const int high = (key / GK) & 3;
    const int turn = (KP == 16 ? low | high << 2 : KP == 8 ? low | high << 1 : high) & (KP - 1);
    return (key * KP + (piece ^ turn)) * 16;
  }
  // Column r of operand c; feature DV / 16 r + c.
  __device__ static int v_at(int r, int c, int piece) {
    return ((16 * c + r) * 4 + (piece ^ (r >> 2 & 3))) * 16;
  }
};

template <int KIND, int DQK, int DV, int R>
__global__ __launch_bounds__(kThreads, 2) void attn_tree_many_kernel(const TreeArgs a,
                                                                     const TreeSplit sp) {
  using Tl = Tile<KIND, DQK, DV>;
  constexpr bool Q8 = KIND != kCacheBf16;
  constexpr int CB = Tl::CB, T = Tl::T, GK = Tl::GK, KP = Tl::KP;
  constexpr int NS = T / 32, KS = DQK / 32, NC = DV / 16;
  constexpr int KL = (Tl::kPieces + kThreads - 1) / kThreads;  // pieces a thread loads
  constexpr int VL = (Tl::vPieces + kThreads - 1) / kThreads;
  constexpr int TB = kBlock / T;                               // tiles of a block
  // Tiles under way: two where the registers hold them.
  constexpr int P = R == 1 ? 2 : 1;
  using Kb = Keys<1, 64 * R, R == 1 ? kBlock + 64 : kWindow>;
  __shared__ __attribute__((aligned(16))) Kb kb[2];
  __shared__ __attribute__((aligned(16))) Tl tiles[2];
  __shared__ Rows<64 * R> rs;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  Part w;
  if (!find_place(a, sp, &w)) return;
  const int first_page = fetch_page(a, w, w.from);
  if (!find_part(a, sp, &w)) return;
  const int lg = w.lg, head = w.head0;
  Ahead<1> h;
  fetch<Q8>(a, w, w.from, first_page, &h);
  if (bound_depths(a, &w)) fetch_pos(a, w, w.from, &h);
  const int w0 = wave * 16 * R;  // the wave's first row within the workgroup's
  const bool idle = w0 >= w.rows;
  const int r = lane % 16, g = lane / 16;
  bf16x8 q[R][KS];
  load_q<KIND, DQK, R>(a, w, w0, head, q);
  f32x4 acc[R][NC];
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int c = 0; c < NC; c++) acc[m][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const float bucket_bias = tid < a.ja.num_buckets ? a.ja.rab_time[tid] : 0.0f;
  const int64_t row_time = tid < w.rows ? a.ja.timestamps[w.o + w.r0 + tid] : 0;
  const int64_t parent = a.parents && lane < w.r0 + w.rows ? a.parents[w.o + lane] : -1;
  rs.rtime[tid] = entry(bucket_bias) * kNegLog2e;
  if (tid < 64 * R) rs.time[tid] = row_time;
  // Tile j of the chunk: loads into one of P sets of registers, then into LDS.
  const int count = (w.to - w.from + T - 1) / T;
  u32x4 kr[P][KL], vr[P][VL];
  auto load = [&](int j, int set) {
    const Kb& k = kb[j / TB % 2];
    const int t0 = j % TB * T;
#pragma unroll
    for (int e = 0; e < KL; e++) {
      const int x = tid + e * kThreads, at = t0 + x / KP;
      if (Tl::kPieces % kThreads && x >= Tl::kPieces) break;
      kr[set][e] = *reinterpret_cast<const u32x4*>(
          (const char*)a.c.kc +
          (k.rows16[at / 16] + ((int64_t)head << lg) + at % 16) * (DQK * CB) + x % KP * 16);
    }
#pragma unroll
    for (int e = 0; e < VL; e++) {
      const int x = tid + e * kThreads, at = t0 + GK * (x % 4);
      if (Tl::vPieces % kThreads && x >= Tl::vPieces) break;
      const int64_t row = k.rows16[at / 16];
      const int place = (int)(row & ((1 << lg) - 1)) + at % 16;
      vr[set][e] = *reinterpret_cast<const u32x4*>(
          (const char*)a.c.vc + (((((row >> lg) + head) * DV + x / 4) << lg) + place) * CB);
    }
  };
  auto is_whole = [&](int j) {
    const int t0 = j % TB * T, all = Q8 ? 3 * kWhole : kWhole << (t0 / 32 % 2);
    const int about = __builtin_amdgcn_readfirstlane(kb[j / TB % 2].about[t0 / 64]);
    return (about & all) == all;
  };
  auto store = [&](int j, int set) {
    Tl& tl = tiles[j % 2];
#pragma unroll
    for (int e = 0; e < KL; e++) {
      const int x = tid + e * kThreads;
      if (Tl::kPieces % kThreads && x >= Tl::kPieces) break;
      *reinterpret_cast<u32x4*>(tl.k + Tl::k_at(x / KP, x % KP)) = kr[set][e];
    }
    if (!is_whole(j)) {  // codes behind the last key count as zeros
      const Kb& k = kb[j / TB % 2];
      const int at = j % TB * T + GK * (tid % 4);
      const int left = max(0, min(GK, k.left16[at / 16] - at % 16));
#pragma unroll
      for (int e = 0; e < VL; e++) vr[set][e] = cut<CB>(vr[set][e], left);
    }
#pragma unroll
    for (int e = 0; e < VL; e++) {
      const int x = tid + e * kThreads;
      if (Tl::vPieces % kThreads && x >= Tl::vPieces) break;
      *reinterpret_cast<u32x4*>(tl.v + Tl::v_at(x / 4 / NC, x / 4 % NC, x % 4)) = vr[set][e];
    }
  };

  int depth[R];
  static_assert(sizeof(tiles) >= kMaxDraft * sizeof(short2), "the depths fit where the tiles go");
  const bool known = w.windowed;
  find_depths<R == 1, R>(a, &w, w0, parent, reinterpret_cast<short2*>(tiles), depth);
  if (!known) fetch_pos(a, w, w.from, &h);
  put_rows(a, w, w.from, h.page, &kb[0]);
  __syncthreads();
  if (count > 0) {
    load(0, 0);
    put_keys<Q8>(a, w, rs, h, &kb[0]);
    if (w.from + kBlock < w.to) {
      fetch<Q8>(a, w, w.from + kBlock, fetch_page(a, w, w.from + kBlock), &h);
      fetch_pos(a, w, w.from + kBlock, &h);
    }
    __syncthreads();
    store(0, 0);
    if (P == 2 && count > 1) load(1, 1);
    __syncthreads();
  }
  auto turn = [&](int j, auto odd) {
    // P tiles ahead, into the registers of the tile that is in LDS by now
    constexpr int set = P == 2 ? decltype(odd)::value : 0;
    if (j + P < count) load(j + P, set);
    // the next block's keys, before their first tile's loads
    const int k1 = w.from + (j / TB + 1) * kBlock;
    if (j % TB == TB - P - 2 && k1 < w.to) {
      put_rows(a, w, k1, h.page, &kb[(j / TB + 1) % 2]);
      put_keys<Q8>(a, w, rs, h, &kb[(j / TB + 1) % 2]);
      if (k1 + kBlock < w.to) {
        fetch<Q8>(a, w, k1 + kBlock, fetch_page(a, w, k1 + kBlock), &h);
        fetch_pos(a, w, k1 + kBlock, &h);
      }
    }
    if (!idle) {
      const Kb& k = kb[j / TB % 2];
      const Tl& tl = tiles[j % 2];
      const int t0 = j % TB * T, k0 = w.from + j / TB * kBlock;
      const int about = __builtin_amdgcn_readfirstlane(k.about[t0 / 64]);
      const bool whole = is_whole(j);
      int left = GK;  // keys of this lane's group
      if (!whole) {
        const int at = t0 + GK * g;
        left = max(0, min(GK, k.left16[at / 16] - at % 16));
      }
      f32x4 bias[NS][R][2];
#pragma unroll
      for (int s = 0; s < NS; s++)
        find_bias<R>(a, w, rs, k, about, k0, t0 + GK * g + 8 * s, w0, depth, bias[s]);
#pragma unroll
      for (int s = 0; s < NS; s++) {
        const int at = t0 + GK * g + 8 * s;
        f32x4 sc[R][2];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const int t = 2 * s + x, key = GK * (r / 4) + 4 * t + r % 4;
#pragma unroll
          for (int m = 0; m < R; m++) sc[m][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
          auto step = [&](int st, bf16x8 kf) {
#pragma unroll
            for (int m = 0; m < R; m++) sc[m][x] = mfma16x16x32(kf, q[m][st], sc[m][x]);
          };
          if constexpr (Q8 && DQK == 32) {
            const uint2 c =
                *reinterpret_cast<const uint2*>(tl.k + Tl::k_at(key, g / 2) + 8 * (g % 2));
            step(0, widen<KIND>(c.x, c.y));
          } else {
#pragma unroll
            for (int u = 0; u < KP / 4; u++) {
              const u32x4 c = *reinterpret_cast<const u32x4*>(tl.k + Tl::k_at(key, 4 * u + g));
              if constexpr (Q8) {
                step(2 * u, widen<KIND>(c[0], c[1]));
                step(2 * u + 1, widen<KIND>(c[2], c[3]));
              } else {
                step(u, as_bf16x8(c));
              }
            }
          }
        }
        f32x4 kf[2], vf[2];
        if constexpr (Q8)
#pragma unroll
          for (int x = 0; x < 2; x++) {
            kf[x] = *reinterpret_cast<const f32x4*>(&k.scales[0][0][at + 4 * x]);
            vf[x] = *reinterpret_cast<const f32x4*>(&k.scales[1][0][at + 4 * x]);
          }
        bf16x8 p[R];
#pragma unroll
        for (int m = 0; m < R; m++)
          p[m] = find_weights<Q8>(sc[m], bias[s][m], kf, vf, whole, left - 8 * s);
#pragma unroll
        for (int c = 0; c < NC; c++) {
          bf16x8 v8;
          const char* src = tl.v + Tl::v_at(r, c, g);
          if constexpr (Q8) {
            const uint2 x = *reinterpret_cast<const uint2*>(src + 8 * s);
            v8 = widen<KIND>(x.x, x.y);
          } else {
            v8 = as_bf16x8(*reinterpret_cast<const u32x4*>(src));
          }
#pragma unroll
          for (int m = 0; m < R; m++) acc[m][c] = mfma16x16x32(p[m], v8, acc[m][c]);
        }
      }
    }
    if (j + 1 < count) store(j + 1, P == 2 ? 1 - set : 0);
    __syncthreads();
  };
  for (int j = 0; j < count; j += 2) {
    turn(j, std::integral_constant<int, 0>{});
    if (j + 1 < count) turn(j + 1, std::integral_constant<int, 1>{});
  }
  if (idle) return;
  if (sp.last) put_out<KIND, DQK, DV, R>(a, w, w0, head, q, acc);
  else put_part<DV, R>(a, sp, w, w0, head, acc);
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
#define HSTU_TREE_R(DQK, DV)                                             \
  if (sp.rows == 16)                                                     \
    return sp.hg == 4 ? go(attn_tree_few_kernel<KIND, DQK, DV, 1, true>)  \
                      : go(attn_tree_few_kernel<KIND, DQK, DV, 1, false>); \
  if (sp.rows == 32)                                                     \
    return sp.hg == 4 ? go(attn_tree_few_kernel<KIND, DQK, DV, 2, true>)  \
                      : go(attn_tree_few_kernel<KIND, DQK, DV, 2, false>); \
  if (sp.rows == 64) return go(attn_tree_many_kernel<KIND, DQK, DV, 1>); \
  return go(attn_tree_many_kernel<KIND, DQK, DV, 2>);
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

// Attention of drafted tokens over the paged cache (include/hstu.h): the kernel,
// instantiated for one kind of cache in each of attn_tree_{bf16,e4m3,int8}.hip.
//
// A workgroup of four waves takes 16 R drafted rows of one user, a chunk of the
// cached keys and `hg` heads; a wave takes one head and every (4 / hg)th tile of
// 64 keys.  Weights are pointwise, so partial sums over chunks simply add up.
//
//   S^T = K Q^T on 16x16x32 matrix instructions, keys in the rows: lane
//   (row r = l % 16, group g = l / 16) of K's operand t reads key 16 (r/4) + 4t +
//   r%4, so that accumulator t leaves keys 16 g + 4 t + 0..3 of query row l % 16
//   in lane l.  That is the layout of the weights as the left operand of O = P V,
//   whose contraction runs over keys 16 g + 8 s + 0..7: no exchange between lanes.
//   The cache holds V transposed, so its operand (keys 16 g .. 16 g + 15 of a
//   feature) is one load.  Nothing passes through LDS but what all heads share.
//
// Codes of 8 bits are exact in bf16; a key's scales multiply the score and the
// weight.  The bias of 256 keys, the same for all heads, is computed once per
// workgroup into LDS, with the keys' scales and pages.
//
// The drafted keys are a part of their own: a tile of 64 nodes, bit masks of
// who sees whom by halving the ways to the roots, the rows' K and V as they are.
#pragma once

#include "kernels.h"

namespace hstu {
namespace tree {

constexpr int kThreads = 256;
constexpr int kTile = 64;         // keys a wave takes at once
constexpr int kBlock = 256;       // keys whose bias is held
constexpr int kBiasLd = kBlock + 4;
constexpr float kMasked = -1e30f;  // SiLU of it is -0

__device__ __forceinline__ float silu(float s) { return s * sigmoid_fast(s); }

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

// Ways to the roots of the nodes below n (parents at `up`, one int64 each): in
// every round a node takes over the node that its own on the way knows of, and
// that one's count of steps (and set of nodes within the tile from `first`).
// Ends with all waves past a barrier and the results in `node` / `seen`.
template <bool MASK>
__device__ __forceinline__ void walk(const int64_t* up, int n, int first, short2* node,
                                     uint64_t* seen) {
  constexpr int M = kMaxDraft / kThreads;
  short2 x[M];
  uint64_t m[M];
  bool more = false;
#pragma unroll
  for (int e = 0; e < M; e++) {
    const int i = threadIdx.x + e * kThreads;
    x[e] = short2{-1, 0};
    m[e] = 0;
    if (i < n) {
      if (up) {
        const int64_t p = up[i];
        if (p >= 0 && p < i) x[e] = short2{(short)p, 1};
      }
      if (MASK && i >= first && i < first + kTile) m[e] = 1ull << (i - first);
      node[i] = x[e];
      if (MASK) seen[i] = m[e];
    }
    more |= x[e].x >= 0;
  }
  while (__syncthreads_or(more)) {
    more = false;
#pragma unroll
    for (int e = 0; e < M; e++)
      if (x[e].x >= 0) {
        const short2 u = node[x[e].x];
        if (MASK) m[e] |= seen[x[e].x];
        x[e] = short2{u.x, (short)(x[e].y + u.y)};
        more |= u.x >= 0;
      }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < M; e++) {
      const int i = threadIdx.x + e * kThreads;
      if (i < n) {
        node[i] = x[e];
        if (MASK) seen[i] = m[e];
      }
    }
  }
}

template <int KIND, int DQK, int DV, int R>
__global__ __launch_bounds__(kThreads) void attn_tree_kernel(const TreeArgs a, const TreeSplit sp) {
  constexpr bool Q8 = KIND != kCacheBf16;     // quantised
  constexpr int CB = Q8 ? 1 : 2;              // bytes of a code
  constexpr int KW = DQK * CB / 16;           // words of a K row a lane reads
  constexpr int VW = 16 * CB / 4;             // words of 16 keys of a feature
  constexpr int KS = DQK / 32, NC = DV / 16;  // contraction steps, column tiles
  __shared__ __attribute__((aligned(16))) float bias[16 * R * kBiasLd];
  __shared__ __attribute__((aligned(16))) char shared_a[2 * 4 * kBlock * 4];
  __shared__ int64_t rows16[kBlock / 16];  // first row of 16 keys for head 0, or -1
  __shared__ short2 node[kMaxDraft];
  __shared__ float rtime[256];
  __shared__ int64_t row_time[16 * R];
  __shared__ int row_pos[16 * R];
  // scales of the cached keys [2][hg][kBlock], or the drafted tile's masks
  float* scales = reinterpret_cast<float*>(shared_a);
  uint64_t* seen = reinterpret_cast<uint64_t*>(shared_a);
  static_assert(sizeof(shared_a) >= kMaxDraft * sizeof(uint64_t), "masks fit");

  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int H = a.ja.num_heads, lg = a.c.lg_page;
  const int item = blockIdx.x % (sp.part ? sp.chunks + 1 : 1);
  const int rb = (blockIdx.x / (sp.part ? sp.chunks + 1 : 1)) % sp.row_blocks;
  const int b = blockIdx.x / (sp.part ? sp.chunks + 1 : 1) / sp.row_blocks;
  const int64_t o = a.ja.seq_offsets[b];
  const int64_t o1 = min(a.ja.seq_offsets[b + 1], a.ja.total_tokens);
  const int L = (int)max((int64_t)0, min(o1 - o, (int64_t)a.max_draft));
  const int r0 = rb * 16 * R;
  if (o < 0 || r0 >= L) return;
  const int cap = a.c.max_pages << lg;
  const int n_b = (int)max((int64_t)0, min(a.c.lengths[b], (int64_t)cap));
  const bool drafted = !sp.part || item == sp.chunks;  // takes the drafted keys (too)
  const int from = sp.part ? item * sp.chunk_len : 0;
  const int to = sp.part ? (drafted ? from : min(n_b, from + sp.chunk_len)) : n_b;
  if (!drafted && from >= n_b) return;
  const int groups = min(R, (L - r0 + 15) / 16);
  const int nodes = min(L, r0 + 16 * R);
  const int waves_hg = sp.hg, ks_count = 4 / sp.hg;
  const int hh = wave % waves_hg, ks = wave / waves_hg;
  const int head = blockIdx.y * sp.hg + hh;
  const int r = lane % 16, g = lane / 16;
  const int N = a.ja.max_seq_len;

  // Q as the right operand: row r of each group, in the order of feature().
  bf16x8 q[R][KS];
#pragma unroll
  for (int m = 0; m < R; m++) {
    const int row = r0 + 16 * m + r;
    const uint16_t* src = (const uint16_t*)a.t.q + (o + row) * a.t.q_stride + (int64_t)head * DQK;
#pragma unroll
    for (int s = 0; s < KS; s++) {
      u32x4 v = zero_u32x4();
      if (row < L) v = *reinterpret_cast<const u32x4*>(src + feature<KIND, DQK>(s, g));
      q[m][s] = as_bf16x8(v);
    }
  }
  f32x4 acc[R][NC];
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int c = 0; c < NC; c++) acc[m][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int i = tid; i < a.ja.num_buckets; i += kThreads) rtime[i] = a.ja.rab_time[i];
  walk<false>(a.parents ? a.parents + o : nullptr, nodes, 0, node, nullptr);
  for (int i = tid; i < 16 * R; i += kThreads) {
    const int row = r0 + i;
    row_pos[i] = n_b + (row < nodes ? node[row].y : 0);
    row_time[i] = row < nodes ? a.ja.timestamps[o + row] : 0;
  }

  // ---- cached keys ----
  for (int k0 = from; k0 < to; k0 += kBlock) {
    __syncthreads();  // row_pos; the block before is done with bias, scales and rows16
    {
      const int j = k0 + tid;
      int64_t page = -1;
      if (j < to) {
        page = a.c.page_table[(int64_t)b * a.c.max_pages + (j >> lg)];
        if (page >= a.c.num_pages) page = -1;
      }
      const bool ok = page >= 0;
      const int place = j & ((1 << lg) - 1);
      if (tid % 16 == 0) rows16[tid / 16] = ok ? ((page * H) << lg) + place : -1;
      const int64_t time = ok ? a.c.tc[(page << lg) + place] : 0;
      if constexpr (Q8)
        for (int x = 0; x < sp.hg; x++) {
          const int64_t at = ((page * H + blockIdx.y * sp.hg + x) << lg) + place;
          scales[x * kBlock + tid] = ok ? a.c.k_scale[at] : 0.0f;
          scales[(4 + x) * kBlock + tid] = ok ? a.c.v_scale[at] : 0.0f;
        }
      const int base = N - 1 + j;
      for (int m = 0; m < 16 * groups; m++) {
        float v = kMasked;
        if (ok)
          v = a.ja.rab_pos[max(0, base - row_pos[m])] +
              rtime[time_bucket64(row_time[m] - time, a.ja.num_buckets)];
        bias[m * kBiasLd + tid] = v;
      }
    }
    __syncthreads();
    const int keys = min(kBlock, to - k0);
    for (int t0 = ks * kTile; t0 < keys; t0 += ks_count * kTile) {
      const bool full = __builtin_amdgcn_readfirstlane(
          t0 + kTile <= keys && rows16[t0 / 16] >= 0 && rows16[t0 / 16 + 1] >= 0 &&
          rows16[t0 / 16 + 2] >= 0 && rows16[t0 / 16 + 3] >= 0);
      uint32_t kw[4][KW];
      uint32_t vw[NC][VW];
      {
        const int64_t row = rows16[t0 / 16 + r / 4];
#pragma unroll
        for (int t = 0; t < 4; t++) {
          const char* src = (const char*)a.c.kc +
                            (row + ((int64_t)head << lg) + 4 * t + r % 4) * (DQK * CB);
          const bool on = full || (row >= 0 && t0 + 16 * (r / 4) + 4 * t + r % 4 < keys);
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
      }
      {
        const int64_t row = rows16[t0 / 16 + g];
        const int place = (int)(row & ((1 << lg) - 1));
        const int64_t ph = (row >> lg) + head;
        const int left = full ? 16 : row < 0 ? 0 : min(16, keys - (t0 + 16 * g));
#pragma unroll
        for (int c = 0; c < NC; c++) {
          const char* src = (const char*)a.c.vc + (((ph * DV + 16 * c + r) << lg) + place) * CB;
#pragma unroll
          for (int u = 0; u < VW / 4; u++) {
            u32x4 v = zero_u32x4();
            if (full || left > 0) v = *reinterpret_cast<const u32x4*>(src + 16 * u);
#pragma unroll
            for (int e = 0; e < 4; e++) {
              uint32_t w = v[e];
              if (!full) {  // codes behind the last key count as zeros
                const int keep = (left * CB - 16 * u - 4 * e) * 8;  // bits
                w = keep >= 32 ? w : keep <= 0 ? 0u : w & ((1u << keep) - 1u);
              }
              vw[c][4 * u + e] = w;
            }
          }
        }
      }
#pragma unroll
      for (int s = 0; s < 2; s++) {
        bf16x8 p[R];
#pragma unroll
        for (int m = 0; m < R; m++) {
          if (m >= groups) break;
          float w[8];
#pragma unroll
          for (int x = 0; x < 2; x++) {
            const int t = 2 * s + x;
            const int at = t0 + 16 * g + 4 * t;
            const f32x4 bv = *reinterpret_cast<const f32x4*>(&bias[(16 * m + r) * kBiasLd + at]);
            f32x4 sc = Q8 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : bv;
#pragma unroll
            for (int st = 0; st < KS; st++) {
              bf16x8 kf;
              if constexpr (Q8) kf = widen<KIND>(kw[t][2 * st], kw[t][2 * st + 1]);
              else kf = as_bf16x8(u32x4{kw[t][4 * st], kw[t][4 * st + 1], kw[t][4 * st + 2],
                                        kw[t][4 * st + 3]});
              sc = mfma16x16x32(kf, q[m][st], sc);
            }
            if constexpr (Q8) {
              const f32x4 kf = *reinterpret_cast<const f32x4*>(&scales[hh * kBlock + at]);
              const f32x4 vf = *reinterpret_cast<const f32x4*>(&scales[(4 + hh) * kBlock + at]);
#pragma unroll
              for (int i = 0; i < 4; i++) w[4 * x + i] = silu(fmaf(sc[i], kf[i], bv[i])) * vf[i];
            } else {
#pragma unroll
              for (int i = 0; i < 4; i++) w[4 * x + i] = silu(sc[i]);
            }
          }
          p[m] = as_bf16x8(pack_bf16x8(w));
        }
#pragma unroll
        for (int c = 0; c < NC; c++) {
          bf16x8 vf;
          if constexpr (Q8) vf = widen<KIND>(vw[c][2 * s], vw[c][2 * s + 1]);
          else vf = as_bf16x8(u32x4{vw[c][4 * s], vw[c][4 * s + 1], vw[c][4 * s + 2],
                                    vw[c][4 * s + 3]});
#pragma unroll
          for (int m = 0; m < R; m++)
            if (m < groups) acc[m][c] = mfma16x16x32(p[m], vf, acc[m][c]);
        }
      }
    }
  }

  // ---- drafted keys ----
  if (drafted) {
    for (int k0 = 0; k0 < nodes; k0 += kTile) {
      __syncthreads();  // row_pos and node; bias and scales are done with
      walk<true>(a.parents ? a.parents + o : nullptr, nodes, k0, node, seen);
      bool any = false;
      for (int i = tid; i < 16 * groups; i += kThreads)
        any |= r0 + i < L && seen[r0 + i] != 0;
      if (!__syncthreads_or(any)) continue;
      {
        const int j = k0 + tid % kTile;
        if (j < nodes) {
          const int64_t time = a.ja.timestamps[o + j];
          const int base = N - 1 + n_b + node[j].y;
          for (int m = tid / kTile; m < 16 * groups; m += kThreads / kTile)
            bias[m * kBiasLd + tid % kTile] =
                a.ja.rab_pos[max(0, min(2 * N - 2, base - row_pos[m]))] +
                rtime[time_bucket64(row_time[m] - time, a.ja.num_buckets)];
        }
      }
      __syncthreads();
      if ((k0 / kTile) % ks_count != ks) continue;
      bf16x8 p[R][2];
#pragma unroll
      for (int s = 0; s < 2; s++) {
        float w[R][8];
#pragma unroll
        for (int x = 0; x < 2; x++) {
          const int t = 2 * s + x;
          const int key = k0 + 16 * (r / 4) + 4 * t + r % 4;
          const uint16_t* src =
              (const uint16_t*)a.t.k + (o + key) * a.t.k_stride + (int64_t)head * DQK;
          f32x4 sc[R];
#pragma unroll
          for (int m = 0; m < R; m++) sc[m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int st = 0; st < KS; st++) {
            u32x4 v = zero_u32x4();
            if (key < nodes) v = *reinterpret_cast<const u32x4*>(src + feature<KIND, DQK>(st, g));
#pragma unroll
            for (int m = 0; m < R; m++) sc[m] = mfma16x16x32(as_bf16x8(v), q[m][st], sc[m]);
          }
#pragma unroll
          for (int m = 0; m < R; m++) {
            const int row = r0 + 16 * m + r;
            const uint64_t mask = row < L ? seen[row] : 0;
            const int at = 16 * g + 4 * t;
            const f32x4 bv = *reinterpret_cast<const f32x4*>(&bias[(16 * m + r) * kBiasLd + at]);
#pragma unroll
            for (int i = 0; i < 4; i++)  // what is not seen may be anything
              w[m][4 * x + i] = (mask >> (at + i)) & 1 ? silu(sc[m][i] + bv[i]) : 0.0f;
          }
        }
#pragma unroll
        for (int m = 0; m < R; m++) p[m][s] = as_bf16x8(pack_bf16x8(w[m]));
      }
      // V as it is: 8 keys of a feature from 8 rows.  Infinities and NaN would
      // reach rows that do not see them (their weight 0 times it): they count
      // as zeros here and are added to the rows that do below.
      uint32_t odd = 0;  // keys 16 g + .. of such values in this lane's features
#pragma unroll
      for (int c = 0; c < NC; c++) {
        const uint16_t* src =
            (const uint16_t*)a.t.v + o * a.t.v_stride + (int64_t)head * DV + 16 * c + r;
#pragma unroll
        for (int s = 0; s < 2; s++) {
          uint32_t e[8];
#pragma unroll
          for (int i = 0; i < 8; i++) {
            const int key = k0 + 16 * g + 8 * s + i;
            e[i] = key < nodes ? src[key * a.t.v_stride] : 0u;
            if ((e[i] & 0x7f80u) == 0x7f80u) {
              odd |= 1u << (8 * s + i);
              e[i] = 0u;
            }
          }
          const bf16x8 vf = as_bf16x8(u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16,
                                            e[4] | e[5] << 16, e[6] | e[7] << 16});
#pragma unroll
          for (int m = 0; m < R; m++) acc[m][c] = mfma16x16x32(p[m][s], vf, acc[m][c]);
        }
      }
      if (__any(odd != 0)) {
#pragma unroll
        for (int x = 1; x < 16; x *= 2) odd |= (uint32_t)__shfl_xor((int)odd, x, 64);
        uint64_t keys = 0;
#pragma unroll
        for (int x = 0; x < 4; x++)
          keys |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)odd, 16 * x) << (16 * x);
        for (; keys; keys &= keys - 1) {
          const int kk = __builtin_ctzll(keys);
          const uint16_t* kr =
              (const uint16_t*)a.t.k + (o + k0 + kk) * a.t.k_stride + (int64_t)head * DQK;
          const uint16_t* vr =
              (const uint16_t*)a.t.v + (o + k0 + kk) * a.t.v_stride + (int64_t)head * DV + r;
#pragma unroll
          for (int m = 0; m < R; m++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
              const int at = 16 * m + 4 * g + i, row = r0 + at;
              if (row >= L || !((seen[row] >> kk) & 1)) continue;
              const uint16_t* qr =
                  (const uint16_t*)a.t.q + (o + row) * a.t.q_stride + (int64_t)head * DQK;
              float sum = bias[at * kBiasLd + kk];
              for (int f = 0; f < DQK; f++)
                sum += bf16_bits_to_f32(qr[f]) * bf16_bits_to_f32(kr[f]);
              sum = silu(sum);
#pragma unroll
              for (int c = 0; c < NC; c++) {
                const uint32_t e = vr[16 * c];
                if ((e & 0x7f80u) == 0x7f80u) acc[m][c][i] += sum * bf16_bits_to_f32(e);
              }
            }
        }
      }
    }
  }

  // ---- the waves of a head add up, in order ----
  for (int x = 1; x < ks_count; x++) {
    __syncthreads();
    float* space = bias + hh * (16 * R * DV);
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
  const float scale = 1.0f / (float)N;
#pragma unroll
  for (int m = 0; m < R; m++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int row = r0 + 16 * m + 4 * g + i;
      if (row >= L) continue;
      const int64_t at = ((o + row) * H + head) * DV + r;
      if (sp.part) {
        float* dst = sp.part + (int64_t)item * a.ja.total_tokens * H * DV + at;
#pragma unroll
        for (int c = 0; c < NC; c++) dst[16 * c] = acc[m][c][i];
      } else {
        uint16_t* dst = (uint16_t*)a.out + at;
#pragma unroll
        for (int c = 0; c < NC; c++) dst[16 * c] = f32_to_bf16_bits(acc[m][c][i] * scale);
      }
    }
}

// The launch for one kind of cache.
template <int KIND>
hipError_t launch(const TreeArgs& a, const TreeSplit& sp, hipStream_t s) {
  const int64_t blocks =
      (int64_t)a.ja.num_seqs * sp.row_blocks * (sp.part ? sp.chunks + 1 : 1);
  const dim3 grid((unsigned)blocks, (unsigned)(a.ja.num_heads / sp.hg));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a, sp);
    return hipGetLastError();
  };
#define HSTU_TREE_R(DQK, DV)                                        \
  if (sp.rows == 16) return go(attn_tree_kernel<KIND, DQK, DV, 1>);        \
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

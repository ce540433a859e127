// The paged cache of keys and values (include/hstu.h): rows are quantised as
// they are written, and read back.
//
// HBM-bound: a row is read once and its codes written once, or the reverse.  A
// workgroup takes a block of 64 positions of one sequence (which no page of 64
// tokens or more, and no group of 16 keys of a smaller one, crosses) and one
// head.  d / 8 neighbouring lanes share a row, so that its largest magnitude
// takes a few lane exchanges.  K rows go where they belong as they are; V goes
// through LDS, because a page holds a feature's keys side by side.  25000 tokens
// of 4 heads of 128, e4m3: written in 22.6 us (3.4 TB/s), read back in 16.0 (4.8;
// a large copy: 5.2); 8 users of 4096-8192, int8, read in 31.8 us (4.8 TB/s); a
// token for each of 64 users: 9.4 and 4.8 us, a chain of dependent loads.
#include "kernels.h"

namespace hstu {
namespace {

constexpr int kThreads = 256;
constexpr int kBlk = 1 << 6;   // positions a workgroup takes
constexpr int kGroup = 16;     // keys of a feature written or read at once
constexpr float kTiny = 7.8886090522101181e-31f;  // 2^-100

// Eight features of a row.
template <typename E>
struct Eight;
template <>
struct Eight<uint16_t> {
  u32x4 raw;
  __device__ void load(const uint16_t* p) { raw = *reinterpret_cast<const u32x4*>(p); }
  __device__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      x[2 * i] = __uint_as_float(raw[i] << 16);
      x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
  }
};
template <>
struct Eight<float> {
  f32x4 lo, hi;
  __device__ void load(const float* p) {
    lo = *reinterpret_cast<const f32x4*>(p);
    hi = *reinterpret_cast<const f32x4*>(p + 4);
  }
  __device__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      x[i] = lo[i];
      x[4 + i] = hi[i];
    }
  }
};

// x / s rounded to the nearest integer, ties to even.  The first guess is off
// by one at most; x - guess * s and s / 2 are exact where the guess is close
// to a tie (both are multiples of half a unit of s's last place, below 2^24 of
// them), so the comparison decides as the exact quotient would.
__device__ __forceinline__ int int8_code(float x, float s, float inv) {
  float g = rintf(x * inv);
  const float r = fmaf(-g, s, x), half = 0.5f * s;
  const bool odd = ((int)g & 1) != 0;
  if (r > half || (odd && r == half)) g += 1.0f;
  else if (r < -half || (odd && r == -half)) g -= 1.0f;
  return (int)g;
}

// Codes of eight features of a row whose largest magnitude has the bits `top`
// (the same in all lanes of the row), and the row's scale.
template <int KIND>
__device__ __forceinline__ uint2 quantise(const float* x, uint32_t top, float* scale) {
  if (top >= 0x7f800000u) {  // an infinity or a NaN in the row
    *scale = __uint_as_float(0x7fc00000u);
    return uint2{0u, 0u};
  }
  const float big = __uint_as_float(top);
  if (big < kTiny) {
    *scale = 1.0f;
    return uint2{0u, 0u};
  }
  uint32_t w[2];
  if constexpr (KIND == kCacheInt8) {
    const float s = big * (1.0f / 127.0f);
    const float inv = 1.0f / s;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      w[i] = 0;
#pragma unroll
      for (int b = 0; b < 4; b++)
        w[i] |= (uint32_t)(int8_code(x[4 * i + b], s, inv) & 255) << (8 * b);
    }
    *scale = s;
  } else {
    // big = 1.m * 2^x: 448 = 1.75 * 2^8, so the exponent is x - 8, one more for m > 0.75.
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(e, 119);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);  // 2^-e; e >= -109
#pragma unroll
    for (int i = 0; i < 2; i++) {
      float y[4];
#pragma unroll
      for (int b = 0; b < 4; b++)
        y[b] = __builtin_amdgcn_fmed3f(x[4 * i + b] * inv, -448.0f, 448.0f);
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
    }
    *scale = __uint_as_float((uint32_t)(127 + e) << 23);
  }
  return uint2{w[0], w[1]};
}

template <int KIND>
__device__ __forceinline__ void dequantise(uint2 c, float s, float* x) {
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const uint32_t w = i ? c.y : c.x;
    if constexpr (KIND == kCacheInt8) {
#pragma unroll
      for (int b = 0; b < 4; b++) x[4 * i + b] = (float)(int8_t)(w >> (8 * b)) * s;
    } else {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
      const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
      x[4 * i] = lo[0] * s;
      x[4 * i + 1] = lo[1] * s;
      x[4 * i + 2] = hi[0] * s;
      x[4 * i + 3] = hi[1] * s;
    }
  }
}

// What a workgroup works on: positions [lo, hi) of sequence `seq`, all in the
// block of kBlk positions from `first`; position x is row row0 + x.
struct Block {
  int seq;
  int64_t first, lo, hi, row0;
};

// Work item `item` of the blocks of all sequences.  Sequence b's items start at
// offsets[b] / kBlk + 2 b: it touches at most (L + 2 kBlk - 2) / kBlk blocks, and
// the next one's start is that far away whatever the offsets.
__device__ __forceinline__ bool find_block(const CacheArgs& a, int64_t item, Block* o) {
  const int lane = __lane_id(), B = a.num_seqs;
  int lo = 0;
  int64_t from, to, start = 0;
  if (B < 64) {  // one load each: lane l knows sequence l
    const int64_t off = lane <= B ? a.seq_offsets[lane] : 0;
    const int64_t st = a.starts && lane < B ? a.starts[lane] : 0;
    const uint64_t below = __ballot(lane < B && off / kBlk + 2 * lane <= item);
    lo = below ? 63 - __builtin_clzll(below) : 0;
    from = readlane64(off, lo);
    to = readlane64(off, lo + 1);
    start = readlane64(st, lo);
  } else {
    int n = B;
    while (n > 1) {
      const int step = (n + 63) / 64;
      const int at = lane * step;
      const int64_t b = lo + (at < n ? at : 0);
      const uint64_t below = __ballot(at < n && a.seq_offsets[b] / kBlk + 2 * b <= item);
      const int last = below ? 63 - __builtin_clzll(below) : 0;
      lo += last * step;
      n = min(step, n - last * step);
    }
    from = a.seq_offsets[lo];
    to = a.seq_offsets[lo + 1];
    if (a.starts) start = a.starts[lo];
  }
  if (from < 0 || to > a.total_tokens) return false;
  // A start may be anything: beyond what pages can hold it only has to stay there.
  const int64_t far = (int64_t)1 << 42;
  start = max(-far, min(far, start));
  const int64_t j = item - (from / kBlk + 2 * (int64_t)lo);
  o->seq = lo;
  o->first = ((start >> 6) + j) * kBlk;
  o->lo = max(start, o->first);
  o->hi = min(start + (to - from), o->first + kBlk);
  o->row0 = from - start;
  return j >= 0 && o->lo < o->hi;
}

// The page of position x of sequence b, or -1.
__device__ __forceinline__ int64_t page_of(const CacheArgs& a, int b, int64_t x) {
  const int64_t i = x >> a.lg_page;
  if (i < 0 || i >= a.max_pages) return -1;
  const int64_t p = a.page_table[(int64_t)b * a.max_pages + i];
  return p >= 0 && p < a.num_pages ? p : -1;
}

// A tile of V in LDS: kBlk rows of D codes, `ld` words apart, so that the four groups
// of 16 keys that neighbouring lanes take lie in different quarters of the banks.
template <int KIND, int D>
struct Tile {
  static constexpr int CB = KIND == kCacheBf16 ? 2 : 1;  // bytes of a code
  static constexpr int FP = 4 / CB;                      // features of a word
  static constexpr int ld = D * CB / 4 + 1;
  uint32_t w[kBlk * ld];
};

// 16 words (keys m, FP features each) <-> FP rows (one feature, 16 keys each).
__device__ __forceinline__ uint32_t bytes(uint32_t hi, uint32_t lo, uint32_t which) {
  return __builtin_amdgcn_perm(hi, lo, which);
}
__device__ __forceinline__ void turn4(const uint32_t* a, uint32_t* o) {  // 4 x 4 bytes
  const uint32_t x = bytes(a[1], a[0], 0x05010400u), y = bytes(a[1], a[0], 0x07030602u);
  const uint32_t z = bytes(a[3], a[2], 0x05010400u), v = bytes(a[3], a[2], 0x07030602u);
  o[0] = bytes(z, x, 0x05040100u);
  o[1] = bytes(z, x, 0x07060302u);
  o[2] = bytes(v, y, 0x05040100u);
  o[3] = bytes(v, y, 0x07060302u);
}
__device__ __forceinline__ void turn2(const uint32_t* a, uint32_t* o) {  // 2 x 2 halfwords
  o[0] = bytes(a[1], a[0], 0x05040100u);
  o[1] = bytes(a[1], a[0], 0x07060302u);
}

// Where the codes of feature c and the keys of group g of a page's V lie.
template <int CB, int D>
__device__ __forceinline__ char* value_at(const CacheArgs& a, int64_t page, int head, int c,
                                          int place) {
  return (char*)a.vc + ((((page * a.num_heads + head) * D + c) << a.lg_page) + place) * CB;
}

// Largest magnitude of a row of D / 8 lanes with eight features each, as bits.
template <int LPR>
__device__ __forceinline__ uint32_t row_top(const float* f) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
  for (int m = 1; m < LPR; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
  return top;
}

// Eight codes of a row (in `w`, 2 or 4 words) and, from its first lane, its scale.
template <typename E, int KIND, int LPR>
__device__ __forceinline__ void encode(const Eight<E>& e, uint32_t* w, float* scale) {
  float f[8];
  e.get(f);
  if constexpr (KIND == kCacheBf16) {
    const u32x4 v = pack_bf16x8(f);
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = v[i];
  } else {
    const uint2 v = quantise<KIND>(f, row_top<LPR>(f), scale);
    w[0] = v.x;
    w[1] = v.y;
  }
}

// Five waves a SIMD: what the registers of all its loads allow (six spill: 44 us against
// 38 for writing and reading 25000 tokens).
template <typename E, int KIND, int DQK, int DV>
__global__ __launch_bounds__(kThreads, 5) void cache_write_kernel(const CacheArgs a) {
  using Tl = Tile<KIND, DV>;
  constexpr int CB = Tl::CB, FP = Tl::FP;
  constexpr int LK = DQK / 8, LV = DV / 8;                              // lanes of a row
  constexpr int NK = kBlk * LK / kThreads, NV = kBlk * LV / kThreads;   // rows of a thread
  __shared__ Tl tile;
  __shared__ int64_t pages[kBlk / kGroup];
  const int head = blockIdx.y, tid = threadIdx.x;
  const int page_mask = (1 << a.lg_page) - 1;
  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    Block blk;
    if (!find_block(a, item, &blk)) continue;
    // every load before any of their results is used
    const int64_t page_of_group =
        tid < kBlk / kGroup ? page_of(a, blk.seq, blk.first + tid * kGroup) : 0;
    Eight<E> ek[NK], ev[NV];
    auto there = [&](int r) { return blk.first + r >= blk.lo && blk.first + r < blk.hi; };
#pragma unroll
    for (int i = 0; i < NK; i++) {
      const int r = tid / LK + i * (kThreads / LK);
      ek[i] = Eight<E>{};
      if (there(r))
        ek[i].load((const E*)a.k + (blk.row0 + blk.first + r) * a.k_stride + (int64_t)head * DQK +
                   8 * (tid % LK));
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int r = tid / LV + i * (kThreads / LV);
      ev[i] = Eight<E>{};
      if (there(r))
        ev[i].load((const E*)a.v + (blk.row0 + blk.first + r) * a.v_stride + (int64_t)head * DV +
                   8 * (tid % LV));
    }
    __syncthreads();  // tile and pages of the item before
    if (tid < kBlk / kGroup) pages[tid] = page_of_group;
    __syncthreads();
    if (head == 0 && tid < kBlk && there(tid) && pages[tid / kGroup] >= 0) {
      const int64_t x = blk.first + tid;
      a.tc[(pages[tid / kGroup] << a.lg_page) + (x & page_mask)] = a.ts[blk.row0 + x];
    }
#pragma unroll
    for (int i = 0; i < NK; i++) {
      const int r = tid / LK + i * (kThreads / LK);
      uint32_t w[2 * CB];
      float scale;
      encode<E, KIND, LK>(ek[i], w, &scale);
      const int64_t page = pages[r / kGroup];
      if (!there(r) || page < 0) continue;
      const int64_t row = ((page * a.num_heads + head) << a.lg_page) +
                          ((blk.first + r) & page_mask);
      char* dst = (char*)a.kc + (row * DQK + 8 * (tid % LK)) * CB;
      if constexpr (CB == 2) {
        *reinterpret_cast<u32x4*>(dst) = u32x4{w[0], w[1], w[2], w[3]};
      } else {
        *reinterpret_cast<uint2*>(dst) = uint2{w[0], w[1]};
        if (tid % LK == 0) a.k_scale[row] = scale;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int r = tid / LV + i * (kThreads / LV);
      uint32_t w[2 * CB];
      float scale;
      encode<E, KIND, LV>(ev[i], w, &scale);
#pragma unroll
      for (int e = 0; e < 2 * CB; e++) tile.w[r * Tl::ld + 2 * CB * (tid % LV) + e] = w[e];
      const int64_t page = pages[r / kGroup];
      if (KIND != kCacheBf16 && tid % LV == 0 && there(r) && page >= 0)
        a.v_scale[((page * a.num_heads + head) << a.lg_page) + ((blk.first + r) & page_mask)] =
            scale;
    }
    __syncthreads();
    // FP features and 16 keys at a time; neighbouring lanes take the groups of one page row
    for (int u = tid; u < DV / FP * (kBlk / kGroup); u += kThreads) {
      const int g = u % (kBlk / kGroup), c = u / (kBlk / kGroup) * FP;
      const int64_t page = pages[g], x0 = blk.first + g * kGroup;
      if (page < 0 || x0 + kGroup <= blk.lo || x0 >= blk.hi) continue;
      uint32_t in[kGroup], out[FP][kGroup / FP];
#pragma unroll
      for (int m = 0; m < kGroup; m++) in[m] = tile.w[(g * kGroup + m) * Tl::ld + c / FP];
#pragma unroll
      for (int m = 0; m < kGroup / FP; m++) {
        uint32_t o[FP];
        if constexpr (FP == 4) turn4(in + FP * m, o);
        else turn2(in + FP * m, o);
#pragma unroll
        for (int f = 0; f < FP; f++) out[f][m] = o[f];
      }
      const bool all = x0 >= blk.lo && x0 + kGroup <= blk.hi;
#pragma unroll
      for (int f = 0; f < FP; f++) {
        char* dst = value_at<CB, DV>(a, page, head, c + f, (int)x0 & page_mask);
        if (all) {
#pragma unroll
          for (int m = 0; m < CB; m++)
            reinterpret_cast<u32x4*>(dst)[m] = u32x4{out[f][4 * m], out[f][4 * m + 1],
                                                     out[f][4 * m + 2], out[f][4 * m + 3]};
        } else {  // keys of other calls lie in the group
#pragma unroll
          for (int m = 0; m < kGroup; m++)
            if (x0 + m >= blk.lo && x0 + m < blk.hi) {
              const uint32_t v = out[f][m / FP] >> (8 * CB * (m % FP));
              if constexpr (CB == 2) reinterpret_cast<uint16_t*>(dst)[m] = (uint16_t)v;
              else reinterpret_cast<uint8_t*>(dst)[m] = (uint8_t)v;
            }
        }
      }
    }
  }
}

// Eight features of a row from its codes.
template <typename E, int KIND>
__device__ __forceinline__ void decode(const uint32_t* w, float scale, bool on, E* dst) {
  float f[8] = {};
  if (on) {
    if constexpr (KIND == kCacheBf16) {
      Eight<uint16_t> e;
      e.raw = u32x4{w[0], w[1], w[2], w[3]};
      e.get(f);
    } else {
      dequantise<KIND>(uint2{w[0], w[1]}, scale, f);
    }
  }
  if constexpr (sizeof(E) == 2) {
    *reinterpret_cast<u32x4*>(dst) = pack_bf16x8(f);
  } else {
    *reinterpret_cast<f32x4*>(dst) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4*>(dst + 4) = f32x4{f[4], f[5], f[6], f[7]};
  }
}

template <typename E, int KIND, int DQK, int DV>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const CacheArgs a) {
  using Tl = Tile<KIND, DV>;
  constexpr int CB = Tl::CB, FP = Tl::FP;
  constexpr int LK = DQK / 8, LV = DV / 8;
  constexpr int NK = kBlk * LK / kThreads, NV = kBlk * LV / kThreads;
  constexpr int kUnits = DV / FP * (kBlk / kGroup);
  constexpr int NU = (kUnits + kThreads - 1) / kThreads;
  __shared__ Tl tile;
  __shared__ int64_t pages[kBlk / kGroup];
  const int head = blockIdx.y, tid = threadIdx.x;
  const int page_mask = (1 << a.lg_page) - 1;
  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    Block blk;
    if (!find_block(a, item, &blk)) continue;
    const int64_t len = a.lengths[blk.seq];
    __syncthreads();  // tile and pages of the item before
    if (tid < kBlk / kGroup) pages[tid] = page_of(a, blk.seq, blk.first + tid * kGroup);
    __syncthreads();
    auto wanted = [&](int r) { return blk.first + r >= blk.lo && blk.first + r < blk.hi; };
    auto there = [&](int r) {
      return wanted(r) && blk.first + r < len && pages[r / kGroup] >= 0;
    };
    auto row_of = [&](int r) {
      return ((pages[r / kGroup] * a.num_heads + head) << a.lg_page) +
             ((blk.first + r) & page_mask);
    };
    // every load before any of their results is used
    uint32_t wk[NK][2 * CB];
    float sk[NK], sv[NV];
#pragma unroll
    for (int i = 0; i < NK; i++) {
      const int r = tid / LK + i * (kThreads / LK);
      sk[i] = 1.0f;
#pragma unroll
      for (int e = 0; e < 2 * CB; e++) wk[i][e] = 0;
      if (!there(r)) continue;
      const int64_t row = row_of(r);
      const char* src = (const char*)a.kc + (row * DQK + 8 * (tid % LK)) * CB;
      if constexpr (CB == 2) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(src);
#pragma unroll
        for (int e = 0; e < 4; e++) wk[i][e] = v[e];
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(src);
        wk[i][0] = v.x;
        wk[i][1] = v.y;
        sk[i] = a.k_scale[row];
      }
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int r = tid / LV + i * (kThreads / LV);
      sv[i] = KIND != kCacheBf16 && there(r) ? a.v_scale[row_of(r)] : 1.0f;
    }
    u32x4 wv[NU][FP][CB];
#pragma unroll
    for (int n = 0; n < NU; n++) {
      const int u = tid + n * kThreads;
      const int g = u % (kBlk / kGroup), c = u / (kBlk / kGroup) * FP;
      const int64_t page = pages[g], x0 = blk.first + g * kGroup;
      const bool on = u < kUnits && page >= 0 && x0 + kGroup > blk.lo && x0 < blk.hi;
#pragma unroll
      for (int f = 0; f < FP; f++)
#pragma unroll
        for (int m = 0; m < CB; m++) {
          wv[n][f][m] = zero_u32x4();
          if (on)
            wv[n][f][m] = reinterpret_cast<const u32x4*>(
                value_at<CB, DV>(a, page, head, c + f, (int)x0 & page_mask))[m];
        }
    }
    if (head == 0 && a.ts_out && tid < kBlk && wanted(tid)) {
      const int64_t x = blk.first + tid;
      a.ts_out[blk.row0 + x] =
          there(tid) ? a.tc[(pages[tid / kGroup] << a.lg_page) + (x & page_mask)] : 0;
    }
#pragma unroll
    for (int n = 0; n < NU; n++) {
      const int u = tid + n * kThreads;
      const int g = u % (kBlk / kGroup), c = u / (kBlk / kGroup) * FP;
      if (u >= kUnits) break;
#pragma unroll
      for (int m = 0; m < kGroup / FP; m++) {
        uint32_t in[FP], out[FP];
#pragma unroll
        for (int f = 0; f < FP; f++) in[f] = wv[n][f][m / 4][m % 4];
        if constexpr (FP == 4) turn4(in, out);
        else turn2(in, out);
#pragma unroll
        for (int f = 0; f < FP; f++)
          tile.w[(g * kGroup + FP * m + f) * Tl::ld + c / FP] = out[f];
      }
    }
#pragma unroll
    for (int i = 0; i < NK; i++) {
      const int r = tid / LK + i * (kThreads / LK);
      if (!wanted(r)) continue;
      decode<E, KIND>(wk[i], sk[i], there(r),
                      (E*)a.k_out + ((blk.row0 + blk.first + r) * a.num_heads + head) * DQK +
                          8 * (tid % LK));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int r = tid / LV + i * (kThreads / LV);
      if (!wanted(r)) continue;
      uint32_t w[2 * CB];
#pragma unroll
      for (int e = 0; e < 2 * CB; e++) w[e] = tile.w[r * Tl::ld + 2 * CB * (tid % LV) + e];
      decode<E, KIND>(w, sv[i], there(r),
                      (E*)a.v_out + ((blk.row0 + blk.first + r) * a.num_heads + head) * DV +
                          8 * (tid % LV));
    }
  }
}

template <typename E, int KIND>
hipError_t run(const CacheArgs& a, bool write, dim3 grid, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
#define HSTU_CACHE_V(DQK, DV)                                    \
  return write ? go(cache_write_kernel<E, KIND, DQK, DV>)        \
               : go(cache_read_kernel<E, KIND, DQK, DV>);
#define HSTU_CACHE(DQK)                           \
  if (a.d_v == 32) { HSTU_CACHE_V(DQK, 32) }      \
  if (a.d_v == 64) { HSTU_CACHE_V(DQK, 64) }      \
  HSTU_CACHE_V(DQK, 128)
  if (a.d_qk == 32) { HSTU_CACHE(32) }
  if (a.d_qk == 64) { HSTU_CACHE(64) }
  HSTU_CACHE(128)
#undef HSTU_CACHE
#undef HSTU_CACHE_V
}

template <typename E>
hipError_t run(const CacheArgs& a, int kind, bool write, dim3 grid, hipStream_t s) {
  return kind == kCacheBf16   ? run<E, kCacheBf16>(a, write, grid, s)
         : kind == kCacheInt8 ? run<E, kCacheInt8>(a, write, grid, s)
                              : run<E, kCacheE4m3>(a, write, grid, s);
}

}  // namespace

hipError_t launch_cache(CacheArgs a, int kind, int is_bf16, bool write, hipStream_t s) {
  if (a.total_tokens <= 0) return hipSuccess;
  a.items = a.total_tokens / kBlk + 2 * (int64_t)a.num_seqs;
  const dim3 grid((unsigned)min(a.items, (int64_t)1 << 22), (unsigned)a.num_heads);
  return is_bf16 ? run<uint16_t>(a, kind, write, grid, s) : run<float>(a, kind, write, grid, s);
}

}  // namespace hstu

// The paged cache of keys and values (include/hstu.h): rows are quantised as
// they are written, and read back.
//
// HBM-bound: a row is read once and its codes written once, or the reverse.  A
// workgroup takes a block of 64 positions of one sequence (which no page of 64
// tokens or more, and no group of 16 keys of a smaller one, crosses) and one
// head.  d / 8 neighbouring lanes share a row, so that its largest magnitude
// takes a few lane exchanges.  K rows go where they belong as they are; V goes
// through LDS, because a page holds a feature's keys side by side.
#include <type_traits>

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
#pragma unroll
    for (int i = 0; i < 2; i++) {
      float y[4];
#pragma unroll
      for (int b = 0; b < 4; b++)
        y[b] = fminf(fmaxf(ldexpf(x[4 * i + b], -e), -448.0f), 448.0f);
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], p, true);
    }
    *scale = ldexpf(1.0f, e);
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
  const int lane = __lane_id();
  int lo = 0, n = a.num_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = lane * step;
    const int64_t b = lo + (at < n ? at : 0);
    const uint64_t below = __ballot(at < n && a.seq_offsets[b] / kBlk + 2 * b <= item);
    const int last = below ? 63 - __builtin_clzll(below) : 0;
    lo += last * step;
    n = min(step, n - last * step);
  }
  const int64_t from = a.seq_offsets[lo], to = a.seq_offsets[lo + 1];
  if (from < 0 || to > a.total_tokens) return false;
  // A start may be anything: beyond what pages can hold it only has to stay there.
  const int64_t far = (int64_t)1 << 42;
  const int64_t start = a.starts ? max(-far, min(far, a.starts[lo])) : 0;
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

template <typename E, int KIND, int D>
__device__ __forceinline__ void write_side(const CacheArgs& a, const Block& blk, const int64_t* pages,
                                           int head, bool values, char* tile) {
  constexpr int LPR = D / 8;                       // lanes of a row
  constexpr int CB = KIND == kCacheBf16 ? 2 : 1;   // bytes of a code
  const int lane = threadIdx.x % LPR;
  const int page_mask = (1 << a.lg_page) - 1;
  const E* src = (const E*)(values ? a.v : a.k);
  const int64_t stride = values ? a.v_stride : a.k_stride;
  for (int r = threadIdx.x / LPR; r < kBlk; r += kThreads / LPR) {
    const int64_t x = blk.first + r;
    const bool on = x >= blk.lo && x < blk.hi;
    Eight<E> e;
    float f[8];
    uint32_t top = 0;
    if (on) {
      e.load(src + (blk.row0 + x) * stride + (int64_t)head * D + 8 * lane);
      e.get(f);
    }
    uint2 code{0u, 0u};
    u32x4 wide{0u, 0u, 0u, 0u};
    float scale = 1.0f;
    if constexpr (KIND == kCacheBf16) {
      if (on) wide = pack_bf16x8(f);
    } else {
      if (on)
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
      for (int m = 1; m < LPR; m *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
      if (on) code = quantise<KIND>(f, top, &scale);
    }
    const int64_t page = pages[r / kGroup];
    const int64_t ph = page * a.num_heads + head;
    const int place = (int)x & page_mask;
    if (on && page >= 0) {
      if constexpr (KIND != kCacheBf16)
        if (lane == 0)
          (values ? a.v_scale : a.k_scale)[(ph << a.lg_page) + place] = scale;
      if (!values) {
        char* dst = (char*)a.kc + (((ph << a.lg_page) + place) * D + 8 * lane) * CB;
        if constexpr (KIND == kCacheBf16) *reinterpret_cast<u32x4*>(dst) = wide;
        else *reinterpret_cast<uint2*>(dst) = code;
      }
    }
    if (values) {
      char* t = tile + (r * D + 8 * lane) * CB;
      if constexpr (KIND == kCacheBf16) *reinterpret_cast<u32x4*>(t) = wide;
      else *reinterpret_cast<uint2*>(t) = code;
    }
  }
  if (!values) return;
  __syncthreads();
  using C = typename std::conditional<KIND == kCacheBf16, uint16_t, uint8_t>::type;
  const C* t = (const C*)tile;
  for (int i = threadIdx.x; i < D * (kBlk / kGroup); i += kThreads) {
    const int c = i % D, g = i / D;
    const int64_t page = pages[g];
    const int64_t x0 = blk.first + g * kGroup;
    if (page < 0 || x0 + kGroup <= blk.lo || x0 >= blk.hi) continue;
    C* dst = (C*)a.vc + (((page * a.num_heads + head) * D + c) << a.lg_page) + ((int)x0 & page_mask);
    union {
      C c[kGroup];
      u32x4 w[sizeof(C)];
    } u;
#pragma unroll
    for (int m = 0; m < kGroup; m++) u.c[m] = t[(g * kGroup + m) * D + c];
    if (x0 >= blk.lo && x0 + kGroup <= blk.hi) {
#pragma unroll
      for (int m = 0; m < (int)sizeof(C); m++) reinterpret_cast<u32x4*>(dst)[m] = u.w[m];
    } else {  // keys of other calls lie in the group
#pragma unroll
      for (int m = 0; m < kGroup; m++)
        if (x0 + m >= blk.lo && x0 + m < blk.hi) dst[m] = u.c[m];
    }
  }
}

template <typename E, int KIND>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(const CacheArgs a) {
  __shared__ __attribute__((aligned(16))) char tile[kBlk * 128 * (KIND == kCacheBf16 ? 2 : 1)];
  __shared__ int64_t pages[kBlk / kGroup];
  const int head = blockIdx.y;
  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    Block blk;
    if (!find_block(a, item, &blk)) continue;
    __syncthreads();  // tile and pages of the item before
    if (threadIdx.x < kBlk / kGroup)
      pages[threadIdx.x] = page_of(a, blk.seq, blk.first + threadIdx.x * kGroup);
    __syncthreads();
    if (head == 0 && threadIdx.x < kBlk) {
      const int64_t x = blk.first + threadIdx.x, page = pages[threadIdx.x / kGroup];
      if (x >= blk.lo && x < blk.hi && page >= 0)
        a.tc[(page << a.lg_page) + (x & ((1 << a.lg_page) - 1))] = a.ts[blk.row0 + x];
    }
    switch (a.d_qk) {
      case 32: write_side<E, KIND, 32>(a, blk, pages, head, false, tile); break;
      case 64: write_side<E, KIND, 64>(a, blk, pages, head, false, tile); break;
      default: write_side<E, KIND, 128>(a, blk, pages, head, false, tile); break;
    }
    switch (a.d_v) {
      case 32: write_side<E, KIND, 32>(a, blk, pages, head, true, tile); break;
      case 64: write_side<E, KIND, 64>(a, blk, pages, head, true, tile); break;
      default: write_side<E, KIND, 128>(a, blk, pages, head, true, tile); break;
    }
  }
}

template <typename E, int KIND, int D>
__device__ __forceinline__ void read_side(const CacheArgs& a, const Block& blk, const int64_t* pages,
                                          int head, bool values, char* tile) {
  constexpr int LPR = D / 8;
  constexpr int CB = KIND == kCacheBf16 ? 2 : 1;
  const int page_mask = (1 << a.lg_page) - 1;
  using C = typename std::conditional<KIND == kCacheBf16, uint16_t, uint8_t>::type;
  if (values) {
    C* t = (C*)tile;
    for (int i = threadIdx.x; i < D * (kBlk / kGroup); i += kThreads) {
      const int c = i % D, g = i / D;
      const int64_t page = pages[g];
      const int64_t x0 = blk.first + g * kGroup;
      if (page < 0 || x0 + kGroup <= blk.lo || x0 >= blk.hi) continue;
      const C* src = (const C*)a.vc + (((page * a.num_heads + head) * D + c) << a.lg_page) +
                     ((int)x0 & page_mask);
      union {
        C c[kGroup];
        u32x4 w[sizeof(C)];
      } u;
#pragma unroll
      for (int m = 0; m < (int)sizeof(C); m++) u.w[m] = reinterpret_cast<const u32x4*>(src)[m];
#pragma unroll
      for (int m = 0; m < kGroup; m++) t[(g * kGroup + m) * D + c] = u.c[m];
    }
    __syncthreads();
  }
  const int lane = threadIdx.x % LPR;
  E* out = (E*)(values ? a.v_out : a.k_out);
  const int64_t len = a.lengths[blk.seq];
  for (int r = threadIdx.x / LPR; r < kBlk; r += kThreads / LPR) {
    const int64_t x = blk.first + r;
    if (x < blk.lo || x >= blk.hi) continue;
    const int64_t page = pages[r / kGroup];
    const int64_t ph = page * a.num_heads + head;
    const int place = (int)x & page_mask;
    float f[8] = {};
    if (page >= 0 && x < len) {
      const char* src = values ? tile + (r * D + 8 * lane) * CB
                               : (const char*)a.kc + (((ph << a.lg_page) + place) * D + 8 * lane) * CB;
      if constexpr (KIND == kCacheBf16) {
        Eight<uint16_t> e;
        e.load((const uint16_t*)src);
        e.get(f);
      } else {
        const float s = (values ? a.v_scale : a.k_scale)[(ph << a.lg_page) + place];
        dequantise<KIND>(*reinterpret_cast<const uint2*>(src), s, f);
      }
    }
    E* dst = out + ((blk.row0 + x) * a.num_heads + head) * D + 8 * lane;
    if constexpr (sizeof(E) == 2) {
      *reinterpret_cast<u32x4*>(dst) = pack_bf16x8(f);
    } else {
      *reinterpret_cast<f32x4*>(dst) = f32x4{f[0], f[1], f[2], f[3]};
      *reinterpret_cast<f32x4*>(dst + 4) = f32x4{f[4], f[5], f[6], f[7]};
    }
  }
}

template <typename E, int KIND>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const CacheArgs a) {
  __shared__ __attribute__((aligned(16))) char tile[kBlk * 128 * (KIND == kCacheBf16 ? 2 : 1)];
  __shared__ int64_t pages[kBlk / kGroup];
  const int head = blockIdx.y;
  for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
    Block blk;
    if (!find_block(a, item, &blk)) continue;
    __syncthreads();
    if (threadIdx.x < kBlk / kGroup)
      pages[threadIdx.x] = page_of(a, blk.seq, blk.first + threadIdx.x * kGroup);
    __syncthreads();
    if (head == 0 && a.ts_out && threadIdx.x < kBlk) {
      const int64_t x = blk.first + threadIdx.x, page = pages[threadIdx.x / kGroup];
      if (x >= blk.lo && x < blk.hi)
        a.ts_out[blk.row0 + x] = page >= 0 && x < a.lengths[blk.seq]
                                     ? a.tc[(page << a.lg_page) + (x & ((1 << a.lg_page) - 1))]
                                     : 0;
    }
    switch (a.d_qk) {
      case 32: read_side<E, KIND, 32>(a, blk, pages, head, false, tile); break;
      case 64: read_side<E, KIND, 64>(a, blk, pages, head, false, tile); break;
      default: read_side<E, KIND, 128>(a, blk, pages, head, false, tile); break;
    }
    switch (a.d_v) {
      case 32: read_side<E, KIND, 32>(a, blk, pages, head, true, tile); break;
      case 64: read_side<E, KIND, 64>(a, blk, pages, head, true, tile); break;
      default: read_side<E, KIND, 128>(a, blk, pages, head, true, tile); break;
    }
  }
}

template <typename E>
hipError_t run(const CacheArgs& a, int kind, bool write, dim3 grid, hipStream_t s) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
  };
  if (write) {
    if (kind == kCacheBf16) return go(cache_write_kernel<E, kCacheBf16>);
    if (kind == kCacheInt8) return go(cache_write_kernel<E, kCacheInt8>);
    return go(cache_write_kernel<E, kCacheE4m3>);
  }
  if (kind == kCacheBf16) return go(cache_read_kernel<E, kCacheBf16>);
  if (kind == kCacheInt8) return go(cache_read_kernel<E, kCacheInt8>);
  return go(cache_read_kernel<E, kCacheE4m3>);
}

}  // namespace

hipError_t launch_cache(CacheArgs a, int kind, int is_bf16, bool write, hipStream_t s) {
  if (a.total_tokens <= 0) return hipSuccess;
  a.items = a.total_tokens / kBlk + 2 * (int64_t)a.num_seqs;
  const dim3 grid((unsigned)min(a.items, (int64_t)1 << 22), (unsigned)a.num_heads);
  return is_bf16 ? run<uint16_t>(a, kind, write, grid, s) : run<float>(a, kind, write, grid, s);
}

}  // namespace hstu

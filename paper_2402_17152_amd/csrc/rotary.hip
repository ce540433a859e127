// Rotary positions of Q and K (include/hstu.h): the first 2 * half features of
// every head turn in pairs by position * inv_freq[m], forward and backward
// (the angle negated).
//
// HBM-bound: a row is read and written once.  The angles belong to a token, not
// to a head, so a workgroup takes `per` tokens, computes their cosines and
// sines once into LDS (fp64 angle, its whole turns taken off before the fp32
// sine and cosine: a position of 2^20 leaves an error of 2^-33 turns) and then
// walks the rows of all heads of Q and K, neighbouring lanes on neighbouring
// features.  52700 tokens of 8 heads of 64, bf16: 47 us, 4.6 TB/s (a large
// copy: 5.2); 45300 tokens of 4 heads of 128: 35 us, 5.2 TB/s; a token for each
// of 64 users: 3.3 us.
#include <algorithm>

#include "kernels.h"

namespace hstu {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;   // tokens of a workgroup (32: 50 and 38 us, 8: 47 and 36)
constexpr int kPairsLds = 2048;  // cosine and sine pairs it holds (16 KB)

template <typename E, int W>
struct alignas(sizeof(E) * W) Chunk {
  E v[W];
};

__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_bits_to_f32(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void from_f32(float x, uint16_t& o) { o = f32_to_bf16_bits(x); }
__device__ __forceinline__ void from_f32(float x, float& o) { o = x; }

// The sequence that owns packed row t: the last b in [0, B) with offs[b] <= t
// (0 for t < offs[0]).  t is the same in all 64 lanes, which probe 64 places
// at a time: one dependent load for B <= 64, two for B <= 4096.
__device__ __forceinline__ int find_seq(const int64_t* __restrict__ offs, int B, int64_t t) {
  const int lane = __lane_id();
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int at = lane * step;
    const uint64_t below = __ballot(at < n && offs[lo + (at < n ? at : 0)] <= t);
    const int last = below ? 63 - __builtin_clzll(below) : 0;
    lo += last * step;
    n = min(step, n - last * step);
  }
  return lo;
}

// E: storage type (bf16 bits or fp32); W: pairs a thread turns at once, the
// width of its two loads and two stores.
template <typename E, int W>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  // Units a thread has under way (1: 48 and 38 us, 4: 52 and 42; without the loads
  // ahead of the angles 54 and 40).
  constexpr int U = 2;
  __shared__ float2 turn[kPairsLds];
  __shared__ double pos[kMaxTokens];
  // a dimension of a grid holds 2^24 such workgroups
  const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.per;
  int64_t end = a.total_tokens;
  if (!a.positions) end = min(end, a.seq_offsets[a.num_seqs]);
  const int n = (int)min((int64_t)a.per, end - t0);
  if (n <= 0) return;
  const int units = a.d / (2 * W);        // two chunks of W features each
  const int turned = a.half / W;          // units that turn; the others are copied
  const int per_token = a.num_heads * units, per_side = n * per_token;
  const int total = per_side * ((a.src[0] != nullptr) + (a.src[1] != nullptr));
  struct Unit {
    int side, t, u, head, fa, fb;
    Chunk<E, W> x, y;
  };
  auto load = [&](int i, Unit& c) {
    if (i >= total) return;
    c.side = !a.src[0] || i >= per_side;
    if (i >= per_side) i -= per_side;
    c.t = i / per_token;
    const int r = i - c.t * per_token;
    c.head = r / units;
    c.u = r - c.head * units;
    if (c.u >= turned || a.interleaved) {
      c.fa = 2 * W * c.u;
      c.fb = c.fa + W;
    } else {
      c.fa = W * c.u;
      c.fb = a.half + W * c.u;
    }
    const E* s = (const E*)(c.side ? a.src[1] : a.src[0]) +
                 (t0 + c.t) * (c.side ? a.stride[1] : a.stride[0]) + c.head * a.d;
    c.x = *reinterpret_cast<const Chunk<E, W>*>(s + c.fa);
    c.y = *reinterpret_cast<const Chunk<E, W>*>(s + c.fb);
  };
  // The first rows are on their way while the angles are found.
  Unit c[U];
#pragma unroll
  for (int e = 0; e < U; e++) load(threadIdx.x + e * kThreads, c[e]);
  if (a.positions) {
    if ((int)threadIdx.x < n) pos[threadIdx.x] = (double)a.positions[t0 + threadIdx.x];
  } else {
    for (int t = threadIdx.x / 64; t < n; t += kThreads / 64) {
      const int b = find_seq(a.seq_offsets, a.num_seqs, t0 + t);
      int64_t x = t0 + t - a.seq_offsets[b];
      if (a.num_targets)
        x = min(x, a.seq_offsets[b + 1] - a.seq_offsets[b] - a.num_targets[b]);
      pos[t] = (double)x;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * a.half; i += kThreads) {
    const int t = i / a.half, m = i - t * a.half;
    const double turns = pos[t] * a.inv_freq[m] * 0.15915494309189535;  // 1 / (2 pi)
    const float f = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * f, &s, &c);
    turn[i] = float2{c * a.amplitude, (a.back ? -s : s) * a.amplitude};
  }
  __syncthreads();
  for (int i0 = threadIdx.x; i0 < total; i0 += U * kThreads) {
#pragma unroll
    for (int e = 0; e < U; e++) {
      if (i0 + e * kThreads >= total) break;
      auto x = c[e].x, y = c[e].y;
      if (c[e].u < turned) {
        const float2* cs = turn + c[e].t * a.half + W * c[e].u;
        E o[2 * W];
#pragma unroll
        for (int w = 0; w < W; w++) {
          const E ea = a.interleaved ? (2 * w < W ? x.v[2 * w % W] : y.v[2 * w % W]) : x.v[w];
          const E eb = a.interleaved ? (2 * w + 1 < W ? x.v[(2 * w + 1) % W] : y.v[(2 * w + 1) % W])
                                     : y.v[w];
          const float fa_ = to_f32(ea), fb_ = to_f32(eb);
          from_f32(fa_ * cs[w].x - fb_ * cs[w].y, o[2 * w]);
          from_f32(fa_ * cs[w].y + fb_ * cs[w].x, o[2 * w + 1]);
        }
#pragma unroll
        for (int w = 0; w < W; w++) {
          x.v[w] = a.interleaved ? o[w] : o[2 * w];
          y.v[w] = a.interleaved ? o[W + w] : o[2 * w + 1];
        }
      }
      E* dst = (E*)(c[e].side ? a.dst[1] : a.dst[0]) +
               ((t0 + c[e].t) * a.num_heads + c[e].head) * a.d;
      *reinterpret_cast<Chunk<E, W>*>(dst + c[e].fa) = x;
      *reinterpret_cast<Chunk<E, W>*>(dst + c[e].fb) = y;
    }
#pragma unroll
    for (int e = 0; e < U; e++) load(i0 + (U + e) * kThreads, c[e]);
  }
}

template <typename E, int W>
hipError_t run(const RotaryArgs& a, hipStream_t s) {
  const int64_t blocks = (a.total_tokens + a.per - 1) / a.per;
  const int64_t width = std::min(blocks, (int64_t)1 << 20);
  hipLaunchKernelGGL((rotary_kernel<E, W>),
                     dim3((unsigned)width, (unsigned)((blocks + width - 1) / width)),
                     dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int is_bf16, hipStream_t s) {
  if (a.total_tokens <= 0) return hipSuccess;
  // Few tokens: one a workgroup, so that all of the card takes part; many: the
  // cosines and sines of several at once, with more threads busy on them.
  a.per = 1;
  while (a.per < kMaxTokens && 2 * a.per * a.half <= kPairsLds && a.total_tokens / (2 * a.per) >= 1024)
    a.per *= 2;
  const int h = a.half;
  if (is_bf16) {
    if (h % 8 == 0) return run<uint16_t, 8>(a, s);
    if (h % 4 == 0) return run<uint16_t, 4>(a, s);
    if (h % 2 == 0) return run<uint16_t, 2>(a, s);
    return run<uint16_t, 1>(a, s);
  }
  if (h % 4 == 0) return run<float, 4>(a, s);
  if (h % 2 == 0) return run<float, 2>(a, s);
  return run<float, 1>(a, s);
}

}  // namespace hstu

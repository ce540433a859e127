// Rotary positions of Q and K (include/hstu.h): the first 2 * half features of
// every head turn in pairs by position * inv_freq[m], forward and backward
// (the angle negated).
//
// HBM-bound: a row is read and written once.  The angles belong to a token, not
// to a head, so a workgroup takes `per` tokens, computes their cosines and
// sines once into LDS (fp64 angle, its whole turns taken off before the fp32
// sine and cosine: a position of 2^20 leaves an error of 2^-33 turns) and then
// walks the rows of all heads of Q and K, neighbouring lanes on neighbouring
// features.
#include <algorithm>

#include "kernels.h"

namespace hstu {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 32;   // tokens of a workgroup
constexpr int kPairsLds = 2048;  // cosine and sine pairs it holds (16 KB)

template <typename E, int W>
struct alignas(sizeof(E) * W) Chunk {
  E v[W];
};

__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_bits_to_f32(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void from_f32(float x, uint16_t& o) { o = f32_to_bf16_bits(x); }
__device__ __forceinline__ void from_f32(float x, float& o) { o = x; }

// E: storage type (bf16 bits or fp32); W: pairs a thread turns at once, the
// width of its two loads and two stores.
template <typename E, int W>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  __shared__ float2 turn[kPairsLds];
  __shared__ double pos[kMaxTokens];
  // a dimension of a grid holds 2^24 such workgroups
  const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.per;
  int64_t end = a.total_tokens;
  if (!a.positions) end = min(end, a.seq_offsets[a.num_seqs]);
  const int n = (int)min((int64_t)a.per, end - t0);
  if (n <= 0) return;
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
  const int units = a.d / (2 * W);        // two chunks of W features each
  const int turned = a.half / W;          // units that turn; the others are copied
  const int per_token = a.num_heads * units;
  for (int side = 0; side < 2; side++) {
    const E* src = (const E*)a.src[side];
    if (!src) continue;
    E* dst = (E*)a.dst[side];
    for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
      const int t = i / per_token, r = i - t * per_token;
      const int head = r / units, u = r - head * units;
      int fa, fb;
      if (u >= turned || a.interleaved) {
        fa = 2 * W * u;
        fb = fa + W;
      } else {
        fa = W * u;
        fb = a.half + W * u;
      }
      const E* s = src + (t0 + t) * a.stride[side] + head * a.d;
      E* o = dst + ((t0 + t) * a.num_heads + head) * a.d;
      auto x = *reinterpret_cast<const Chunk<E, W>*>(s + fa);
      auto y = *reinterpret_cast<const Chunk<E, W>*>(s + fb);
      if (u < turned) {
        const float2* cs = turn + t * a.half + W * u;
        E e[2 * W];
#pragma unroll
        for (int w = 0; w < W; w++) {
          const E ea = a.interleaved ? (2 * w < W ? x.v[2 * w % W] : y.v[2 * w % W]) : x.v[w];
          const E eb = a.interleaved ? (2 * w + 1 < W ? x.v[(2 * w + 1) % W] : y.v[(2 * w + 1) % W])
                                     : y.v[w];
          const float fa_ = to_f32(ea), fb_ = to_f32(eb);
          from_f32(fa_ * cs[w].x - fb_ * cs[w].y, e[2 * w]);
          from_f32(fa_ * cs[w].y + fb_ * cs[w].x, e[2 * w + 1]);
        }
#pragma unroll
        for (int w = 0; w < W; w++) {
          x.v[w] = a.interleaved ? e[w] : e[2 * w];
          y.v[w] = a.interleaved ? e[W + w] : e[2 * w + 1];
        }
      }
      *reinterpret_cast<Chunk<E, W>*>(o + fa) = x;
      *reinterpret_cast<Chunk<E, W>*>(o + fb) = y;
    }
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

// Rotary positions of query and key rows.
//
// Dims are taken in pairs (x1, x2) -- (2i, 2i + 1) interleaved, else
// (i, i + rot / 2) -- and pair i < rot / 2 of a row at position p turns by
// the angle p * freqs[i]:
//   y1 = m (x1 cos - x2 sin),  y2 = m (x2 cos + x1 sin);
// the backward pass is the transposed map (the sine's sign changed); dims at
// and past rot are copied.
//
// The angle is formed in turns in float64 and reduced there (a position of
// 2^22 times a frequency of 1 leaves no correct digit of a turn in float32);
// sine and cosine of what is left are float32.
//
// One workgroup takes one token: its first wave computes the token's up to
// 64 sines and cosines once for all heads while the rows are on their way,
// then every thread turns 16 dims of a row at a time.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8.h"

namespace glide {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kThreads = 256;
constexpr int kPairs = kHeadDim / 2;

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

// Eight consecutive elements.
__device__ __forceinline__ void load8(float (&x)[8], const uint16_t* p) {
  const u32x4_t w = *(const u32x4_t*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(float (&x)[8], const float* p) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  *(u32x4_t*)p = w;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }

// Depth of node t: its ancestors, followed up by one lane (a chain of at most
// 63 parents; those outside [-1, node) count as -1).
__device__ __forceinline__ int depth_of(const int32_t* parents, int t) {
  int d = 0, n = t;
  while (true) {
    const int p = parents[n];
    if (p < 0 || p >= n) return d;
    n = p;
    ++d;
  }
}

// LAYOUT 0: pairs (2i, 2i + 1); 1: (i, i + rot / 2), both at multiples of 8;
// 2: (i, i + rot / 2) one by one.
template <class T, int LAYOUT>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, float sign) {
  const int t = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int half = a.rot / 2;
  __shared__ float2 cs[kPairs];
  if (tid < kPairs) {
    float c = 1.f, s = 0.f;
    if (tid < half) {
      int pos;
      if (a.positions) {
        pos = a.positions[(size_t)b * a.T + t];
      } else {
        pos = a.seq_lens ? a.seq_lens[b] : 0;
        pos += a.parents ? depth_of(a.parents + (size_t)b * a.T, t) : t;
      }
      const double turns = (double)pos * (a.freqs[tid] * 0.15915494309189533577);  // 1 / (2 pi)
      const float left = (float)(turns - rint(turns));
      sincospif(2.f * left, &s, &c);
      c *= a.mscale;
      s *= a.mscale * sign;
    }
    cs[tid] = make_float2(c, s);
  }
  __syncthreads();
  // item: 8 pairs of one row
  const int items = (a.q.H + a.k.H) * (kPairs / 8);
  for (int i = tid; i < items; i += kThreads) {
    int h = i / (kPairs / 8);
    const int p0 = i % (kPairs / 8) * 8;
    const bool is_k = h >= a.q.H;
    const RopeRows& r = is_k ? a.k : a.q;
    if (is_k) h -= a.q.H;
    const T* in = (const T*)r.in + b * r.in_sb + t * r.in_st + h * r.in_sh;
    T* out = (T*)r.out + b * r.out_sb + t * r.out_st + h * r.out_sh;
    float x1[8], x2[8];  // pair p0 + e
    int d1 = 0, d2 = 0;  // first dims of the two runs of eight
    if (LAYOUT == 0) {
      float lo[8], hi[8];
      d1 = 2 * p0, d2 = d1 + 8;
      load8(lo, in + d1);
      load8(hi, in + d2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x1[e] = lo[2 * e], x2[e] = lo[2 * e + 1];
        x1[4 + e] = hi[2 * e], x2[4 + e] = hi[2 * e + 1];
      }
    } else if (LAYOUT == 1) {
      d1 = p0 < half ? p0 : a.rot + 2 * (p0 - half);
      d2 = p0 < half ? p0 + half : d1 + 8;
      load8(x1, in + d1);
      load8(x2, in + d2);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + e;
        x1[e] = load1(in + (p < half ? p : 2 * p));
        x2[e] = load1(in + (p < half ? p + half : 2 * p + 1));
      }
    }
    float y1[8], y2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float2 w = cs[p0 + e];
      const bool turn = p0 + e < half;  // a copied dim may be infinite
      y1[e] = turn ? x1[e] * w.x - x2[e] * w.y : x1[e];
      y2[e] = turn ? x2[e] * w.x + x1[e] * w.y : x2[e];
    }
    if (LAYOUT == 0) {
      float lo[8], hi[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[2 * e] = y1[e], lo[2 * e + 1] = y2[e];
        hi[2 * e] = y1[4 + e], hi[2 * e + 1] = y2[4 + e];
      }
      store8(out + d1, lo);
      store8(out + d2, hi);
    } else if (LAYOUT == 1) {
      store8(out + d1, y1);
      store8(out + d2, y2);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int p = p0 + e;
        store1(out + (p < half ? p : 2 * p), y1[e]);
        store1(out + (p < half ? p + half : 2 * p + 1), y2[e]);
      }
    }
  }
}

template <class T>
hipError_t launch_type(const RopeArgs& a, bool interleaved, float sign, hipStream_t stream) {
  const dim3 grid(a.T, a.B), block(kThreads);
  if (interleaved)
    hipLaunchKernelGGL((rope_kernel<T, 0>), grid, block, 0, stream, a, sign);
  else if (a.rot % 16 == 0)
    hipLaunchKernelGGL((rope_kernel<T, 1>), grid, block, 0, stream, a, sign);
  else
    hipLaunchKernelGGL((rope_kernel<T, 2>), grid, block, 0, stream, a, sign);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, bool bf16, bool interleaved, bool backward, hipStream_t stream) {
  const float sign = backward ? -1.f : 1.f;
  return bf16 ? launch_type<uint16_t>(a, interleaved, sign, stream) : launch_type<float>(a, interleaved, sign, stream);
}

}  // namespace glide

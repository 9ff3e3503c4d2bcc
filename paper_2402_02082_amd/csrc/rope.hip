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
// One workgroup takes one to four tokens (enough rows for its threads): a wave
// computes a token's up to 64 sines and cosines once for all heads while the
// rows are on their way, then every thread turns two 16-byte pieces of a row at a
// time, which lie side by side across its lanes (two pieces of a lane side by side
// instead: 37 us).  Bound: the memory's copy rate (four 2048-token sequences of 40
// heads, 168 MB in 33 us, 5.1 TB/s); a decoding step's few rows take a launch,
// and a tree's one load more an ancestor.
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

// A 16-byte piece of a row: kPiece<T> elements as float32.
template <class T>
constexpr int kPiece = 16 / sizeof(T);

__device__ __forceinline__ void load_piece(float (&x)[8], const uint16_t* p) {
  const u32x4_t w = *(const u32x4_t*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load_piece(float (&x)[4], const float* p) {
  const float4 a = *(const float4*)p;
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
}
__device__ __forceinline__ void store_piece(uint16_t* p, const float (&x)[8]) {
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  *(u32x4_t*)p = w;
}
__device__ __forceinline__ void store_piece(float* p, const float (&x)[4]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
}

// Depth of node t: its ancestors, one load behind the other, followed up by every
// lane with an angle (at most 63; parents outside [-1, node) count as -1).  Nodes
// in one chain behind 512 tokens, 32 heads: five 3.3 us, 64 8.6; 64 roots 3.2.
__device__ __forceinline__ int depth_of(const int32_t* parents, int t) {
  int d = 0, n = t;
  while (true) {
    const int p = parents[n];
    if (p < 0 || p >= n) return d;
    n = p;
    ++d;
  }
}

// What a wave's lanes wrote to LDS before is there for its other lanes behind this.
__device__ __forceinline__ void wave_meets() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Two pieces of one row.  LAYOUT
//   0: pairs (2i, 2i + 1): piece j of either half of the row;
//   1: pairs (i, i + rot / 2) where the pieces of a pair's two dims are whole
//      (rot / 2 a multiple of a piece): V pairs from V j on, past rot / 2 two
//      pieces of copied dims;
//   2: the same pairs where they are not: pieces as in 0, and each dim finds the
//      other one of its pair in a copy of the row in LDS (element by element from
//      memory 120 us for 8192 tokens of 40 heads, now 34).
template <class T, int LAYOUT>
struct Item {
  static constexpr int V = kPiece<T>, kPerRow = kPairs / V;
  T* out;
  int d1, d2;
  float x1[V], x2[V];

  __device__ __forceinline__ void load(const RopeArgs& a, int b, int t, int i) {
    int h = i / kPerRow;
    const int j = i % kPerRow * V, half = a.rot / 2;
    const bool is_k = h >= a.q.H;
    const RopeRows& r = is_k ? a.k : a.q;
    if (is_k) h -= a.q.H;
    const T* in = (const T*)r.in + b * r.in_sb + t * r.in_st + h * r.in_sh;
    out = (T*)r.out + b * r.out_sb + t * r.out_st + h * r.out_sh;
    d1 = LAYOUT == 1 && j >= half ? 2 * j : j;
    d2 = LAYOUT == 1 ? (j < half ? j + half : 2 * j + V) : j + kPairs;
    load_piece(x1, in + d1);
    load_piece(x2, in + d2);
  }

  // `row`: the row's copy in LDS (LAYOUT 2).  Dims past rot are as they were,
  // infinities among them.
  __device__ __forceinline__ void turn_and_store(const float2* cs, int rot, float* row) {
    const int half = rot / 2;
    if (LAYOUT == 0) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        if (d1 + e < rot) turn(x1[e], x1[e + 1], cs[(d1 + e) / 2]);
        if (d2 + e < rot) turn(x2[e], x2[e + 1], cs[(d2 + e) / 2]);
      }
    } else if (LAYOUT == 1) {
      if (d1 < half)
#pragma unroll
        for (int e = 0; e < V; ++e) turn(x1[e], x2[e], cs[d1 + e]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) row[d1 + e] = x1[e], row[d2 + e] = x2[e];
      wave_meets();  // a row is one wave's
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x1[e] = turned(x1[e], d1 + e, cs, rot, half, row);
        x2[e] = turned(x2[e], d2 + e, cs, rot, half, row);
      }
      wave_meets();
    }
    store_piece(out + d1, x1);
    store_piece(out + d2, x2);
  }

  static __device__ __forceinline__ void turn(float& a, float& b, float2 w) {
    const float x = a;
    a = x * w.x - b * w.y;
    b = b * w.x + x * w.y;
  }

  static __device__ __forceinline__ float turned(float x, int d, const float2* cs, int rot, int half, const float* row) {
    if (d >= rot) return x;
    const bool first = d < half;
    const float2 w = cs[first ? d : d - half];
    const float y = row[first ? d + half : d - half];
    return first ? x * w.x - y * w.y : x * w.x + y * w.y;
  }
};

template <class T, int LAYOUT, int TOKENS>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, float sign) {
  typedef Item<T, LAYOUT> item_t;
  constexpr int kRowsAtOnce = LAYOUT == 2 ? kThreads / item_t::kPerRow : 1;
  const int b = blockIdx.y, tid = threadIdx.x;
  // the threads of a token; their number is a multiple of a wave's 64
  const int mine = tid / (kThreads / TOKENS), t = blockIdx.x * TOKENS + mine, at = tid % (kThreads / TOKENS);
  const int items = t < a.T ? (a.q.H + a.k.H) * item_t::kPerRow : 0;
  __shared__ float2 cs[TOKENS][kPairs];
  __shared__ float rows[kRowsAtOnce][kHeadDim + 1];
  item_t item;
  if (at < items) item.load(a, b, t, at);  // on its way while the angles are formed
  if (at < kPairs) {
    float c = 1.f, s = 0.f;
    if (at < a.rot / 2 && t < a.T) {
      int pos;
      if (a.positions) {
        pos = a.positions[(size_t)b * a.T + t];
      } else {
        pos = a.seq_lens ? a.seq_lens[b] : 0;
        pos += a.parents ? depth_of(a.parents + (size_t)b * a.T, t) : t;
      }
      const double turns = (double)pos * (a.freqs[at] * 0.15915494309189533577);  // 1 / (2 pi)
      const float left = (float)(turns - rint(turns));
      sincospif(2.f * left, &s, &c);
      c *= a.mscale;
      s *= a.mscale * sign;
    }
    cs[mine][at] = make_float2(c, s);
  }
  __syncthreads();
  for (int i = at; i < items; i += kThreads / TOKENS) {
    item.turn_and_store(cs[mine], a.rot, rows[LAYOUT == 2 ? tid / item_t::kPerRow : 0]);
    if (i + kThreads / TOKENS < items) item.load(a, b, t, i + kThreads / TOKENS);
  }
}

template <class T, int LAYOUT>
void launch_layout(const RopeArgs& a, float sign, hipStream_t stream) {
  const int items = (a.q.H + a.k.H) * Item<T, LAYOUT>::kPerRow;
  const dim3 block(kThreads);
  if (items <= kThreads / 4)
    hipLaunchKernelGGL((rope_kernel<T, LAYOUT, 4>), dim3((a.T + 3) / 4, a.B), block, 0, stream, a, sign);
  else if (items <= kThreads / 2)
    hipLaunchKernelGGL((rope_kernel<T, LAYOUT, 2>), dim3((a.T + 1) / 2, a.B), block, 0, stream, a, sign);
  else
    hipLaunchKernelGGL((rope_kernel<T, LAYOUT, 1>), dim3(a.T, a.B), block, 0, stream, a, sign);
}

template <class T>
hipError_t launch_type(const RopeArgs& a, bool interleaved, float sign, hipStream_t stream) {
  if (interleaved)
    launch_layout<T, 0>(a, sign, stream);
  else if (a.rot % (2 * kPiece<T>) == 0)
    launch_layout<T, 1>(a, sign, stream);
  else
    launch_layout<T, 2>(a, sign, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, bool bf16, bool interleaved, bool backward, hipStream_t stream) {
  const float sign = backward ? -1.f : 1.f;
  return bf16 ? launch_type<uint16_t>(a, interleaved, sign, stream) : launch_type<float>(a, interleaved, sign, stream);
}

}  // namespace glide

// Writing, reading and committing a key/value cache held in 8 bits.
//
// A block of 32 tokens of one head is quantised once, when its last token is
// final, K and V apart: with x the block's 32 x 128 bfloat16 values and M the
// largest magnitude of the type (448 for e4m3, 127 for int8),
//   scale = max |x| / M,   code = round to nearest even (x / scale),
// both quotients float32 (so the codes are a function of the inputs alone and
// equal on any side that divides).  Rows that are not final -- the tree rows
// of a verification step, and fewer than 32 accepted rows behind the last
// whole block -- stay bfloat16 in the ring, so a rejected token never touches
// a scale and nothing is quantised twice.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8.h"

namespace glide {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kThreads = 256;
constexpr int kChunks = kHeadDim / 8;  // 16-byte pieces of a bf16 row

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

// Scales below the smallest normal number count as 0: their block is zeros.
constexpr float kTinyScale = 1.17549435e-38f;

template <bool INT8>
__device__ __forceinline__ float scale_of(uint32_t amax_bits) {
  const float s = __uint_as_float(amax_bits << 16) / (INT8 ? 127.f : 448.f);
  return s < kTinyScale ? 0.f : s;
}

// Codes of four values (already divided), one byte each.
template <bool INT8>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  constexpr float kMost = INT8 ? 127.f : 448.f;
  a = fminf(fmaxf(a, -kMost), kMost), b = fminf(fmaxf(b, -kMost), kMost);
  c = fminf(fmaxf(c, -kMost), kMost), d = fminf(fmaxf(d, -kMost), kMost);
  if (INT8) {
    const uint32_t w = (uint32_t)((int)rintf(a) + 128) | (uint32_t)((int)rintf(b) + 128) << 8;
    return w | (uint32_t)((int)rintf(c) + 128) << 16 | (uint32_t)((int)rintf(d) + 128) << 24;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}

struct BlockLds {
  uint32_t amax[2][kThreads / 64];
  __attribute__((aligned(16))) uint8_t codes[kQ8BlockBytes];
};

// Quantises a block and writes it: the thread holds 16-byte chunks tid and
// tid + 256 (row chunk / 16, dims 8 (chunk % 16) ..) of K (x[0]) and V (x[1]).
// Called by the whole workgroup; the codes gather in LDS in the block's byte
// order and leave it 16 bytes a lane.
template <bool INT8>
__device__ __forceinline__ void quantise_block(const u32x4_t (&x)[2][2], uint8_t* block, float* scales, BlockLds& lds) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t top = 0;  // |x| as bits: their order is that of the magnitudes, NaN above all
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        top = max(top, x[m][j][e] & 0x7fffu);
        top = max(top, (x[m][j][e] >> 16) & 0x7fffu);
      }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((tid & 63) == 0) lds.amax[m][tid >> 6] = top;
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) top = max(top, lds.amax[m][w]);
    const float s = scale_of<INT8>(top);
    if (tid == 0) scales[m] = s;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int chunk = tid + kThreads * j, row = chunk / kChunks, dim = chunk % kChunks * 8;
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[2 * e] = s == 0.f ? 0.f : __uint_as_float(x[m][j][e] << 16) / s;
        y[2 * e + 1] = s == 0.f ? 0.f : __uint_as_float(x[m][j][e] & 0xffff0000u) / s;
      }
      const u32x2_t w = {codes4<INT8>(y[0], y[1], y[2], y[3]), codes4<INT8>(y[4], y[5], y[6], y[7])};
      if (m == 0) {
        *(u32x2_t*)(lds.codes + q8_k_byte(row, dim)) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          lds.codes[kQ8PartBytes + q8_v_byte(row, dim + e)] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const int at = m * kQ8PartBytes + tid * 16;
    *(u32x4_t*)(block + at) = *(const u32x4_t*)(lds.codes + at);
  }
}

__device__ __forceinline__ uint16_t* ring(const Q8Cache& c, size_t head, int m) {
  return c.tail + head * kQ8TailElems + m * (kQ8Tail * kHeadDim);
}

template <bool INT8, bool HOLD>
__global__ __launch_bounds__(kThreads) void q8_append_kernel(Q8AppendArgs a) {
  const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int cap = a.n_blocks * kQ8Block;
  const int L = min(max(a.seq_lens[b], 0), cap);
  int n = a.counts ? min(max(a.counts[b], 0), a.T) : a.T;
  if (!HOLD) n = min(n, cap - L);
  const int end = L + n;
  const size_t head = (size_t)b * a.H + h;
  const int64_t from = b * a.sb + h * a.sh;
  const int block = L / kQ8Block + i;
  if (!HOLD && (block + 1) * kQ8Block <= end) {
    __shared__ BlockLds lds;
    u32x4_t x[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int chunk = tid + kThreads * j, tok = block * kQ8Block + chunk / kChunks, dim = chunk % kChunks * 8;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const uint16_t* src = tok < L ? ring(a.cache, head, m) + (tok & (kQ8Tail - 1)) * kHeadDim
                                      : (m ? a.v : a.k) + from + (tok - L) * a.st;
        x[m][j] = *(const u32x4_t*)(src + dim);
      }
    }
    const size_t at = head * a.n_blocks + block;
    quantise_block<INT8>(x, a.cache.blocks + at * kQ8BlockBytes, a.cache.scales + at * 2, lds);
  }
  if (i > 0) return;
  // the rows behind the last whole block; the first block's workgroup writes
  // them, once it has read the ring rows that they may take the place of
  const int t0 = HOLD ? 0 : max(L, end / kQ8Block * kQ8Block) - L;
  __syncthreads();
  for (int u = tid; u < 2 * (n - t0) * kChunks; u += kThreads) {
    const int m = u & 1, t = t0 + (u >> 1) / kChunks, dim = (u >> 1) % kChunks * 8;
    const u32x4_t x = *(const u32x4_t*)((m ? a.v : a.k) + from + t * a.st + dim);
    *(u32x4_t*)(ring(a.cache, head, m) + ((L + t) & (kQ8Tail - 1)) * kHeadDim + dim) = x;
  }
}

template <bool INT8>
__device__ __forceinline__ float value_of(uint8_t code) {
  return INT8 ? (float)((int)code - 128) : __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  *(u32x4_t*)p = w;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(f32x4_t*)p = f32x4_t{x[0], x[1], x[2], x[3]};
  *(f32x4_t*)(p + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
}

template <bool INT8, class T>
__global__ __launch_bounds__(kThreads) void q8_read_kernel(Q8ReadArgs a) {
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int block = a.start / kQ8Block + blockIdx.x;
  const int L = min(max(a.seq_lens[b], 0), a.n_blocks * kQ8Block);
  const int first = block * kQ8Block;
  if (first >= L) return;  // rows behind the sequence stay as they are
  const size_t head = (size_t)b * a.H + h;
  const bool whole = first + kQ8Block <= L;
  __shared__ __attribute__((aligned(16))) uint8_t codes[kQ8BlockBytes];
  float s[2] = {0.f, 0.f};
  if (whole) {
    const size_t at = head * a.n_blocks + block;
    s[0] = a.cache.scales[at * 2], s[1] = a.cache.scales[at * 2 + 1];
#pragma unroll
    for (int m = 0; m < 2; ++m)
      *(u32x4_t*)(codes + m * kQ8PartBytes + tid * 16) =
          *(const u32x4_t*)(a.cache.blocks + at * kQ8BlockBytes + m * kQ8PartBytes + tid * 16);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = j >> 1, chunk = tid + kThreads * (j & 1), row = chunk / kChunks, dim = chunk % kChunks * 8;
    const int tok = first + row;
    if (tok < a.start || tok >= a.start + a.T || tok >= L) continue;
    float x[8];
    if (whole) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = value_of<INT8>(codes[m ? kQ8PartBytes + q8_v_byte(row, dim + e) : q8_k_byte(row, dim + e)]) * s[m];
    } else {
      const u32x4_t w = *(const u32x4_t*)(ring(a.cache, head, m) + (tok & (kQ8Tail - 1)) * kHeadDim + dim);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    }
    store8((T*)(m ? a.v_out : a.k_out) + (head * a.T + (tok - a.start)) * kHeadDim + dim, x);
  }
}

// The accepted path of (layer, head, sequence): with L the old length and a
// the accepted count, token L + d is the ring row of path node d.  Blocks that
// are whole with the new length are quantised straight from those rows; what
// is left behind them (at most 31 rows) moves to its place in the ring, all
// of it read before any of it is written.
template <bool INT8>
__global__ __launch_bounds__(kThreads) void q8_commit_kernel(Q8CommitArgs a) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const Q8Cache& cache = a.cache[blockIdx.z];
  const int cap = a.n_blocks * kQ8Block;
  const int L = min(max(a.seq_lens[b], 0), cap);
  const int n = min(min(max(a.accept_len[b], 0), a.N), cap - L);
  const int end = L + n;
  if (h == 0 && blockIdx.z == 0 && tid == 0) a.seq_lens_out[b] = end;
  if (n == 0) return;
  const size_t head = (size_t)b * a.H + h;
  const int32_t* path = a.path ? a.path + (size_t)b * a.N : nullptr;
  // ring row that holds token tok before the commit; nodes outside [0, N)
  // count as the chain's
  auto held = [&](int tok) {
    int d = tok - L;
    if (d >= 0 && path) {
      const int node = path[d];
      if (node >= 0 && node < a.N) d = node;
    }
    return (L + d) & (kQ8Tail - 1);
  };
  __shared__ BlockLds lds;
  const int whole = end / kQ8Block;
  for (int block = L / kQ8Block; block < whole; ++block) {
    u32x4_t x[2][2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int chunk = tid + kThreads * j, row = held(block * kQ8Block + chunk / kChunks), dim = chunk % kChunks * 8;
#pragma unroll
      for (int m = 0; m < 2; ++m) x[m][j] = *(const u32x4_t*)(ring(cache, head, m) + row * kHeadDim + dim);
    }
    const size_t at = head * a.n_blocks + block;
    quantise_block<INT8>(x, cache.blocks + at * kQ8BlockBytes, cache.scales + at * 2, lds);
    __syncthreads();  // lds is used again
  }
  const int first = max(L, whole * kQ8Block), rows = end - first;
  u32x4_t x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = tid + kThreads * j, m = u & 1, r = (u >> 1) / kChunks;
    if (r < rows) x[j] = *(const u32x4_t*)(ring(cache, head, m) + held(first + r) * kHeadDim + (u >> 1) % kChunks * 8);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int u = tid + kThreads * j, m = u & 1, r = (u >> 1) / kChunks;
    if (r < rows)
      *(u32x4_t*)(ring(cache, head, m) + ((first + r) & (kQ8Tail - 1)) * kHeadDim + (u >> 1) % kChunks * 8) = x[j];
  }
}

}  // namespace

hipError_t launch_q8_append(const Q8AppendArgs& a, bool int8, bool hold, hipStream_t stream) {
  const dim3 block(kThreads);
  if (hold) {
    hipLaunchKernelGGL((q8_append_kernel<false, true>), dim3(1, a.H, a.B), block, 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid((kQ8Block - 1 + a.T) / kQ8Block, a.H, a.B);
  if (int8)
    hipLaunchKernelGGL((q8_append_kernel<true, false>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_append_kernel<false, false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_q8_read(const Q8ReadArgs& a, bool int8, bool out_bf16, hipStream_t stream) {
  const dim3 block(kThreads);
  const dim3 grid((a.start % kQ8Block + a.T + kQ8Block - 1) / kQ8Block, a.H, a.B);
  if (int8 && out_bf16)
    hipLaunchKernelGGL((q8_read_kernel<true, uint16_t>), grid, block, 0, stream, a);
  else if (int8)
    hipLaunchKernelGGL((q8_read_kernel<true, float>), grid, block, 0, stream, a);
  else if (out_bf16)
    hipLaunchKernelGGL((q8_read_kernel<false, uint16_t>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_read_kernel<false, float>), grid, block, 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_q8_commit(const Q8CommitArgs& a, bool int8, hipStream_t stream) {
  const dim3 grid(a.H, a.B, a.layers), block(kThreads);
  if (int8)
    hipLaunchKernelGGL((q8_commit_kernel<true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_commit_kernel<false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace glide

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
//
// One wave takes K or V of a block, without barriers: its lanes load the values
// that their units of the block hold (K: 16 dims of a token; V: eight dims of
// eight tokens), so that the transposed V is a matter of byte order in registers,
// and every store is 1 KB in a row.  The waves of a workgroup take neighbouring
// heads, whose rows of a token lie together.  (A wave for both parts of a block:
// append 42 us where it takes 41.)
//
// Bound: the memory's copy rate.  Append, a prompt's 134 MB read and 67 written:
// 41 us, 4.9 TB/s, where a large copy reaches 5.1; the read-back is below.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "q8.h"

namespace glide {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kChunks = kHeadDim / 8;  // 16-byte pieces of a bf16 row

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The larger magnitude of each half, as bits (their order is that of the sizes,
// with NaN above all), and the maximum over a wave.
__device__ __forceinline__ uint32_t max_size(uint32_t top, uint32_t bf16s) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, top),
                                                                __builtin_bit_cast(u16x2_t, bf16s & 0x7fff7fffu)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_moved(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_moved<0x140>(max_moved<0x141>(max_moved<0x4E>(max_moved<0xB1>(v))));
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// x / scale, rounded like the division itself, for a whole block's x.  With the
// scale's rounded reciprocal, a first correction by the remainder brings the
// quotient within one unit of the last place, and a second one, whose remainder
// is exact then, gives the rounded quotient (Markstein, 1990; five operations a
// value where a division takes about ten).  A scale below the smallest normal
// number counts as 0.
struct Divider {
  float s, inv;
  __device__ __forceinline__ float operator()(float x) const {
    float q = x * inv;
    q = fmaf(fmaf(-q, s, x), inv, q);
    return fmaf(fmaf(-q, s, x), inv, q);
  }
};

// Codes of four values (already divided), one byte each.  A quotient passes the
// largest code by a few units of the last place at most, and rounds to it.
// int8: added to 1.5 * 2^23 + 128 a value is rounded to an integer, ties to even,
// which the sum's low byte holds.
template <bool INT8>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  if (INT8) {
    constexpr float kShift = 12583040.f;
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + kShift), __float_as_uint(a + kShift), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + kShift), __float_as_uint(c + kShift), 0x04000c0cu);
    return lo | hi;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w;
}

// Quantises and writes K or V of a block, called by a whole wave; at(t, d) is where
// token t's values from dim d on are.  Lane 16 g + c takes of K, for each (kt, h), token
// 16 kt + c, dims 64 h + 16 g + (0..15): x[4 kt + 2 h + half]; of V the tokens
// 16 (i / 4) + 4 g + i % 4, dims 8 c + (0..7): x[i].
template <bool INT8, class At>
__device__ __forceinline__ void quantise_part(bool v, int lane, uint8_t* part, float* scale_out, At at) {
  const int c = lane & 15, g = lane >> 4;
  u32x4_t x[8];
  if (v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = *(const u32x4_t*)at(16 * (i >> 2) + 4 * g + (i & 3), 8 * c);
  } else {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[4 * kt + i] = *(const u32x4_t*)at(16 * kt + c, 16 * g + 64 * (i >> 1) + 8 * (i & 1));
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max_size(top, x[i][e]);
  top = wave_max(max(top & 0xffffu, top >> 16));

  constexpr float kTiny = 1.17549435e-38f, kSmall = 8.67361738e-19f;  // 2^-126, 2^-60
  float scale = __uint_as_float(top << 16) / (INT8 ? 127.f : 448.f);
  if (scale < kTiny) scale = 0.f;
  if (lane == 0) *scale_out = scale;
  Divider d{scale, scale == 0.f ? 0.f : 1.f / scale};
  if (scale < kSmall && scale != 0.f) {
    // x and scale times 2^64, so that remainders are no denormals (of quotients
    // large enough for a code that is not 0)
    constexpr float kUp = 18446744073709551616.f;
    d = Divider{scale * kUp, 1.f / (scale * kUp)};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = pack_bf16x2(low_half(x[i][e]) * kUp, high_half(x[i][e]) * kUp);
  }

  if (v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      u32x4_t w;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t t0 = x[4 * j][u], t1 = x[4 * j + 1][u], t2 = x[4 * j + 2][u], t3 = x[4 * j + 3][u];
        w[j] = codes4<INT8>(d(low_half(t0)), d(low_half(t1)), d(low_half(t2)), d(low_half(t3)));
        w[2 + j] = codes4<INT8>(d(high_half(t0)), d(high_half(t1)), d(high_half(t2)), d(high_half(t3)));
      }
      *(u32x4_t*)(part + 1024 * u + 16 * lane) = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4_t w;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t lo = x[2 * i + (q >> 1)][2 * (q & 1)], hi = x[2 * i + (q >> 1)][2 * (q & 1) + 1];
        w[q] = codes4<INT8>(d(low_half(lo)), d(high_half(lo)), d(low_half(hi)), d(high_half(hi)));
      }
      *(u32x4_t*)(part + 1024 * i + 16 * lane) = w;
    }
  }
}

__device__ __forceinline__ uint16_t* ring(const Q8Cache& c, size_t head, int m) {
  return c.tail + head * kQ8TailElems + m * (kQ8Tail * kHeadDim);
}

// Final rows: workgroup (block of the call, four heads of K or V, sequence).
template <bool INT8>
__global__ __launch_bounds__(kThreads) void q8_append_kernel(Q8AppendArgs a) {
  const int i = blockIdx.x, b = blockIdx.z, lane = threadIdx.x & 63, m = blockIdx.y & 1;
  const int h = kWaves * (blockIdx.y >> 1) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (h >= a.H) return;
  const int cap = a.n_blocks * kQ8Block;
  const int L = min(max(a.seq_lens[b], 0), cap);
  const int n = min(a.counts ? min(max(a.counts[b], 0), a.T) : a.T, cap - L);
  const int end = L + n, block = L / kQ8Block + i;
  const size_t head = (size_t)b * a.H + h;
  const uint16_t* from = (m ? a.v : a.k) + b * a.sb + h * a.sh;
  uint16_t* held = ring(a.cache, head, m);
  if ((block + 1) * kQ8Block <= end) {
    const size_t at = head * a.n_blocks + block;
    quantise_part<INT8>(m, lane, a.cache.blocks + at * kQ8BlockBytes + m * kQ8PartBytes, a.cache.scales + at * 2 + m,
                        [&](int t, int d) {
                          const int tok = block * kQ8Block + t;
                          return (tok < L ? held + (tok & (kQ8Tail - 1)) * kHeadDim : from + (tok - L) * a.st) + d;
                        });
  }
  if (i > 0) return;
  // The rows behind the last whole block; the wave of the first block writes
  // them, behind its own reads of ring rows that they may take the place of.
  const int t0 = max(L, end / kQ8Block * kQ8Block) - L;
  for (int u = lane; u < (n - t0) * kChunks; u += 64) {
    const int t = t0 + u / kChunks, dim = u % kChunks * 8;
    *(u32x4_t*)(held + ((L + t) & (kQ8Tail - 1)) * kHeadDim + dim) = *(const u32x4_t*)(from + t * a.st + dim);
  }
}

// Tree rows: one 16-byte piece a thread, the heads of a token together.
__global__ __launch_bounds__(kThreads) void q8_hold_kernel(Q8AppendArgs a) {
  const int b = blockIdx.y, u = blockIdx.x * kThreads + threadIdx.x;
  const int dim = u % kChunks * 8, m = u / kChunks & 1, h = u / (2 * kChunks) % a.H, t = u / (2 * kChunks) / a.H;
  const int n = a.counts ? min(a.counts[b], a.T) : a.T;
  if (t >= n) return;
  const int L = min(max(a.seq_lens[b], 0), a.n_blocks * kQ8Block);
  const u32x4_t x = *(const u32x4_t*)((m ? a.v : a.k) + b * a.sb + t * a.st + h * a.sh + dim);
  *(u32x4_t*)(ring(a.cache, (size_t)b * a.H + h, m) + ((L + t) & (kQ8Tail - 1)) * kHeadDim + dim) = x;
}

template <bool INT8>
__device__ __forceinline__ float value_of(uint8_t code) {
  return INT8 ? (float)((int)code - 128) : __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

// A 16-byte piece of an output row.
__device__ __forceinline__ void store_piece(uint16_t* p, const float (&x)[8]) {
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  *(u32x4_t*)p = w;
}
__device__ __forceinline__ void store_piece(float* p, const float (&x)[4]) { *(f32x4_t*)p = f32x4_t{x[0], x[1], x[2], x[3]}; }

// Workgroup (block, head, sequence): the codes change order in LDS, so that every
// store takes whole rows (from the lanes' own units K would go out in pieces of 32
// bytes: 43 us for 32750 tokens of eight heads; with a wave a block 41; now 37,
// 201 MB at 5.4 TB/s).
template <bool INT8, class T>
__global__ __launch_bounds__(kThreads) void q8_read_kernel(Q8ReadArgs a) {
  constexpr int V = 16 / sizeof(T), kPieces = kHeadDim / V;  // dims of a piece, pieces of a row
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
  constexpr int kTurns = kQ8Block * kPieces / kThreads;  // of K, and of V
#pragma unroll
  for (int j = 0; j < 2 * kTurns; ++j) {
    const int m = j / kTurns, piece = tid + kThreads * (j % kTurns), row = piece / kPieces, dim = piece % kPieces * V;
    const int tok = first + row;
    if (tok < a.start || tok >= a.start + a.T || tok >= L) continue;
    float x[V];
    if (whole) {
#pragma unroll
      for (int e = 0; e < V; ++e)
        x[e] = value_of<INT8>(codes[m ? kQ8PartBytes + q8_v_byte(row, dim + e) : q8_k_byte(row, dim + e)]) * s[m];
    } else {
      const uint16_t* w = ring(a.cache, head, m) + (tok & (kQ8Tail - 1)) * kHeadDim + dim;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const uint32_t two = *(const uint32_t*)(w + e);
        x[e] = low_half(two), x[e + 1] = high_half(two);
      }
    }
    store_piece((T*)(m ? a.v_out : a.k_out) + (head * a.T + (tok - a.start)) * kHeadDim + dim, x);
  }
}

// The accepted path of (layer, head, sequence), a wave for K and one for V: with L
// the old length and n the accepted count, token L + d is the ring row of path
// node d.  Blocks that are whole with the new length are quantised straight from
// those rows; what is left behind them (at most 31 rows) moves to its place in
// the ring, all of it read before any of it is written.
//
// Bound: the latency of the waves that quantise (lengths, rows, codes: about 4 us),
// of which a 13B target's 40 layers have 1.6 rounds at eight a SIMD: 42 MB in
// 12.9 us (17.8 with K and V in one wave, 13.6 in 167 registers, three a SIMD).
template <bool INT8>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(8))) void q8_commit_kernel(Q8CommitArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  const int id = kWaves * blockIdx.x + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = id >> 1, m = id & 1;
  const Q8Cache& cache = a.cache[blockIdx.z];
  const int on_path = a.path ? a.path[(size_t)b * a.N + min(lane, a.N - 1)] : lane;
  const int len = a.seq_lens[b], accepted = a.accept_len[b];
  // node at each depth; nodes outside [0, N) count as the chain's
  const int node = lane < a.N && on_path >= 0 && on_path < a.N ? on_path : lane;
  const int cap = a.n_blocks * kQ8Block;
  const int L = __builtin_amdgcn_readfirstlane(min(max(len, 0), cap));
  const int n = __builtin_amdgcn_readfirstlane(min(min(max(accepted, 0), a.N), cap - L));
  const int end = L + n;
  if (id == 0 && blockIdx.z == 0 && lane == 0) a.seq_lens_out[b] = end;
  if (n == 0 || h >= a.H) return;
  const size_t head = (size_t)b * a.H + h;
  uint16_t* rows = ring(cache, head, m);
  // ring row that holds token tok before the commit (called by whole waves)
  auto held = [&](int tok) {
    const int moved = __shfl(node, (tok - L) & 63);
    return (tok < L ? tok : L + moved) & (kQ8Tail - 1);
  };
  const int whole = end / kQ8Block;
  for (int block = L / kQ8Block; block < whole; ++block) {
    const size_t at = head * a.n_blocks + block;
    quantise_part<INT8>(m, lane, cache.blocks + at * kQ8BlockBytes + m * kQ8PartBytes, cache.scales + at * 2 + m,
                        [&](int t, int d) { return rows + (unsigned)(held(block * kQ8Block + t) * kHeadDim + d); });
  }
  // The rows left, four a load; a path that starts down the chain keeps the rows
  // that are in place.
  const int first = max(L, whole * kQ8Block), left = end - first;
  const int dim = lane % kChunks * 8, q = lane / kChunks;
  u32x4_t x[kQ8Block / 4];
  bool moves[kQ8Block / 4];
#pragma unroll
  for (int j = 0; j < kQ8Block / 4; ++j) {
    if (4 * j >= left) break;
    const int tok = first + 4 * j + q, source = held(tok);
    moves[j] = 4 * j + q < left && source != (tok & (kQ8Tail - 1));
    if (moves[j]) x[j] = *(const u32x4_t*)(rows + (unsigned)(source * kHeadDim + dim));
  }
#pragma unroll
  for (int j = 0; j < kQ8Block / 4; ++j) {
    if (4 * j >= left) break;
    if (moves[j]) *(u32x4_t*)(rows + (unsigned)(((first + 4 * j + q) & (kQ8Tail - 1)) * kHeadDim + dim)) = x[j];
  }
}

}  // namespace

hipError_t launch_q8_append(const Q8AppendArgs& a, bool int8, bool hold, hipStream_t stream) {
  const dim3 block(kThreads);
  if (hold) {
    const unsigned pieces = (unsigned)a.T * a.H * 2 * kChunks;
    hipLaunchKernelGGL(q8_hold_kernel, dim3((pieces + kThreads - 1) / kThreads, a.B), block, 0, stream, a);
    return hipGetLastError();
  }
  const dim3 grid((kQ8Block - 1 + a.T) / kQ8Block, 2 * ((a.H + kWaves - 1) / kWaves), a.B);
  if (int8)
    hipLaunchKernelGGL((q8_append_kernel<true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_append_kernel<false>), grid, block, 0, stream, a);
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
  const dim3 grid((2 * a.H + kWaves - 1) / kWaves, a.B, a.layers), block(kThreads);
  if (int8)
    hipLaunchKernelGGL((q8_commit_kernel<true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_commit_kernel<false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace glide

// Attention of a few query rows against a key/value cache held in 8 bits
// (q8.h), under the tree mask of a verification step or over the prefix alone.
//
//   out = SoftMax(scale Q K^T + mask) V,   K, V = code * scale of its block
// for the tokens of whole blocks, and the ring's bfloat16 rows for those
// behind them and for the tree.
//
// Work decomposition.  The query rows of a cached head (N rows of each of the
// H / H_kv query heads that share it) are cut into groups of up to 32, its keys
// into units of 32 tokens: the whole blocks, then the ring's rows.  Each pair
// (sequence, cached head) is split into as many runs of units as its length
// asks for, so that all runs of a call are of about the same size whatever the
// sequences' lengths; a workgroup takes one run.  A pair of one run is finished
// there; of the others each run leaves a state, counts itself in, and the one
// that completes the pair joins the states in order, whichever that is: one
// launch.
// A workgroup's waves (eight or four) take units in turn, each for all of the
// group's rows.  Groups of one run lie on the same XCD, so that all but one of them
// read its keys from L2 (64 rows in one workgroup instead, four waves for each half:
// 166 us where two groups take 145, 622 and 454 for long contexts).
//
// Per unit and wave, on v_mfma_f32_16x16x32:
//   S^T[key, query] = K Q^T, softmax on S^T with one query per lane column,
//   O^T[dim, query] += V^T P^T with P^T straight from the S^T registers.
// A code is exact in fp16, so both products of a block run on fp16 operands:
//  * q enters as fp16 of q * 2^(14 - e) with e the exponent of the row's
//    largest value: a bfloat16 has 8 significant bits, so what is lost are
//    values 2^-38 of that one; K's scale and 2^(e - 14) multiply the score;
//  * P enters as fp16 of p * s * c, s the block's V scale and c a factor of
//    the query row that keeps the largest of these products at 2^7 .. 2^15.
//    It moves up only when one passes 2^15 (like the running maximum, c moves
//    rarely), so a product keeps 11 bits down to 2^-21 of the largest.  With
//    bfloat16 the rounding of P alone is as far off as that of the output.
//    c ends at 2^126; where it would pass that, the accumulators fall instead.
// Ring rows are bfloat16: their products take bfloat16 operands, P as the sum
// of two.  Sums, maxima and outputs are float32.
//
// Bound: the memory where keys are long (sixteen sequences of 16 to 32 thousand
// tokens, 32 heads, five rows: 3.23 GB in 465 us, 6.9 TB/s; the matrix cores busy
// a tenth of it).  Short ones take 7 to 9 us more than a plain stream of their
// bytes: 1.3 until a workgroup knows its run, 2 until queries and first blocks are
// there, 1 for the join of the waves and as much for their different ends, 1 to
// count a run in and 2 to join those of a pair (four sequences of 40 heads, 32 tree
// rows, 110 MB: 25.4 us; sixteen sequences, four query heads to each of eight
// cached ones, 168 MB: 32.4).  A 7B layer's chain of five behind 512 tokens takes
// 6.1 us.  Code that runs once costs as much as the trips to memory it waits for:
// what is rare stands apart, and little is unrolled outside the loop over blocks.
// Several groups of rows are bound by the conversions, the softmax and the matrix
// instructions in turn (eight sequences of 52 heads, 64 tree rows, 677 MB: 145 us,
// 4.7 TB/s; the vector units busy half of it, the matrix cores a quarter).
// Many short pairs pay what lies around the stream once for every 256 of them (32
// sequences of 52 heads, one row, 100 tokens, 46 MB: 46 us).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "q8.h"

namespace glide {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

constexpr int kD = kHeadDim;

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum and sum over the four 16-lane groups that hold a query column.
__device__ __forceinline__ float max_across_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_across_groups(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2_t));
}
__device__ __forceinline__ f16x8_t as_f16x8(u32x4_t v) { return __builtin_bit_cast(f16x8_t, v); }
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t v) { return __builtin_bit_cast(bf16x8_t, v); }

// Eight codes (two dwords) as fp16 values.
//   e4m3: the conversion instruction, two at a time.
//   int8: a byte u = value + 128 under the exponent of 1024 is the fp16 number
//   1024 + u; less 1152 it is the value.
template <bool INT8>
__device__ __forceinline__ u32x4_t decode8(uint32_t lo, uint32_t hi) {
  u32x4_t r;
  if (INT8) {
    const f16x2_t off = {(_Float16)1152.f, (_Float16)1152.f};
    const uint32_t w[4] = {__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u),
                           __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u),
                           __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u),
                           __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)};
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, w[e]) - off);
  } else {
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
  }
  return r;
}

// The larger magnitude of each half, as bits (their order is that of the sizes).
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
__device__ __forceinline__ uint32_t max_size(uint32_t top, uint32_t bf16s) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, top),
                                                                __builtin_bit_cast(u16x2_t, bf16s & 0x7fff7fffu)));
}
__device__ __forceinline__ uint32_t larger_half(uint32_t v) { return max(v & 0xffffu, v >> 16); }

// Maximum over a wave: within the 16-lane rows (neighbours, pairs, half mirror,
// mirror), then across them.
template <int CTRL>
__device__ __forceinline__ uint32_t max_moved(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_moved<0x140>(max_moved<0x141>(max_moved<0x4E>(max_moved<0xB1>(v))));
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// Ancestor-or-self mask of node `lane` (bit m: node m) from its parent, by
// pointer doubling; parents outside [-1, lane) count as -1.  Called by a whole
// wave.
__device__ __forceinline__ uint64_t ancestor_mask(int p, int lane) {
  if (p < -1 || p >= lane) p = -1;
  uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
  for (int round = 0; round < 6 && __any(p >= 0); ++round) {
    const int src = p < 0 ? lane : p;
    const uint32_t l = __shfl(lo, src), u = __shfl(hi, src);
    const int up = __shfl(p, src);
    if (p >= 0) lo |= l, hi |= u, p = up;
  }
  return ((uint64_t)hi << 32) | lo;
}

constexpr int kRingCost = 4;  // blocks that take a wave about as long as a unit of ring rows

constexpr float kRescaleSlack = 8.f;  // how far a score may pass the reference maximum (log2)
constexpr float kProductTop = 15.f;   // log2 of a product p * s * c at which c moves,
constexpr float kProductAim = 7.f;    // and of where the largest is put
constexpr float kFactorMost = 126.f;  // log2 of c at most
constexpr float kNoFactor = 1e30f;

// State of one query row (lane column) over the keys that its wave has seen.
struct RowState {
  float m;   // reference maximum of the scaled scores (log2 units); -inf: none
  float l;   // sum of 2^(score - m) over this lane's keys
  float c;   // accumulators are sums of 2^(score - m) * c * value; 0: none but zeros yet
  float lc;  // log2 of c; kNoFactor: c is 0
};

// Turns the raw scores x[8] of a unit (masked ones -inf), to be multiplied by
// k >= 0, into 2^(x k - m), moving m and c where needed; ls is log2 of the
// size of the unit's values (a code counts as 1).
__device__ __forceinline__ void softmax_unit(float (&x)[8], RowState& st, f32x4_t (&acc)[8], float k, float ls) {
  float mx = __builtin_elementwise_maximum(
      __builtin_elementwise_maximum(__builtin_elementwise_maximum(x[0], x[1]), x[2]),
      __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_elementwise_maximum(x[3], x[4]), x[5]),
                                    __builtin_elementwise_maximum(x[6], x[7])));
  mx *= k;
  if (__any(mx > st.m + kRescaleSlack)) {
    const float m_new = fmaxf(st.m, max_across_groups(mx));
    if (st.m != neg_inf()) {
      st.l *= fast_exp2(st.m - m_new);
      if (st.lc != kNoFactor) {
        // c grows as the weights of earlier keys fall, and the accumulators stay;
        // where it would pass its most (values below about 2^-100) they fall
        const float lc = st.lc + (m_new - st.m);
        st.lc = fminf(lc, kFactorMost);
        st.c = fast_exp2(st.lc);
        if (lc > kFactorMost) {
          const float r = fast_exp2(kFactorMost - lc);
#pragma unroll
          for (int t = 0; t < 8; ++t) acc[t] *= r;
        }
      }
    }
    st.m = m_new;
  }
  const float m_ref = st.m == neg_inf() ? 0.f : st.m;
  if (__any((mx - m_ref) + (ls + st.lc) > kProductTop)) {
    const float col = max_across_groups(mx) - m_ref;
    if (col + (ls + st.lc) > kProductTop) {
      const float lc = fminf(kProductAim - col - ls, kFactorMost);
      const float r = st.lc == kNoFactor ? 0.f : fast_exp2(lc - st.lc);
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= r;
      st.lc = lc;
      st.c = fast_exp2(lc);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fast_exp2(fmaf(x[i], k, -m_ref));
  st.l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// Infinities and NaN of a unit's values reach only the rows that see them.  They
// are taken out of the eight tokens w of a V^T operand (0 times infinity would be
// NaN), and rows that see one get an infinity of its sign added (of both signs for
// NaN, which gives NaN): ones in pos and neg mark them.
__device__ __forceinline__ void take_not_finite(u32x4_t& w, u32x4_t& pos, u32x4_t& neg) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    pos[e] = neg[e] = 0;
#pragma unroll
    for (int hi = 0; hi < 32; hi += 16) {
      const uint32_t y = (w[e] >> hi) & 0xffffu;
      if ((y & 0x7f80u) == 0x7f80u) {
        const bool nan = y & 0x7fu;
        if (nan || !(y & 0x8000u)) pos[e] |= 0x3f80u << hi;
        if (nan || (y & 0x8000u)) neg[e] |= 0x3f80u << hi;
        w[e] &= ~(0xffffu << hi);
      }
    }
  }
}
// What a query column gets added; seen: bit per token of the lane.
__device__ __forceinline__ f32x4_t add_not_finite(u32x4_t pos, u32x4_t neg, uint32_t seen) {
  u32x4_t vis;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    vis[e] = ((seen >> (2 * e)) & 1 ? 0x3f80u : 0u) | ((seen >> (2 * e + 1)) & 1 ? 0x3f800000u : 0u);
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  const f32x4_t up = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(pos), as_bf16x8(vis), zero, 0, 0, 0);
  const f32x4_t dn = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(neg), as_bf16x8(vis), zero, 0, 0, 0);
  f32x4_t add;
#pragma unroll
  for (int r = 0; r < 4; ++r) add[r] = (up[r] > 0.f ? -neg_inf() : 0.f) + (dn[r] > 0.f ? neg_inf() : 0.f);
  return add;
}

// A block's codes as they lie in memory: four 1 KB loads of K, four of V.
struct RawUnit {
  u32x4_t k[4], v[4];
};

// Buffer descriptor of one block, empty where the unit is past the last: such
// loads return zeros without touching memory, so the pipeline needs no guard.
constexpr int kBufferDesc3 = 0x00020000;  // 32-bit data, raw addressing
__device__ __forceinline__ __amdgpu_buffer_rsrc_t unit_rsrc(const uint8_t* blocks, int u, int u_end) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(blocks) + (size_t)u * kQ8BlockBytes, (short)0,
                                           u < u_end ? kQ8BlockBytes : 0, kBufferDesc3);
}
// Cache policy of these loads: non-temporal where every byte is read once.
constexpr int kKeep = 0, kStream = 2;
template <int CPOL>
__device__ __forceinline__ void load_k(RawUnit& f, __amdgpu_buffer_rsrc_t r, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f.k[i] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16 + 1024 * i, 0, CPOL));
}
template <int CPOL>
__device__ __forceinline__ void load_v(RawUnit& f, __amdgpu_buffer_rsrc_t r, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f.v[i] = __builtin_bit_cast(
        u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16 + kQ8PartBytes + 1024 * i, 0, CPOL));
}

// Tokens of sequence b, and units of a sequence of L tokens.  One without keys
// counts as one unit, so that some workgroup writes its zeros.
__device__ __forceinline__ int tokens(const Q8AttnArgs& a, int b) {
  return min(max(a.seq_lens[b], 0), a.n_blocks * kQ8Block);
}
__device__ __forceinline__ int units_of(const Q8AttnArgs& a, bool tree, int L) {
  return max(1, (L + (tree ? a.N : 0) + kQ8Block - 1) / kQ8Block);
}

// Inclusive sum over a wave, by moves inside and across its 16-lane rows.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int scan64(int v) {
  v = add_moved<0x111, 0xF>(v);  // one, two, four, eight lanes up
  v = add_moved<0x112, 0xF>(v);
  v = add_moved<0x114, 0xF>(v);
  v = add_moved<0x118, 0xF>(v);
  v = add_moved<0x142, 0xA>(v);  // row 0's and 2's last lane to the row behind
  return add_moved<0x143, 0xC>(v);  // lane 31 to the upper half
}

// The run of a workgroup: units [u0, u1) of (b, hk) with L tokens, the first of
// `n` runs of that pair being number `first` and the others a.H_kv apart.
struct Run {
  int b, hk, L, u0, u1, n, first;
};

// Runs of a pair of so many units: of up to `per` units each, and no more than the
// root of units * a.join_ratio, where joining another run takes as long as it saves.
__device__ __forceinline__ int runs_of(const Q8AttnArgs& a, int units, int per) {
  if (a.splits) return a.splits;
  const int most = (int)__builtin_amdgcn_sqrtf((float)units * a.join_ratio);
  return units <= a.whole_units ? 1 : min((units + per - 1) / per, max(most, 1));
}

// Units of sequence b, 0 past the last; `mine`: of the lane's among the first 64.
__device__ __forceinline__ int units_at(const Q8AttnArgs& a, bool tree, int b, int lane, int mine) {
  return b == lane ? mine : (b < a.B ? units_of(a, tree, tokens(a, b)) : 0);
}

// Sum over all sequences of their units (per == 0) or runs.  Called by whole
// waves; sequences are looked through 64 at a time, one a lane.
__device__ __forceinline__ int sum_of(const Q8AttnArgs& a, bool tree, int per, int lane, int mine) {
  int sum = 0;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    const int units = units_at(a, tree, b0 + lane, lane, mine);
    sum += per == 0 || units == 0 ? units : runs_of(a, units, per);
  }
  return __builtin_amdgcn_readlane(scan64(sum), 63);
}

// Run number `run`; false past the last.  Called by whole waves.  Each lane has
// the length of one of the first 64 sequences, so that most calls read the lengths
// once.
__device__ __forceinline__ bool find_run(const Q8AttnArgs& a, bool tree, int run, int lane, Run* r) {
  int b = 0, before = 0, per = 1;
  int len = 0;
  if (a.B > 1) len = tokens(a, min(lane, a.B - 1));
  if (a.splits) {
    b = run / (a.splits * a.H_kv);
    if (b >= a.B) return false;
    before = b * a.splits * a.H_kv;
    if (a.splits == 1 && a.B >= 2 && a.B <= 64) {
      // the b-th longest sequence (of equals the first): the longest start first,
      // and the shorter ones fill in as CUs come free
      int rank = 0;
      for (int j = 0; j < a.B; ++j) {
        const int lj = __builtin_amdgcn_readlane(len, j);
        rank += lj > len || (lj == len && j < lane);
      }
      b = __ffsll((long long)__ballot(lane < a.B && rank == b)) - 1;
    }
  } else if (a.B == 1) {
    const int units = units_of(a, tree, __builtin_amdgcn_readfirstlane(tokens(a, 0)));
    const int n = max(1, a.target / a.H_kv);
    per = max((units + n - 1) / n, a.min_units);
  } else {
    // about the fewest units a run with which no more than `most` runs come out;
    // n pairs of any lengths have about n / 2 runs more than whole ones would be
    const int mine = lane < a.B ? units_of(a, tree, len) : 0;
    const int total = sum_of(a, tree, 0, lane, mine) * a.H_kv;
    const int most = total >= a.target * a.long_run ? a.target : (a.target + 1) / 2;
    const int whole = max(1, most - a.B * a.H_kv / 2);
    per = max((total + whole - 1) / whole, a.min_units);
    for (int i = 0; i < 16 && sum_of(a, tree, per, lane, mine) * a.H_kv > most; ++i) per += (per + 7) / 8;
    int sum = 0;
    bool found = false;
    for (int b0 = 0; b0 < a.B && !found; b0 += 64) {
      const int units = units_at(a, tree, b0 + lane, lane, mine);
      const int n = units ? runs_of(a, units, per) * a.H_kv : 0;
      const int incl = sum + scan64(n);
      const uint64_t hit = __ballot(run < incl);
      found = hit != 0;
      const int l = found ? __ffsll((long long)hit) - 1 : 63;
      b = b0 + l;
      before = __builtin_amdgcn_readlane(incl - n, l);
      sum = __builtin_amdgcn_readlane(incl, 63);
    }
    if (!found) return false;
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int L = __builtin_amdgcn_readfirstlane(a.B > 1 && a.B <= 64 ? __builtin_amdgcn_readlane(len, b) : tokens(a, b));
  const int units = units_of(a, tree, L);
  const int n = runs_of(a, units, per), rest = run - before, i = rest / a.H_kv;
  if (i >= n) return false;  // (a single sequence: past its last run)
  const int size = (units + n - 1) / n;
  r->b = b, r->hk = rest - i * a.H_kv, r->L = L, r->n = n, r->first = before + r->hk;
  r->u0 = min(units, i * size), r->u1 = min(units, r->u0 + size);
  return true;
}

// States are written and read with the device-scope cache policy (sc1), so that
// the joining workgroup sees them whichever XCD wrote them.
constexpr int kDeviceScope = 16;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t state_rsrc(void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, (short)0, bytes, kBufferDesc3);
}

// Counts a run's state in once its stores have completed at device scope;
// true in the workgroup that completes the pair (which resets the counter).
__device__ __forceinline__ bool last_to_arrive(unsigned* counter, int n, int* flag) {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const bool last = before == (unsigned)(n - 1);
    if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last;
  }
  __syncthreads();
  return *flag != 0;
}

constexpr int kPitch = kD + 4;  // floats between LDS rows, so that rows start in other banks
template <int WAVES, int ROWS>  // query rows of a wave
struct JoinLds {
  float m[WAVES][ROWS], l[WAVES][ROWS];
  __attribute__((aligned(16))) float o[WAVES][ROWS][kPitch];
  int flag;
};

// 1 / sum of a row's probabilities; 0 where it saw no key, and NaN stays.
__device__ __forceinline__ float reciprocal(float l) { return l > 0.f ? __builtin_amdgcn_rcpf(l) : (l == 0.f ? 0.f : l); }

// Maximum and sum of a row over the waves.
template <int WAVES, class Lds>
__device__ __forceinline__ void join_sums(const Lds& lds, int row, float& M, float& L) {
  float m[WAVES], l[WAVES];
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m[w] = lds.m[w][row], l[w] = lds.l[w][row];
  M = m[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) M = fmaxf(M, m[w]);
  const float ref = M == neg_inf() ? 0.f : M;
  L = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) L += fast_exp2(m[w] - ref) * l[w];
}

// The states of a pair joined in run order into output rows.  State i of n is in
// the slot of its run, first + i * H_kv; `rows` of the group's kRows are in use.
// 16 lanes take a row, so a wave takes four at a time; where the rows do not fill
// the waves, several waves share a row's states.  Bound: two trips to memory, and
// that of the code itself, which runs once: with 8 states a batch 13B's two and
// three runs take 0.7 us more, with 16 1.5.
template <int WAVES, int kRows, class Lds>
__device__ __forceinline__ void join_states(const Q8AttnArgs& a, int first, int n, int grp, int rows, uint16_t* out,
                                            int row_first, int G, Lds& lds) {
  constexpr int kBatch = 4;  // states; two batches are requested at once
  // All states: at most 2048 pairs and groups of 64 runs, so 2^31 bytes; past them
  // nothing is read and zeros come back.
  constexpr unsigned kNowhere = 0xC0000000u;
  const __amdgpu_buffer_rsrc_t rm = state_rsrc(a.part_ml, a.runs * a.groups * (kRows * 8));
  const __amdgpu_buffer_rsrc_t ro = state_rsrc(a.part_o, (unsigned)(a.runs * a.groups) * (kRows * kD * 4u));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int quads = (rows + 3) / 4;
  const int parts = quads == 1 ? WAVES : (quads == 2 ? WAVES / 2 : (quads <= 4 ? WAVES / 4 : 1));  // waves that share a row
  const int part = wave % parts, d = lane % 16 * 8;
  // waves that share rows meet at a barrier, so all of them take one turn, with
  // rows past the last (zeros, by the descriptors) or without
  for (int quad = wave / parts; quad < (parts > 1 ? WAVES / parts : quads); quad += WAVES / parts) {
    const int row = 4 * quad + lane / 16;
    const bool live = row < rows;
    float M = neg_inf(), L = 0.f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
    const unsigned ml_at = row * 8, o_at = (row * kD + d) * 4;
    f32x2_t ml[2][kBatch];
    f32x4_t x[2][kBatch][2];
    auto request = [&](int half, int s0) {
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = s0 + j * parts;
        const unsigned at = (unsigned)((first + i * a.H_kv) * a.groups + grp) * kRows;
        ml[half][j] = __builtin_bit_cast(
            f32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rm, (i < n ? at * 8 : kNowhere) + ml_at, 0, kDeviceScope));
#pragma unroll
        for (int h = 0; h < 2; ++h)
          x[half][j][h] = __builtin_bit_cast(
              f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ro, (i < n ? at * kD * 4 : kNowhere) + o_at + 16 * h, 0,
                                                             kDeviceScope));
      }
    };
    auto join = [&](int half) {
      float m = M;
#pragma unroll
      for (int j = 0; j < kBatch; ++j)  // sum 0: it saw no key, or there is none
        m = ml[half][j][1] == 0.f ? m : fmaxf(m, ml[half][j][0]);
      const float ref = m == neg_inf() ? 0.f : m, keep = fast_exp2(M - ref);
      M = m, L *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= keep;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const float w = ml[half][j][1] == 0.f ? 0.f : fast_exp2(ml[half][j][0] - ref) * ml[half][j][1];
        L += w;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(w, x[half][j][e >> 2][e & 3], o[e]);
      }
    };
    for (int s0 = part; s0 < n; s0 += 2 * kBatch * parts) {
      const bool more = s0 + kBatch * parts < n;
      request(0, s0);
      if (more) request(1, s0 + kBatch * parts);
      join(0);
      if (more) join(1);
    }
    if (parts > 1) {  // up to 16 rows
      const int slot = row;
      lds.m[part][slot] = M, lds.l[part][slot] = L;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *(f32x4_t*)&lds.o[part][slot][d + 4 * h] = f32x4_t{o[4 * h], o[4 * h + 1], o[4 * h + 2], o[4 * h + 3]};
      __syncthreads();
      M = neg_inf(), L = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = 0.f;
      for (int p = 0; p < parts; ++p) M = fmaxf(M, lds.m[p][slot]);
      for (int p = 0; p < parts; ++p) {
        if (lds.l[p][slot] == 0.f) continue;
        const float w = fast_exp2(lds.m[p][slot] - (M == neg_inf() ? 0.f : M));
        L += w * lds.l[p][slot];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += w * lds.o[p][slot][d + e];
      }
    }
    if (live && part == 0) {
      const float inv = reciprocal(L);
      const int r = row_first + row, node = r / G;
      u32x4_t w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
      *(u32x4_t*)(out + ((size_t)node * a.H + (r - node * G)) * kD + d) = w;
    }
  }
}

// SHARED: several groups read the same keys.
template <int WAVES, int NT, bool SHARED, bool INT8, bool TREE>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2)))
void q8_attn_kernel(Q8AttnArgs a) {
  constexpr int kThreads = 64 * WAVES;
  constexpr int kStages = NT == 1 ? 2 : 1;
  constexpr int kPolicy = SHARED ? kKeep : kStream;
  constexpr int kRows = 16 * NT;  // query rows of a workgroup
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups go to the eight XCDs in turn; the groups of a run are eight apart, on
  // the same XCD and so on the same L2, which they share its keys in.  The last
  // runs, fewer than eight, have their groups on all XCDs.
  int grp = 0, run = blockIdx.x;
  if (SHARED) {
    const int even = a.runs / 8 * 8, id = blockIdx.x, rest = id - even * a.groups;
    grp = rest < 0 ? id / 8 % a.groups : rest / (a.runs - even);
    run = rest < 0 ? id / (8 * a.groups) * 8 + id % 8 : even + rest % (a.runs - even);
  }
  const int G = a.G, R = a.N * G, row0 = grp * kRows;
  __shared__ JoinLds<WAVES, kRows> lds;

  // Query rows: row r is node r / G of query head hk * G + r % G.  MFMA step
  // 2 h + e holds dims 64 h + 16 g + 8 e + (0..7).  A single sequence's are
  // requested before its length is known.
  int node[NT], q_row[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const unsigned r = row0 + 16 * nt + c < R ? row0 + 16 * nt + c : 0;  // rows past the last: copies of the first
    node[nt] = r / (unsigned)G;
    q_row[nt] = node[nt] * (a.H - G) + r;
  }
  u32x4_t qf[NT][4];
  auto load_queries = [&](int b, int hk) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint16_t* q = a.q + ((size_t)b * a.N * a.H + q_row[nt] + hk * G) * kD;
#pragma unroll
      for (int st = 0; st < 4; ++st) qf[nt][st] = *(const u32x4_t*)(q + 64 * (st >> 1) + 16 * g + 8 * (st & 1));
    }
  };
  if (a.B == 1) load_queries(0, run % a.H_kv);

  Run rn;
  if (!find_run(a, TREE, run, lane, &rn)) return;
  const int b = rn.b, hk = rn.hk, u0 = rn.u0, u1 = rn.u1;
  const int L = rn.L, end = L + (TREE ? a.N : 0);
  const int whole = L / kQ8Block;
  const size_t head = (size_t)b * a.H_kv + hk;
  const uint8_t* blocks = a.cache.blocks + head * a.n_blocks * (size_t)kQ8BlockBytes;
  const float* scales = a.cache.scales + head * a.n_blocks * 2;

  // The run's units among the waves.  The last waves take one ring unit each
  // (a ring holds at most 95 rows, three units); the blocks go in turn, but that
  // waves without a ring unit take kRingCost of them before.
  static_assert(WAVES > 3, "a ring unit a wave");
  const int ue = min(u1, whole), ring_units = max(0, u1 - max(u0, whole));
  const bool ring = wave >= WAVES - ring_units;
  const int early_waves = ring_units ? WAVES - ring_units : 0, turns = u0 + early_waves * kRingCost;
  int u = early_waves && !ring ? u0 + wave : turns + wave;
  auto next = [&](int at) {
    const int more = at + early_waves;
    return at >= turns ? at + WAVES : (more < turns ? more : turns + wave);
  };
  RawUnit raw[kStages];
  float2 unit_scale[kStages];  // of K, of V
  auto load_scale = [&](int at) { return *(const float2*)(scales + 2 * min(at, a.n_blocks - 1)); };
  auto prefetch = [&] {
#pragma unroll
    for (int i = 0; i < kStages; ++i) {
      const int at = i ? next(u) : u;
      unit_scale[i] = load_scale(at);
      const __amdgpu_buffer_rsrc_t r = unit_rsrc(blocks, at, ue);
      load_k<kPolicy>(raw[i], r, lane);
      load_v<kPolicy>(raw[i], r, lane);
    }
  };
  if (a.B > 1) load_queries(b, hk);

  const int j0 = (max(u0, whole) + WAVES - 1 - wave) * kQ8Block;  // the ring unit's first token
  int parent = -1;
  u32x4_t kf[2][4], v[8];
  auto load_ring = [&] {
    if (TREE) parent = a.parents[(size_t)b * a.N + min(lane, a.N - 1)];
    const uint16_t* kt_rows = a.cache.tail + head * kQ8TailElems + (j0 & (kQ8Tail - 1)) * kD;
    const uint16_t* vt_rows = kt_rows + kQ8Tail * kD;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int st = 0; st < 4; ++st)
        kf[kt][st] = *(const u32x4_t*)(kt_rows + (16 * kt + c) * kD + 64 * (st >> 1) + 16 * g + 8 * (st & 1));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *(const u32x4_t*)(vt_rows + (16 * (i >> 2) + 4 * g + (i & 3)) * kD + 8 * c);
  };

  // Ring rows are requested first, since what is waited for comes back in order,
  // and the first blocks behind them; a wave with registers for one stage only
  // requests the blocks behind the ring rows' scores.
  constexpr bool kTogether = kStages > 1;
  if (kTogether && ring) load_ring();
  if (kTogether || !ring) prefetch();

  RowState sm[NT];
  f32x4_t acc[NT][8];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    sm[nt] = RowState{neg_inf(), 0.f, 0.f, kNoFactor};
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[nt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // Ring rows, taken first.
  if (ring) {
    if (!kTogether) load_ring();
    uint32_t top = 0;  // the largest size of the unit's values
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] &= j0 + 16 * (i >> 2) + 4 * g + (i & 3) < end ? ~0u : 0u;  // rows that hold no token: zeros
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max_size(top, v[i][e]);
    }
    top = larger_half(top);
    const bool odd = __any(top >= 0x7f80u);  // an infinity or NaN among them
    if (odd) {
      top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = v[i][e] & 0x7fffu, hi = (v[i][e] >> 16) & 0x7fffu;
          top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
        }
    }
    // (the logarithm takes a subnormal number for zero, so they count as the least normal one)
    top = wave_max(top);
    if (top != 0) top = max(top, 0x80u);
    const float ls = __builtin_amdgcn_logf(__uint_as_float(top << 16)) - 8.f;  // as if the largest were a code of 256
    uint64_t mine = 0;  // ancestor mask of node `lane`
    if (TREE) mine = ancestor_mask(lane < a.N ? parent : -1, lane);
    u32x4_t vt[8];  // V^T operands: tile t holds dim 8 c + t of the lane's eight tokens
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        vt[2 * w][e] = __builtin_amdgcn_perm(v[2 * e + 1][w], v[2 * e][w], 0x05040100u);
        vt[2 * w + 1][e] = __builtin_amdgcn_perm(v[2 * e + 1][w], v[2 * e][w], 0x07060302u);
      }
    f32x4_t s[2][NT];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st)
          x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[kt][st]), as_bf16x8(qf[nt][st]), x, 0, 0, 0);
        s[kt][nt] = x;
      }
    if (!kTogether) prefetch();
    u32x4_t ph[NT], pl[NT];
    uint32_t seen[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      uint64_t anc = 0;
      if (TREE)
        anc = ((uint64_t)(uint32_t)__shfl((uint32_t)(mine >> 32), node[nt]) << 32) | (uint32_t)__shfl((uint32_t)mine, node[nt]);
      float x[8];
      seen[nt] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = j0 + 16 * (i >> 2) + 4 * g + (i & 3);
        uint32_t vis = j < L;
        if (TREE) vis |= (uint32_t)(anc >> ((j - L) & 63)) & (uint32_t)(j >= L) & (uint32_t)(j < end);
        seen[nt] |= vis << i;
        x[i] = vis ? s[i >> 2][nt][i & 3] : neg_inf();
      }
      softmax_unit(x, sm[nt], acc[nt], a.scale_log2, ls);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = x[2 * e] * sm[nt].c, p1 = x[2 * e + 1] * sm[nt].c;
        ph[nt][e] = pack_bf16x2(p0, p1);
        pl[nt][e] = pack_bf16x2(p0 - __uint_as_float(ph[nt][e] << 16), p1 - __uint_as_float(ph[nt][e] & 0xffff0000u));
      }
    }
    if (odd) {
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        u32x4_t pos, neg;
        take_not_finite(vt[t], pos, neg);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[nt][t] += add_not_finite(pos, neg, seen[nt]);
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt[t]), as_bf16x8(ph[nt]), acc[nt][t], 0, 0, 0);
        acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vt[t]), as_bf16x8(pl[nt]), acc[nt][t], 0, 0, 0);
      }
  }

  // From here on q is fp16: of q * 2^(14 - e), e the exponent of the row's largest.
  float qscale[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    uint32_t top = 0;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max_size(top, qf[nt][st][e]);
    const float col = max_across_groups(__uint_as_float(min(larger_half(top), 0x7f7fu) << 16));
    const int ex = max((int)(__float_as_uint(col) >> 23), 15);  // biased exponent; q * 2^(141 - ex) is below 2^15
    const float up = __uint_as_float((uint32_t)(268 - ex) << 23);
    qscale[nt] = a.scale_log2 * __uint_as_float((uint32_t)(ex - 14) << 23);
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        qf[nt][st][e] = pack_f16x2(__uint_as_float(qf[nt][st][e] << 16) * up, __uint_as_float(qf[nt][st][e] & 0xffff0000u) * up);
  }

  // Blocks: a stage is loaded again as soon as its codes have been converted.
  while (u < ue) {
#pragma unroll
    for (int stage = 0; stage < kStages; ++stage) {
      if (u < ue) {
        const float ks = unit_scale[stage].x, vs = unit_scale[stage].y;
        const int further = kStages == 1 ? next(u) : next(next(u));
        unit_scale[stage] = load_scale(further);
        const __amdgpu_buffer_rsrc_t ahead = unit_rsrc(blocks, further, ue);
        RawUnit& f = raw[stage];
        f32x4_t s[2][NT];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          u32x4_t kf[4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            kf[2 * h] = decode8<INT8>(f.k[2 * kt + h][0], f.k[2 * kt + h][1]);
            kf[2 * h + 1] = decode8<INT8>(f.k[2 * kt + h][2], f.k[2 * kt + h][3]);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < 4; ++st)
              x = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(kf[st]), as_f16x8(qf[nt][st]), x, 0, 0, 0);
            s[kt][nt] = x;
          }
        }
        load_k<kPolicy>(f, ahead, lane);
        u32x4_t vf[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vf[2 * i] = decode8<INT8>(f.v[i][0], f.v[i][1]);
          vf[2 * i + 1] = decode8<INT8>(f.v[i][2], f.v[i][3]);
        }
        load_v<kPolicy>(f, ahead, lane);
        const float ls = __builtin_amdgcn_logf(vs);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[8];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * kt + r] = s[kt][nt][r];
          softmax_unit(x, sm[nt], acc[nt], qscale[nt] * ks, ls);
          const float w = vs * sm[nt].c;
          u32x4_t pf;
#pragma unroll
          for (int e = 0; e < 4; ++e) pf[e] = pack_f16x2(x[2 * e] * w, x[2 * e + 1] * w);
#pragma unroll
          for (int t = 0; t < 8; ++t)
            acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(vf[t]), as_f16x8(pf), acc[nt][t], 0, 0, 0);
        }
        u = next(u);
      }
    }
  }

  // The waves' states join in LDS: first maxima and sums, then every wave's output
  // times 2^(m - M) / (c L), to be added up.  Lane (c, g) holds row c of each
  // tile, dims 32 g + 8 r + t.
  const bool finished = rn.n == 1;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = sum_across_groups(sm[nt].l);
    if (g == 0) lds.m[wave][16 * nt + c] = sm[nt].m, lds.l[wave][16 * nt + c] = l;
  }
  __syncthreads();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float M, Lsum;
    join_sums<WAVES>(lds, 16 * nt + c, M, Lsum);
    const float part = (sm[nt].m == neg_inf() ? 0.f : fast_exp2(sm[nt].m - M)) * reciprocal(Lsum);
    const float unit = sm[nt].lc == kNoFactor ? 0.f : fast_exp2(-sm[nt].lc);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < 8; t += 4) {
        f32x4_t o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = acc[nt][t + e][r] * part * unit;
        *(f32x4_t*)&lds.o[wave][16 * nt + c][32 * g + 8 * r + t] = o;
      }
  }
  __syncthreads();
  {
    constexpr int kTPR = kThreads / kRows, kDims = kD / kTPR;  // threads a row, dims a thread
    const int in = tid / kTPR, d = tid % kTPR * kDims, r = grp * kRows + in;
    f32x4_t o[kDims / 4];
#pragma unroll
    for (int i = 0; i < kDims / 4; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
#pragma unroll
      for (int i = 0; i < kDims / 4; ++i) o[i] += *(const f32x4_t*)&lds.o[w][in][d + 4 * i];
    if (r < R && finished) {
      const int n = r / G;
      uint16_t* dst = a.out + (((size_t)b * a.N + n) * a.H + hk * G + (r - n * G)) * kD + d;
#pragma unroll
      for (int i = 0; i < kDims / 4; ++i)
        *(u32x2_t*)(dst + 4 * i) = u32x2_t{pack_bf16x2(o[i][0], o[i][1]), pack_bf16x2(o[i][2], o[i][3])};
    } else if (r < R) {
      const size_t at = ((size_t)run * a.groups + grp) * kRows;
      if (d == 0) {
        float M, Lsum;
        join_sums<WAVES>(lds, in, M, Lsum);
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2_t, f32x2_t{M, Lsum}),
                                              state_rsrc(a.part_ml + at, kRows * 8), in * 8, 0, kDeviceScope);
      }
      const __amdgpu_buffer_rsrc_t ro = state_rsrc(a.part_o + at * kD, kRows * kD * 4);
#pragma unroll
      for (int i = 0; i < kDims / 4; ++i)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, o[i]), ro, (in * kD + d + 4 * i) * 4, 0,
                                               kDeviceScope);
    }
  }
  if (finished) return;
  unsigned* counter = a.counters + (head * a.groups + grp) * kCounterStride;
  if (last_to_arrive(counter, rn.n, &lds.flag))
    join_states<WAVES, kRows>(a, rn.first, rn.n, grp, min(kRows, R - grp * kRows),
                       a.out + ((size_t)b * a.N * a.H + hk * G) * kD, grp * kRows, G, lds);
}

template <int WAVES, int NT, bool SHARED>
hipError_t launch_rows(const Q8AttnArgs& a, bool int8, hipStream_t stream) {
  const dim3 grid((unsigned)((long)a.runs * a.groups)), block(64 * WAVES);
  if (a.parents && int8)
    hipLaunchKernelGGL((q8_attn_kernel<WAVES, NT, SHARED, true, true>), grid, block, 0, stream, a);
  else if (a.parents)
    hipLaunchKernelGGL((q8_attn_kernel<WAVES, NT, SHARED, false, true>), grid, block, 0, stream, a);
  else if (int8)
    hipLaunchKernelGGL((q8_attn_kernel<WAVES, NT, SHARED, true, false>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_attn_kernel<WAVES, NT, SHARED, false, false>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

Q8AttnPlan plan_q8_attn(int B, int N, int H, int H_kv, int n_blocks, int max_splits) {
  Q8AttnPlan p{};
  const int R = N * (H / H_kv);
  p.rows = R <= 16 ? 16 : 32;
  p.groups = (R + p.rows - 1) / p.rows;
  p.waves = 8;
  const long pairs = (long)B * H_kv, most = n_blocks + (kQ8Block - 1 + N + kQ8Block - 1) / kQ8Block;
  const long wgs = pairs * p.groups;  // one a pair and group
  // Enough for every CU: nothing is split (nor past the counters).
  if (max_splits == 1 || most == 1 || wgs > (max_splits ? kCounterSlots : kNumCU - 1)) {
    // Several groups of more workgroups than CUs: four waves, two a CU (8 sequences
    // of 52 heads, 64 rows: 145 us, with eight waves 158; 16 of 8 heads, 128 pairs of
    // two groups: 57.5 and 45.8).  One group reads each key once and keeps eight
    // (8 sequences of 40 heads, 32 rows: 41.3 us, with four 44.9).
    if (p.groups > 1 && wgs > kNumCU) p.waves = 4;
    p.splits = 1;
    p.runs = pairs;
    return p;
  }
  // Up to 16 rows of few pairs take four waves, two workgroups a CU; all others
  // eight, one a CU (32 rows of 16 long pairs with four: 62 us, with eight 45).
  const bool few = wgs <= kNumCU / 2;
  if (p.rows == 16 && few) p.waves = 4;
  if (max_splits > 0) {
    p.splits = (int)min((long)max_splits, most);
    p.runs = pairs * p.splits;
  } else {
    // Joining runs takes 3 us, so short pairs are not split, and where workgroups
    // take more than half of the CUs only those that are long for their call are
    // (one sequence of 32 heads, five rows, 25 units: 6.9 us whole, 8.0 in three runs;
    // of 40 heads, 32 rows: 32 units 12.3 and 12.9 in two, 48 units 14.8 and 13.2 in
    // three).
    p.whole_units = few ? (p.waves == 4 ? 28 : 40) : 48;
    p.min_units = p.waves == 4 ? 8 : 16;
    // Up to one run a CU (7B layer of 2048 tokens: 8 runs a pair 9.3 us, 9 11.1; one
    // head group of 60000 tokens, 32 runs a pair 24.5, 63 26.6); of four waves and
    // sequences that may differ in length two, from 32 units a run on (sixteen
    // sequences of 64 to 256 units, 8 heads: 33.1 us, with one run a CU 34.4; where
    // all are 160 long 32.3 and 31.5).
    const bool two = p.waves == 4 && B > 1;
    p.target = max(1, (two ? 2 : 1) * kNumCU / p.groups);
    p.long_run = two ? 32 : 0;
    // One pair of 16000 tokens, 32 rows: 12 to 16 runs 18.8 us, 32 21.4; of 60000
    // 32 runs 27.2, 64 33.0; one row of 30000 tokens 32 runs 12.8, 64 13.5, 128 17.7.
    p.join_ratio = p.waves == 4 ? 2.5f : 0.5f;
    p.runs = max(pairs, min(pairs + p.target, pairs * ((most + p.min_units - 1) / p.min_units)));
    if (most <= p.whole_units) return p;  // no pair will be split: no states
  }
  const size_t states = (size_t)p.runs * p.groups * p.rows;
  p.part_ml_off = kCounterBytes;
  p.part_o_off = (p.part_ml_off + states * sizeof(float2) + 255) & ~(size_t)255;
  p.ws_bytes = p.part_o_off + states * kD * sizeof(float);
  return p;
}

hipError_t launch_q8_attn(const Q8AttnArgs& a, bool int8, int rows, int waves, hipStream_t stream) {
  if (rows == 16) return waves == 4 ? launch_rows<4, 1, false>(a, int8, stream) : launch_rows<8, 1, false>(a, int8, stream);
  if (a.groups == 1) return launch_rows<8, 2, false>(a, int8, stream);
  return waves == 4 ? launch_rows<4, 2, true>(a, int8, stream) : launch_rows<8, 2, true>(a, int8, stream);
}

}  // namespace glide

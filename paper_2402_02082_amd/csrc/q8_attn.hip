// Attention of a few query rows against a key/value cache held in 8 bits
// (q8.h), under the tree mask of a verification step or over the prefix alone.
//
//   out = SoftMax(scale Q K^T + mask) V,   K, V = code * scale of its block
// for the tokens of whole blocks, and the ring's bfloat16 rows for those
// behind them and for the tree.
//
// Work decomposition: the query rows of a cached head (N rows of each of the
// H / H_kv query heads that share it) are cut into groups of up to 64, the
// keys into units of 32 tokens -- the whole blocks, then the ring's rows --
// and the units into splits.  One workgroup of four waves takes one split of
// one group; its waves take units in turn, each for all of the group's rows,
// so a byte of the cache is fetched and converted by one wave.
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
// Ring rows are bfloat16: their products take bfloat16 operands, P as the sum
// of two.  Sums, maxima and outputs are float32.
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
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

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

// Ancestor-or-self mask of node `lane` (bit m: node m), by pointer doubling;
// parents outside [-1, lane) count as -1.  Called by a whole wave.
__device__ __forceinline__ uint64_t ancestor_mask(const int32_t* parents, int N, int lane) {
  int p = lane < N ? parents[lane] : -1;
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

constexpr float kRescaleSlack = 8.f;     // log2: how far a score may pass the reference maximum
constexpr float kProductTop = 32768.f;   // a product p * s * c at which c moves
constexpr float kProductAim = 128.f;     // and where the largest is put
constexpr float kFactorMost = 8.507e37f;  // c at most 2^126

// State of one query row (lane column) over the keys that its wave has seen.
struct RowState {
  float m;  // reference maximum of the scaled scores (log2 units); -inf: none
  float l;  // sum of 2^(score - m) over this lane's keys
  float c;  // accumulators are sums of 2^(score - m) * c * value; 0: none but zeros yet
};

// Turns the scores x[8] of a unit (masked ones -inf) into 2^(x - m), moving m
// and c where needed; s is the size of the unit's values (a code counts as 1).
__device__ __forceinline__ void softmax_unit(float (&x)[8], RowState& st, f32x4_t (&acc)[8], float s) {
  float mx = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = __builtin_elementwise_maximum(mx, x[i]);
  if (__any(mx > st.m + kRescaleSlack)) {
    const float m_new = fmaxf(st.m, max_across_groups(mx));
    if (st.m != neg_inf()) {
      st.l *= fast_exp2(st.m - m_new);
      st.c = fminf(st.c * fast_exp2(m_new - st.m), kFactorMost);
    }
    st.m = m_new;
  }
  const float m_ref = st.m == neg_inf() ? 0.f : st.m;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fast_exp2(x[i] - m_ref);
  st.l += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
  const float f = s * st.c;
  const float top = fast_exp2(mx - m_ref);
  if (__any(top * f > kProductTop || (st.c == 0.f && top > 0.f && s > 0.f))) {
    const float col = max_across_groups(top);
    if (col * f > kProductTop || (st.c == 0.f && col > 0.f && s > 0.f)) {
      const float c = fminf(kProductAim / col / s, kFactorMost);
      const float r = st.c > 0.f ? c / st.c : 0.f;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] *= r;
      st.c = c;
    }
  }
}

// Infinities and NaN of a unit's values reach only the rows that see them:
// takes them out of the eight tokens w of a V^T operand (0 times infinity would
// be NaN) and returns what rows that see one get added, an infinity of its sign
// (of both signs for NaN, which gives NaN).  seen: bit per token of the lane.
__device__ __forceinline__ f32x4_t add_not_finite(u32x4_t& w, uint32_t seen) {
  u32x4_t pos, neg, vis;
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
    vis[e] = ((seen >> (2 * e)) & 1 ? 0x3f80u : 0u) | ((seen >> (2 * e + 1)) & 1 ? 0x3f800000u : 0u);
  }
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  const f32x4_t up = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(pos), as_bf16x8(vis), zero, 0, 0, 0);
  const f32x4_t dn = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(neg), as_bf16x8(vis), zero, 0, 0, 0);
  f32x4_t add;
#pragma unroll
  for (int r = 0; r < 4; ++r) add[r] = (up[r] > 0.f ? -neg_inf() : 0.f) + (dn[r] > 0.f ? neg_inf() : 0.f);
  return add;
}

template <int NT, bool INT8, bool TREE>
__global__ __launch_bounds__(kThreads) void q8_attn_kernel(Q8AttnArgs a) {
  const int hk = blockIdx.x % a.H_kv, grp = blockIdx.x / a.H_kv, b = blockIdx.y, split = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.H / a.H_kv, R = a.N * G, row0 = grp * 16 * NT;
  const int cap = a.n_blocks * kQ8Block;
  const int L = __builtin_amdgcn_readfirstlane(min(max(a.seq_lens[b], 0), cap));
  const int end = L + (TREE ? a.N : 0);
  const int whole = L / kQ8Block, units = (end + kQ8Block - 1) / kQ8Block;
  const int per = (units + a.splits - 1) / a.splits;
  const int u0 = split * per, u1 = min(units, u0 + per);

  const size_t head = (size_t)b * a.H_kv + hk;
  const uint8_t* blocks = a.cache.blocks + head * a.n_blocks * (size_t)kQ8BlockBytes;
  const float* scales = a.cache.scales + head * a.n_blocks * 2;

  // Query rows: row r is node r / G of query head hk * G + r % G.
  const uint16_t* qrow[NT];
  bool live[NT];
  int node[NT];
  u32x4_t qf[NT][4];   // MFMA step 2 h + e: dims 64 h + 16 g + 8 e + (0..7)
  float qscale[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = row0 + 16 * nt + c;
    live[nt] = r < R;
    node[nt] = live[nt] ? r / G : 0;
    qrow[nt] = a.q + (((size_t)b * a.N + node[nt]) * a.H + hk * G + (live[nt] ? r % G : 0)) * kD;
    u32x4_t raw[4];
    uint32_t top = 0;
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      raw[st] = live[nt] ? *(const u32x4_t*)(qrow[nt] + 64 * (st >> 1) + 16 * g + 8 * (st & 1)) : u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, max(raw[st][e] & 0x7fffu, (raw[st][e] >> 16) & 0x7fffu));
    }
    const float col = max_across_groups(__uint_as_float(min(top, 0x7f7fu) << 16));
    const int ex = max((int)(__float_as_uint(col) >> 23), 15);  // biased exponent; q * 2^(141 - ex) is below 2^15
    const float up = __uint_as_float((uint32_t)(268 - ex) << 23);
    qscale[nt] = a.scale_log2 * __uint_as_float((uint32_t)(ex - 14) << 23);
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        qf[nt][st][e] = pack_f16x2(__uint_as_float(raw[st][e] << 16) * up, __uint_as_float(raw[st][e] & 0xffff0000u) * up);
  }

  RowState sm[NT];
  f32x4_t acc[NT][8];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    sm[nt] = RowState{neg_inf(), 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 8; ++t) acc[nt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  int u = u0 + wave;
  for (; u < min(u1, whole); u += kWaves) {
    const uint8_t* p = blocks + (size_t)u * kQ8BlockBytes + lane * 16;
    const float ks = scales[2 * u], vs = scales[2 * u + 1];
    u32x4_t kraw[4], vraw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) kraw[i] = *(const u32x4_t*)(p + 1024 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i) vraw[i] = *(const u32x4_t*)(p + kQ8PartBytes + 1024 * i);
    f32x4_t s[2][NT];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      u32x4_t kf[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4_t w = kraw[2 * kt + h];
        kf[2 * h] = decode8<INT8>(w[0], w[1]);
        kf[2 * h + 1] = decode8<INT8>(w[2], w[3]);
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
    u32x4_t vf[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      vf[2 * i] = decode8<INT8>(vraw[i][0], vraw[i][1]);
      vf[2 * i + 1] = decode8<INT8>(vraw[i][2], vraw[i][3]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float k = qscale[nt] * ks;
      float x[8];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) x[4 * kt + r] = s[kt][nt][r] * k;
      softmax_unit(x, sm[nt], acc[nt], vs);
      const float f = vs * sm[nt].c;
      u32x4_t pf;
#pragma unroll
      for (int e = 0; e < 4; ++e) pf[e] = pack_f16x2(x[2 * e] * f, x[2 * e + 1] * f);
#pragma unroll
      for (int t = 0; t < 8; ++t)
        acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_f16x8(vf[t]), as_f16x8(pf), acc[nt][t], 0, 0, 0);
    }
  }

  // At most one unit of ring rows a wave (a ring holds at most 95 rows).
  if (u < u1) {
    const int j0 = u * kQ8Block;
    const uint16_t* kt_rows = a.cache.tail + head * kQ8TailElems + (j0 & (kQ8Tail - 1)) * kD;
    const uint16_t* vt_rows = kt_rows + kQ8Tail * kD;
    u32x4_t kf[2][4], v[8];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int st = 0; st < 4; ++st)
        kf[kt][st] = *(const u32x4_t*)(kt_rows + (16 * kt + c) * kD + 64 * (st >> 1) + 16 * g + 8 * (st & 1));
    bool odd = false;  // a value that is not finite
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 16 * (i >> 2) + 4 * g + (i & 3);
      v[i] = *(const u32x4_t*)(vt_rows + row * kD + 8 * c);
      if (j0 + row >= end) v[i] = u32x4_t{0, 0, 0, 0};  // rows that hold no token
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = v[i][e] & 0x7fffu, hi = (v[i][e] >> 16) & 0x7fffu;
        odd |= max(lo, hi) >= 0x7f80u;
        top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
    }
    odd = __any(odd);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const float size = __uint_as_float(top << 16) * (1.f / 256);  // as if the largest value were a code of 256
    uint64_t mine = 0;  // ancestor mask of node `lane`
    if (TREE) mine = ancestor_mask(a.parents + (size_t)b * a.N, a.N, lane);
    u32x4_t vt[8];  // V^T operands: tile t holds dim 8 c + t of the lane's eight tokens
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        vt[2 * w][e] = __builtin_amdgcn_perm(v[2 * e + 1][w], v[2 * e][w], 0x05040100u);
        vt[2 * w + 1][e] = __builtin_amdgcn_perm(v[2 * e + 1][w], v[2 * e][w], 0x07060302u);
      }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      u32x4_t qb[4];
#pragma unroll
      for (int st = 0; st < 4; ++st)
        qb[st] = live[nt] ? *(const u32x4_t*)(qrow[nt] + 64 * (st >> 1) + 16 * g + 8 * (st & 1)) : u32x4_t{0, 0, 0, 0};
      uint64_t anc = 0;
      if (TREE)
        anc = ((uint64_t)(uint32_t)__shfl((uint32_t)(mine >> 32), node[nt]) << 32) | (uint32_t)__shfl((uint32_t)mine, node[nt]);
      float x[8];
      uint32_t seen = 0;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st)
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[kt][st]), as_bf16x8(qb[st]), s, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = j0 + 16 * kt + 4 * g + r;
          const bool vis = j < L || (TREE && j < end && ((anc >> (j - L)) & 1));
          seen |= (vis ? 1u : 0u) << (4 * kt + r);
          x[4 * kt + r] = vis ? s[r] * a.scale_log2 : neg_inf();
        }
      }
      softmax_unit(x, sm[nt], acc[nt], size);
      const float f = sm[nt].c;
      u32x4_t ph, pl;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p0 = x[2 * e] * f, p1 = x[2 * e + 1] * f;
        ph[e] = pack_bf16x2(p0, p1);
        pl[e] = pack_bf16x2(p0 - __uint_as_float(ph[e] << 16), p1 - __uint_as_float(ph[e] & 0xffff0000u));
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        u32x4_t w = vt[t];
        if (odd) acc[nt][t] += add_not_finite(w, seen);
        acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(ph), acc[nt][t], 0, 0, 0);
        acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(pl), acc[nt][t], 0, 0, 0);
      }
    }
  }

  // The waves' states join in LDS, a query tile at a time: lane (c, g) holds
  // row c, dims 32 g + 8 r + t.  Each wave's output enters divided by its own
  // sum, with the weight 2^(m - M) l.
  __shared__ float lds_m[kWaves][16], lds_l[kWaves][16];
  constexpr int kPitch = kD + 4;
  __shared__ __attribute__((aligned(16))) float lds_o[kWaves][16][kPitch];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const float l = sum_across_groups(sm[nt].l);
    if (g == 0) lds_m[wave][c] = sm[nt].m, lds_l[wave][c] = l;
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);  // NaN stays
    const float unit = sm[nt].c > 0.f ? 1.f / sm[nt].c : 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < 8; t += 4) {
        f32x4_t o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = acc[nt][t + e][r] * inv * unit;
        *(f32x4_t*)&lds_o[wave][c][32 * g + 8 * r + t] = o;
      }
    __syncthreads();
    const int row = tid / 16, d = tid % 16 * 8, r = row0 + 16 * nt + row;
    if (r < R) {
      float M = neg_inf(), Lsum = 0.f, o[8];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, lds_m[w][row]);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float lw = lds_l[w][row];
        const float wt = lw == 0.f ? 0.f : fast_exp2(lds_m[w][row] - (M == neg_inf() ? 0.f : M)) * lw;
        Lsum += wt;
        if (lw != 0.f)
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += wt * lds_o[w][row][d + e];
      }
      const float inv_l = Lsum > 0.f ? 1.f / Lsum : (Lsum == 0.f ? 0.f : Lsum);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= inv_l;
      if (a.splits == 1) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(o[2 * e], o[2 * e + 1]);
        *(u32x4_t*)(a.out + (((size_t)b * a.N + r / G) * a.H + hk * G + r % G) * kD + d) = w;
      } else {
        const size_t at = ((head * a.groups + grp) * a.splits + split) * (16 * NT) + 16 * nt + row;
        if (d == 0) a.part_ml[at] = make_float2(M, Lsum);
        *(f32x4_t*)(a.part_o + at * kD + d) = f32x4_t{o[0], o[1], o[2], o[3]};
        *(f32x4_t*)(a.part_o + at * kD + d + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
      }
    }
    __syncthreads();
  }
}

// Joins the splits' outputs in split order: 16 threads a row.
template <int NT>
__global__ __launch_bounds__(kThreads) void q8_attn_combine(Q8AttnArgs a) {
  const int G = a.H / a.H_kv, R = a.N * G;
  const size_t id = (size_t)blockIdx.x * 16 + threadIdx.x / 16;
  const size_t head = id / R;
  const int r = id % R, d = threadIdx.x % 16 * 8;
  if (head >= (size_t)a.B * a.H_kv) return;
  const int grp = r / (16 * NT), in = r % (16 * NT);
  const size_t first = (head * a.groups + grp) * a.splits * (16 * NT) + in;
  float M = neg_inf(), L = 0.f, o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, a.part_ml[first + (size_t)s * 16 * NT].x);
  for (int s = 0; s < a.splits; ++s) {
    const size_t at = first + (size_t)s * 16 * NT;
    const float2 ml = a.part_ml[at];
    if (ml.y == 0.f) continue;
    const float w = fast_exp2(ml.x - (M == neg_inf() ? 0.f : M)) * ml.y;
    L += w;
    const f32x4_t x = *(const f32x4_t*)(a.part_o + at * kD + d), y = *(const f32x4_t*)(a.part_o + at * kD + d + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += w * x[e], o[4 + e] += w * y[e];
  }
  const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
  u32x4_t w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
  const int b = head / a.H_kv, hk = head % a.H_kv;
  *(u32x4_t*)(a.out + (((size_t)b * a.N + r / G) * a.H + hk * G + r % G) * kD + d) = w;
}

template <int NT, bool INT8>
void launch_nt(const Q8AttnArgs& a, hipStream_t stream) {
  const dim3 grid(a.H_kv * a.groups, a.B, a.splits), block(kThreads);
  if (a.parents)
    hipLaunchKernelGGL((q8_attn_kernel<NT, INT8, true>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((q8_attn_kernel<NT, INT8, false>), grid, block, 0, stream, a);
}

template <int NT>
hipError_t launch_tiles(const Q8AttnArgs& a, bool int8, hipStream_t stream) {
  if (int8)
    launch_nt<NT, true>(a, stream);
  else
    launch_nt<NT, false>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const size_t rows = (size_t)a.B * a.N * a.H;
  hipLaunchKernelGGL((q8_attn_combine<NT>), dim3((rows + 15) / 16), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

Q8AttnPlan plan_q8_attn(int B, int N, int H, int H_kv, int n_blocks, int max_splits) {
  Q8AttnPlan p{};
  const int R = N * (H / H_kv);
  p.tiles = R <= 16 ? 1 : (R <= 32 ? 2 : 4);
  p.groups = (R + 16 * p.tiles - 1) / (16 * p.tiles);
  const long wgs = (long)B * H_kv * p.groups;
  const int most = max(1, min(kMaxSplits, n_blocks / 4));
  const int want = max_splits > 0 ? max_splits : (int)min((2L * kNumCU + wgs - 1) / wgs, (long)kMaxSplits);
  p.splits = max(1, min(want, most));
  if (p.splits > 1) {
    const size_t rows = (size_t)wgs * p.splits * 16 * p.tiles;
    p.part_ml_off = kCounterBytes;  // the counters of a shared workspace stay as they are
    p.part_o_off = (p.part_ml_off + rows * sizeof(float2) + 255) & ~(size_t)255;
    p.ws_bytes = p.part_o_off + rows * kD * sizeof(float);
  }
  return p;
}

hipError_t launch_q8_attn(const Q8AttnArgs& a, bool int8, int tiles, hipStream_t stream) {
  if (tiles == 1) return launch_tiles<1>(a, int8, stream);
  if (tiles == 2) return launch_tiles<2>(a, int8, stream);
  return launch_tiles<4>(a, int8, stream);
}

}  // namespace glide

// What the kernels over the paged cache share: packing, exponentials, and the tiles of 32
// entries in which the attention kernels go through a cache.
#pragma once

#include <math.h>

#include "rk_internal.h"

namespace rk {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes of cache elements as floats and back (one rounding to nearest even)
template <typename T> struct Pack;
template <> struct Pack<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ v4u put(const float* f) {
    v4u u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f2bf(f[2 * i]) | ((uint32_t)f2bf(f[2 * i + 1]) << 16);
    return u;
  }
};
template <> struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
  static __device__ __forceinline__ v4u put(const float* f) {
    v4u u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(f[i]);
    return u;
  }
};

// e^x of a difference to a running maximum.  The difference is formed before the factor
// log2(e): scaling the scores themselves would put that factor's rounding, times a
// score of 50, into the weights.
__device__ __forceinline__ float exp_diff(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// unit e^x with the product's rounding and log2(e)'s made good, for the weights of fp32
// caches, whose outputs show them: e^-10 is off by 5e-7 without.  (Rescales and joins do
// without: what they are off by is no more than the rounding of a score as large.)
__device__ __forceinline__ float exp_diff_exact(float x, float unit) {
  x = x < -200.f ? -200.f : x;   // 0 either way; a NaN stays
  const float t = x * kLog2e, r = fmaf(x, kLog2e, -t) + x * 1.925963033500e-8f;
  return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.6931471806f * unit, unit);
}

// The largest bf16 below a positive x, as the bits of a float; 0 of 0.  What is left, x minus
// it, is positive again, never 0 (at the least one step of x).
__device__ __forceinline__ uint32_t bf16_below(float x) {
  return __builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xffff0000u;
}

// Two pieces of a weight x stand for x times this: the first is x cut off, the second, of which 0
// would make an infinite value NaN, so stays positive.
constexpr float kTwoPieces = 1.f + 0x1p-18f;
__device__ __forceinline__ uint32_t f2bf_pair(float x, float y) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  typedef float pair_f __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(pair_f{x, y}, pair));
}

// Values of 8 bits (4 exponent and 3 mantissa bits, largest 448, NaN but no infinity) in
// rows that share a power of two: byte b of a row's scale stands for 2^(b - 127).
struct e4m3_t { uint8_t bits; };
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float e4m3_scale(uint32_t b) { return __uint_as_float(b << 23); }
// eight values times a power of two, as bf16: exact, but for what is out of bf16's range
__device__ __forceinline__ v4u e4m3_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return v4u{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
             __builtin_bit_cast(uint32_t, d)};
}
// The scale of a row whose largest finite value is amax: 2^e, e the least with amax <= 448 2^e
// (448 = 1.75 2^8), at least 2^-117, so that every value of the row is a normal bf16 number.
__device__ __forceinline__ uint32_t e4m3_scale_of(float amax) {
  return (uint32_t)min(max((int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8, 10), 247);
}
// what a value counts for the scale of its row
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// Eight values in units of scale byte b, rounded to nearest even; infinities and NaN become
// NaN; what would round to 2^128 becomes the largest value below it.
__device__ __forceinline__ v2u to_e4m3(const float* x, uint32_t b) {
  const float inv = __uint_as_float((254u - b) << 23), top = b == 247 ? 240.f : 448.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fabsf(x[i]) < INFINITY ? __builtin_amdgcn_fmed3f(x[i] * inv, -top, top) : NAN;
  v2u u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
    u[i] = (uint32_t)w;
  }
  return u;
}
__device__ __forceinline__ void from_e4m3(v2u u, uint32_t b, float* x) {
  const float scale = e4m3_scale(b);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u[i], true);
    x[4 * i] = lo[0] * scale; x[4 * i + 1] = lo[1] * scale;
    x[4 * i + 2] = hi[0] * scale; x[4 * i + 3] = hi[1] * scale;
  }
}

// 16 bytes of values: infinities and NaN become 0 (sign 0), or all others do, and those of that
// sign and NaN become 2 or -2 (sign 1 or -1); whether there are any.  scale: 8-bit rows' byte.
template <typename C> __device__ __forceinline__ bool take_out(v4u& v, int sign, uint32_t scale = 127);
template <> __device__ __forceinline__ bool take_out<bf16_t>(v4u& v, int sign, uint32_t) {
  bool any = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (sign == 0) {   // an exponent of ones carries into the bit above it
      const uint32_t over = ((v[w] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
      any |= over != 0;
      v[w] &= ~((over >> 15) * 0xffffu);
      continue;
    }
    uint32_t r = 0;
#pragma unroll
    for (int at = 0; at < 32; at += 16) {
      const uint32_t x = v[w] >> at & 0xffffu;
      const bool bad = (x & 0x7f80u) == 0x7f80u, mine = bad && ((x & 0x7fu) || (x >> 15) == (sign < 0));
      any |= bad;
      r |= (mine ? (sign < 0 ? 0xc000u : 0x4000u) : 0u) << at;
    }
    v[w] = r;
  }
  return any;
}
// NaN, and what a scale byte above 246 takes to 2^128 or more, an infinity as bf16: a code c of exponent
// c >> 3 stands for 2^((c >> 3) - 7 + scale - 127) or more, so c from 8 (262 - scale) on.
template <> __device__ __forceinline__ bool take_out<e4m3_t>(v4u& v, int sign, uint32_t scale) {
  const uint32_t carry = (uint32_t)max(1, 8 * ((int)scale - 246));   // takes the least of them to 0x80, NaN's 0x7f too
  bool any = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (sign == 0) {
      const uint32_t over = ((v[w] & 0x7f7f7f7fu) + carry * 0x01010101u) & 0x80808080u;
      any |= over != 0;
      v[w] &= ~((over >> 7) * 0xffu);
      continue;
    }
    uint32_t r = 0;
#pragma unroll
    for (int at = 0; at < 32; at += 8) {
      const uint32_t x = v[w] >> at & 0xffu, code = x & 0x7fu;
      const bool bad = code + carry >= 0x80u, mine = bad && (code == 0x7fu || (x >> 7) == (sign < 0));
      any |= bad;
      r |= (mine ? (sign < 0 ? 0xc0u : 0x40u) : 0u) << at;
    }
    v[w] = r;
  }
  return any;
}
template <> __device__ __forceinline__ bool take_out<float>(v4u& v, int sign, uint32_t) {
  bool any = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float x = __uint_as_float(v[w]);
    const bool bad = !(fabsf(x) < INFINITY), mine = bad && (x != x || (x < 0.f) == (sign < 0));
    any |= bad;
    v[w] = __float_as_uint(sign == 0 ? (bad ? 0.f : x) : mine ? 2.f * sign : 0.f);
  }
  return any;
}

// Bounds keep a NaN.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ int min_i(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int max_i(int a, int b) { return a > b ? a : b; }

__device__ __forceinline__ int table_length(const PagedTable& tab, int row, int page_shift) {
  return max_i(0, (int)min((int64_t)tab.lengths[row], (int64_t)tab.max_pages << page_shift));
}

constexpr int kDecodeWaves = 4, kTile = 32;

// A wave's tile of 32 entries of one KV head, and what is done with it for 16 columns (a column is
// a query row of one head):
//   scores  S^T[entry, column] = K Q^T: the cache's rows are the A operand as they lie
//           in memory, so K goes from memory to the matrix unit's registers directly;
//   values  O^T[d, column] += V^T P^T: a lane's scores are already the B operand of that
//           product (entries 4 g + i of its 16-lane group g), and V^T comes out of a
//           row-major LDS tile with transposing reads (bf16) or from memory with d
//           spread over the product's rows (fp32).
template <typename C, int DH> struct CacheTile;

// Transposed values from LDS and weights in PIECES bf16 numbers, all positive, for tiles of
// bf16 values: three pieces hold all 24 bits of a weight, two 16 or more.
template <int DH> struct StagedValues {
  static constexpr int CH = DH / 8;          // 16-byte pieces of a row
  static constexpr int ND = DH / 16;         // 16-row blocks of O^T
  static constexpr int LDS = kTile * DH * 2; // bytes per wave

  // the 32-byte pair of pieces that ds_read_b64_tr_b16 takes from a row, placed so
  // that eight consecutive rows use all 64 banks
  static __device__ __forceinline__ int swz(int row) { return DH == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }

  // 16 channels of 32 entries, as the A operand
  static __device__ __forceinline__ v4u transposed(int b, const char* lds, int lane) {
    const int g = lane >> 4, jj = lane & 15, r = 4 * g + (jj >> 2), ch = 2 * b + ((jj & 3) >> 1);
    const char* at = lds + (r * CH + (ch ^ swz(r))) * 16 + (jj & 1) * 8;   // swz(r + 16) = swz(r)
    const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * CH * 16));
    return v4u{__builtin_bit_cast(v2u, a0)[0], __builtin_bit_cast(v2u, a0)[1], __builtin_bit_cast(v2u, a1)[0],
               __builtin_bit_cast(v2u, a1)[1]};
  }
  // a lane's weights as the B operand
  template <int PIECES>
  static __device__ __forceinline__ void pieces(const f32x4_t* p, v4u* part) {
    static_assert(PIECES == 2 || PIECES == 3, "weights");
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float x = p[e >> 2][e & 3], y = p[e >> 2][(e & 3) + 1];
      if constexpr (PIECES == 3) {
        const uint32_t x0 = bf16_below(x), y0 = bf16_below(y);
        const float x1 = x - __uint_as_float(x0), y1 = y - __uint_as_float(y0);
        part[0][e / 2] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);   // the upper halves
        const uint32_t x2 = bf16_below(x1), y2 = bf16_below(y1);
        part[1][e / 2] = __builtin_amdgcn_perm(y2, x2, 0x07060302u);
        part[2][e / 2] = (uint32_t)f2bf(x1 - __uint_as_float(x2)) | ((uint32_t)f2bf(y1 - __uint_as_float(y2)) << 16);
      } else {
        const uint32_t x0 = __float_as_uint(x), y0 = __float_as_uint(y);
        part[0][e / 2] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
        part[1][e / 2] = f2bf_pair(fmaf(x, kTwoPieces, -__uint_as_float(x0 & 0xffff0000u)),
                                   fmaf(y, kTwoPieces, -__uint_as_float(y0 & 0xffff0000u)));
      }
    }
  }
  // .. times the values, for N blocks of columns.  Two pieces: a block's values are read while those
  // of the one before are multiplied (left alone, the compiler waits for each; three pieces take long
  // enough for that).  8 caches of 500 .. 4096, 26 drafts: 40 -> 38 us.
  template <int N, int PIECES>
  static __device__ __forceinline__ void add(const v4u (*part)[PIECES], f32x4_t (*o)[ND], const char* lds, int lane) {
    constexpr bool kAhead = PIECES == 2;
    v4u a[2];
    if (kAhead) a[0] = transposed(0, lds, lane);
#pragma unroll
    for (int b = 0; b < ND; ++b) {
      const int next = b + kAhead;
      if (next < ND) a[next & 1] = transposed(next, lds, lane);
      if (kAhead) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int n = 0; n < N; ++n)
          o[n][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a[b & 1]),
                                                            __builtin_bit_cast(bf16x8_t, part[n][i]), o[n][b], 0, 0, 0);
      if (kAhead) __builtin_amdgcn_sched_barrier(0);
    }
  }
  // weights of 24 bits: the matrix unit has the time
  static __device__ __forceinline__ void accumulate(const f32x4_t* p, f32x4_t* o, char* lds, int lane) {
    v4u part[1][3];
    pieces<3>(p, part[0]);
    add<1, 3>(part, reinterpret_cast<f32x4_t (*)[ND]>(o), lds, lane);
    wave_sync();
  }
  // channel of element i of output block b in 16-lane group g
  static __device__ __forceinline__ int channel(int b, int g, int i) { return b * 16 + 4 * g + i; }
};

template <int DH> struct CacheTile<bf16_t, DH> : StagedValues<DH> {
  using Base = StagedValues<DH>;
  static constexpr int CH = Base::CH;
  static constexpr int NC = DH / 32;         // k-steps of the scores
  static constexpr int NV = kTile * CH / 64; // 16-byte loads of V per lane
  struct Query { bf16x8_t q[NC]; };
  v4u k[2][NC], v[NV];

  static __device__ __forceinline__ void load_q(Query& q, const bf16_t* qp, int lane) {   // row of this lane's column
#pragma unroll
    for (int c = 0; c < NC; ++c)
      q.q[c] = __builtin_bit_cast(bf16x8_t, *(const v4u*)(qp + c * 32 + (lane >> 4) * 8));
  }
  // rows of the tile's two 16-entry halves, by their index in the cache
  __device__ __forceinline__ void load_k(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const bf16_t *k0 = (const bf16_t*)cache.k + r0 * DH, *k1 = (const bf16_t*)cache.k + r1 * DH;
    const uint32_t at = (lane & 15) * DH + (lane >> 4) * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      k[0][c] = *(const v4u*)(k0 + at + c * 32);
      k[1][c] = *(const v4u*)(k1 + at + c * 32);
    }
  }
  __device__ __forceinline__ void load_v(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const bf16_t *v0 = (const bf16_t*)cache.v + r0 * DH, *v1 = (const bf16_t*)cache.v + r1 * DH;
    // a load covers 64 / CH rows, all of one half
    const uint32_t at = lane * 8;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = *(const v4u*)((i < NV / 2 ? v0 : v1) + at + i % (NV / 2) * 512);
  }
  __device__ __forceinline__ void clear_values(uint32_t seen, int lane) {   // bit r: row r counts
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!(seen >> ((i * 64 + lane) / CH) & 1)) v[i] = v4u{0, 0, 0, 0};
  }
  __device__ __forceinline__ void scores(const Query& q, f32x4_t* s) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[t][c]), q.q[c], s[t], 0, 0, 0);
    }
  }
  __device__ __forceinline__ bool take_out_values(int sign) {   // see take_out
    bool any = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) any |= take_out<bf16_t>(v[i], sign);
    return any;
  }
  // the values' registers are free after stage_v
  __device__ __forceinline__ void stage_v(char* lds, int lane) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int slot = i * 64 + lane, row = slot / CH, ch = slot % CH;
      *(v4u*)(lds + (row * CH + (ch ^ Base::swz(row))) * 16) = v[i];
    }
    wave_sync();
  }
  static constexpr bool kStaged = true;
  __device__ __forceinline__ void values(const f32x4_t* p, f32x4_t* o, char* lds, int lane) const {
    Base::accumulate(p, o, lds, lane);
  }
};

// 8-bit values with a scale for each row: both become bf16 numbers on the way, which hold
// them exactly, keys as they enter the product, values as they enter LDS; from there on a
// cache of those numbers would give the same sums.  A lane's 16 bytes of a key are two
// k-steps' operands, so the queries' channels are taken in that order.
template <int DH> struct CacheTile<e4m3_t, DH> : StagedValues<DH> {
  using Base = StagedValues<DH>;
  static constexpr int CH = Base::CH;
  static constexpr int NC = DH / 32;             // k-steps of the scores
  static constexpr int CB = DH / 16;             // 16-byte pieces of a cache row
  static constexpr int NV = kTile * CB / 64;     // 16-byte loads of V per lane
  struct Query { bf16x8_t q[NC]; };
  v4u k[2][NC / 2], v[NV];
  uint32_t ks[2], vs[NV];                        // scale bytes

  static __device__ __forceinline__ void load_q(Query& q, const bf16_t* qp, int lane) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
      q.q[c] = __builtin_bit_cast(bf16x8_t, *(const v4u*)(qp + c / 2 * 64 + (lane >> 4) * 16 + c % 2 * 8));
  }
  __device__ __forceinline__ void load_k(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const uint8_t *k0 = (const uint8_t*)cache.k + r0 * DH, *k1 = (const uint8_t*)cache.k + r1 * DH;
    const uint32_t at = (lane & 15) * DH + (lane >> 4) * 16;
#pragma unroll
    for (int c = 0; c < NC / 2; ++c) {
      k[0][c] = *(const v4u*)(k0 + at + c * 64);
      k[1][c] = *(const v4u*)(k1 + at + c * 64);
    }
    ks[0] = (cache.k_scales + r0)[lane & 15];
    ks[1] = (cache.k_scales + r1)[lane & 15];
  }
  __device__ __forceinline__ void load_v(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const uint8_t *v0 = (const uint8_t*)cache.v + r0 * DH, *v1 = (const uint8_t*)cache.v + r1 * DH;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = *(const v4u*)((i < NV / 2 ? v0 : v1) + lane * 16 + i % (NV / 2) * 1024);
      vs[i] = (cache.v_scales + (i < NV / 2 ? r0 : r1))[i % (NV / 2) * (64 / CB) + lane / CB];
    }
  }
  __device__ __forceinline__ void clear_values(uint32_t seen, int lane) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!(seen >> ((i * 64 + lane) / CB) & 1)) { v[i] = v4u{0, 0, 0, 0}; vs[i] = 127; }
  }
  __device__ __forceinline__ bool take_out_values(int sign) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      any |= take_out<e4m3_t>(v[i], sign, vs[i]);
      if (sign != 0) vs[i] = 127;
    }
    return any;
  }
  __device__ __forceinline__ void scores(const Query& q, f32x4_t* s) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float scale = e4m3_scale(ks[t]);
      s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const v4u a = e4m3_to_bf16(k[t][c / 2][c % 2 * 2], k[t][c / 2][c % 2 * 2 + 1], scale);
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), q.q[c], s[t], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void stage_v(char* lds, int lane) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int slot = i * 64 + lane, row = slot / CB, ch = slot % CB * 2;
      const float scale = e4m3_scale(vs[i]);
      v4u* at = (v4u*)(lds + (row * CH + (ch ^ Base::swz(row))) * 16);   // swz is even: both pieces together
      at[0] = e4m3_to_bf16(v[i][0], v[i][1], scale);
      at[1] = e4m3_to_bf16(v[i][2], v[i][3], scale);
    }
    wave_sync();
  }
  static constexpr bool kStaged = true;
  __device__ __forceinline__ void values(const f32x4_t* p, f32x4_t* o, char* lds, int lane) const {
    Base::accumulate(p, o, lds, lane);
  }
};

template <int DH> struct CacheTile<float, DH> {
  static constexpr int NC = DH / 16;
  static constexpr int VEC = DH >= 64 ? 4 : 2;   // channels per lane and load of V
  static constexpr int NP = DH / (16 * VEC);     // loads per entry
  static constexpr int ND = DH / 16;
  static constexpr int LDS = 0;
  typedef float vecf __attribute__((ext_vector_type(VEC)));
  struct Query { f32x4_t q[NC]; };
  f32x4_t k[2][NC];
  vecf v[2][4][NP];

  static __device__ __forceinline__ void load_q(Query& q, const float* qp, int lane) {
#pragma unroll
    for (int c = 0; c < NC; ++c) q.q[c] = *(const f32x4_t*)(qp + c * 16 + (lane >> 4) * 4);
  }
  __device__ __forceinline__ void load_k(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const float *k0 = (const float*)cache.k + r0 * DH, *k1 = (const float*)cache.k + r1 * DH;
    const uint32_t at = (lane & 15) * DH + (lane >> 4) * 4;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      k[0][c] = *(const f32x4_t*)(k0 + at + c * 16);
      k[1][c] = *(const f32x4_t*)(k1 + at + c * 16);
    }
  }
  __device__ __forceinline__ void load_v(const PagedView& cache, int64_t r0, int64_t r1, int lane) {
    const float *v0 = (const float*)cache.v + r0 * DH, *v1 = (const float*)cache.v + r1 * DH;
    const uint32_t at = (lane >> 4) * 4 * DH + (lane & 15) * VEC;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < NP; ++c) {
        v[0][i][c] = *(const vecf*)(v0 + at + i * DH + c * 16 * VEC);
        v[1][i][c] = *(const vecf*)(v1 + at + i * DH + c * 16 * VEC);
      }
  }
  static constexpr bool kStaged = false;
  __device__ __forceinline__ void stage_v(char*, int) const {}
  __device__ __forceinline__ void clear_values(uint32_t seen, int lane) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(seen >> (t * 16 + 4 * (lane >> 4) + i) & 1))
#pragma unroll
          for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[t][i][c][e] = 0.f;
  }
  __device__ __forceinline__ bool take_out_values(int sign) {
    bool any = false;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NP; ++c) {
          v4u u = {0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < VEC; ++e) u[e] = __float_as_uint(v[t][i][c][e]);
          any |= take_out<float>(u, sign);
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[t][i][c][e] = __uint_as_float(u[e]);
        }
    return any;
  }
  __device__ __forceinline__ void scores(const Query& q, f32x4_t* s) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // four sums over a quarter of the channels each: shorter chains, and none waits for another
      f32x4_t a[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) a[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][c][e], q.q[c][e], a[e], 0, 0, 0);
      }
      s[t] = (a[0] + a[1]) + (a[2] + a[3]);
    }
  }
  __device__ __forceinline__ void values(const f32x4_t* p, f32x4_t* o, char*, int) const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            o[c * VEC + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][i][c][e], p[t][i], o[c * VEC + e], 0, 0, 0);
  }
  static __device__ __forceinline__ int channel(int b, int g, int i) {
    return (b / VEC) * 16 * VEC + VEC * (4 * g + i) + b % VEC;
  }
};

// Entries of one part of a length: whole tiles for every wave, at most n_parts parts.
__device__ __forceinline__ int part_entries(int len, int n_parts) {
  constexpr int unit = kTile * kDecodeWaves;
  const int per = (len + n_parts - 1) / n_parts;
  return max_i((per + unit - 1) / unit, 1) * unit;
}

// Dispatch on the rows' and the cache's element types and the head size.
#define RK_PAGED_DISPATCH(view, CALL)                                              \
  do {                                                                             \
    const int dh_ = (view).head_dim;                                               \
    if ((view).e4m3) {                                                             \
      if (dh_ == 64) { CALL(bf16_t, e4m3_t, 64); } else { CALL(bf16_t, e4m3_t, 128); } \
    } else if ((view).bf16) {                                                      \
      if (dh_ == 64) { CALL(bf16_t, bf16_t, 64); } else { CALL(bf16_t, bf16_t, 128); } \
    } else {                                                                       \
      if (dh_ == 32) { CALL(float, float, 32); }                                   \
      else if (dh_ == 64) { CALL(float, float, 64); }                              \
      else { CALL(float, float, 128); }                                            \
    }                                                                              \
  } while (0)

}  // namespace rk

// Tiles of 32 cached positions against rows of queries on the matrix cores
// (iq_decode_tree.hip describes the products and the layouts; iq_prefill.hip
// attends chunks of prompts the same way).  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include "iq_span_device.h"

namespace iq {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
// global memory, by pointers whose origin the compiler no longer sees
#define IQ_GLOBAL __attribute__((address_space(1)))
typedef const IQ_GLOBAL uint8_t* global_bytes_t;
typedef const IQ_GLOBAL float* global_floats_t;
typedef uint32_t u32_a1_t __attribute__((aligned(1)));

constexpr int kTile = 32;                  // positions of a tile
constexpr int kKeyStride = 2 * kDim + 16;  // bytes of a tile's key: 16 banks of four apart
constexpr int kValStride = 2 * kTile + 16; // bytes of a dimension's values
constexpr int kORow = kDim + 4;            // floats of an output row in LDS
constexpr float kSlack = 4.0f;             // log2 units by which a score may exceed the reference
constexpr int kUnitBits = 10;              // weights are at most 2^(kUnitBits + 1 + kSlack)

__device__ __forceinline__ f32x16_t mfma32(u32x4_t a, u32x4_t b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a),
                                                __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

// Where slot s (16 bytes) of dimension d's values lies in its row: the two halves
// of the row change places every 16 dimensions.  A wave writes the values of 8
// dims 4 apart in u and 4 records apart at once (rows 640 bytes apart: without
// the change every fourth write met 16 others in its bank, 64 cycles each).  With it
// a write takes 8 cycles for 4 and a read of 32 rows 8 for 4 (measured apart, by
// counters).
__device__ __forceinline__ int value_slot(int d, int s) { return s ^ ((d >> 4 & 1) << 1); }

// The rests p0 - hi[0], p1 - hi[1] of a pair of weights (exact) as fp16, to
// nearest: the mixed-precision multiply-add takes the half as it is and places
// its result, where conversions, subtractions and a pack are six instructions.
// (minus_one: -1, opaque; a constant becomes a subtraction, which has no such
// form.)
__device__ __forceinline__ uint32_t rest_pair(uint32_t hi, float p0, float p1, float minus_one) {
  const half2_t h = __builtin_bit_cast(half2_t, hi);
  const float h0 = static_cast<float>(h[0]), h1 = static_cast<float>(h[1]);
  return __builtin_bit_cast(
      uint32_t, half2_t{static_cast<_Float16>(__builtin_fmaf(h0, minus_one, p0)),
                        static_cast<_Float16>(__builtin_fmaf(h1, minus_one, p1))});
}

constexpr int kKeyBytes = kTile * kKeyStride;    // a tile's keys
constexpr int kValueBytes = kDim * kValStride;   // and values

// The sum over a wave's lanes, in every lane (see wave64_max).
__device__ __forceinline__ float wave64_sum(float x) {
  x += xor_lane<1>(x);
  x += xor_lane<2>(x);
  x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x124, 0xF,
                                                          0xF, true));
  x += xor_lane<8>(x);
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x142,
                                                             0xA, 0xF, false));
  x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x143,
                                                             0xC, 0xF, false));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// Dims of a record's 2 pairs at bit `sh` of w (see window_pairs).
template <int kBits>
__device__ __forceinline__ void value_half(const uint32_t* lut, uint32_t w, uint32_t sh,
                                           uint32_t& p0, uint32_t& p1) {
  const uint32_t x = w >> sh;
  if constexpr (kBits == 3) {
    const uint32_t xu = w >> (sh + 4);
    p0 = lut_at(lut, low6x4<0>(x));
    p1 = lut_at(lut, top6x4<0>(xu));
  } else if constexpr (kBits == 4) {
    p0 = lut_at(lut, byte4x4<0>(x));
    p1 = lut_at(lut, byte4x4<1>(x));
  } else {
    const uint32_t lo = x << 2, hi = x >> 2;
    p0 = lut_at(lut, nib4x4<0>(lo));
    p1 = lut_at(lut, nib4x4<0>(hi));
  }
}

// The decoding of tiles, dealt to the lanes of a group's kRows waves: a lane has
// kTasks tasks of keys (kKeyDims dims of a record) and of values (kValDims dims of
// 4 records), each within one half of the tile (16 positions): half i of a task,
// or rw % 2 where there are several waves.  A wave's writes are 16 keys at once, free
// of bank conflicts, or values 4 records apart times 4 rows apart (see value_slot).
// A lookup in the table of 3-bit pairs takes 3.4 cycles for 2 (2 bits: 2, 4 bits:
// 4.6).  With eight waves of rows the values' reads make half of the conflicts, the
// lookups a fifth, the values' writes an eighth.
template <int kRows, int kBits>
struct TileDecode {
  static constexpr int kRB = record_bytes<kBits>();
  static constexpr int kTasks = kRows == 1 ? 2 : 1;
  static constexpr int kKeyDims = kRows == 4 ? 16 : 32;
  static constexpr int kValDims = kRows == 4 ? 4 : 8;
  static constexpr int kKeyWords = (kKeyDims * kBits + 31) / 32;
  int key, quad;           // key record in the half, its first dim / kKeyDims; values: see below
  int chunk, vdim;         // (records 4 quad .., dims kValDims * vdim ..)
  uint32_t koff, voff;     // offsets of a half's first record for them
  uint32_t vshift;
  uint32_t raw_k[kTasks][kKeyWords], raw_v[kTasks][4];

  __device__ __forceinline__ void setup(int rw, int lane) {
    const int high = kRows == 4 ? rw >> 1 : 0;
    key = lane & 15;
    chunk = (lane >> 4) + 4 * high;
    quad = lane & 3;
    vdim = (lane >> 2) + 16 * high;
    koff = static_cast<uint32_t>(key * kRB + kKeyDims * kBits / 8 * chunk);
    // the dword with a value task's codes, or the record's last one where that
    // one reaches past it
    const int bit = kValDims * kBits * vdim, byte = bit >> 3;
    const int at = byte < kRB - 4 ? byte : kRB - 4;
    vshift = static_cast<uint32_t>(8 * (byte - at) + (bit & 7));
    voff = static_cast<uint32_t>(4 * quad * kRB + at);
  }
  // Task i's loads: a half's first record (keys, values), with `more` records
  // after it (whole: at least 15).
  __device__ __forceinline__ void load(int i, global_bytes_t kc, global_bytes_t vc, int more,
                                       bool whole) {
    uint32_t ko = koff;
    if (!whole) ko -= static_cast<uint32_t>((key > more ? key - more : 0) * kRB);
    const global_bytes_t k = kc + ko;
    if constexpr (kKeyDims * kBits % 32 == 0) {
#pragma unroll
      for (int e = 0; e < kKeyWords; ++e) raw_k[i][e] = ((const IQ_GLOBAL uint32_t*)k)[e];
    } else {   // 48 bits, at an even address
      raw_k[i][0] = *(const IQ_GLOBAL u32_a1_t*)k;
      raw_k[i][1] = *(const IQ_GLOBAL uint16_t*)(k + 4);
    }
    if (whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        raw_v[i][e] = *(const IQ_GLOBAL u32_a1_t*)(vc + (voff + static_cast<uint32_t>(e * kRB)));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * quad + e;
        raw_v[i][e] = *(const IQ_GLOBAL u32_a1_t*)(
            vc + (voff + static_cast<uint32_t>(((r < more ? r : more) - 4 * quad) * kRB)));
      }
    }
  }
  // Task i decoded into the tile's keys and values; half: the tile's half.
  __device__ __forceinline__ void store(const uint32_t* lut, int i, int half, char* k, char* v) {
    uint32_t w[kBits];
#pragma unroll
    for (int e = 0; e < kBits; ++e) w[e] = e < kKeyWords ? raw_k[i][e < kKeyWords ? e : 0] : 0u;
    u32x4_t p[4];
    key_pairs<kBits>(lut, w, p);
    char* kd = k + (key + 16 * half) * kKeyStride + 2 * kKeyDims * chunk;
#pragma unroll
    for (int e = 0; e < kKeyDims / 8; ++e) *reinterpret_cast<u32x4_t*>(kd + 16 * e) = p[e];
    u32x4_t q[4];
    if constexpr (kValDims == 8) {
      window_pairs<kBits>(lut, raw_v[i], vshift, q);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint32_t a, b;
        value_half<kBits>(lut, raw_v[i][r], vshift, a, b);
        q[0][r] = a;
        q[1][r] = b;
      }
    }
    // a dim's 4 records are 8 bytes, in the order of the weights (see the top):
    // records 4 q4 .. in half q4 / 2 % 2 of slot 2 (q4 / 4) + q4 % 2
    const int q4 = quad + 4 * half, d = kValDims * vdim;
    char* vd = v + d * kValStride + 16 * value_slot(d, 2 * half + (q4 & 1)) + 8 * (q4 >> 1 & 1);
#pragma unroll
    for (int n = 0; n < kValDims / 2; ++n) {
      *reinterpret_cast<uint2*>(vd + 2 * n * kValStride) =
          uint2{__builtin_amdgcn_perm(q[n][1], q[n][0], 0x05040100u),
                __builtin_amdgcn_perm(q[n][3], q[n][2], 0x05040100u)};
      *reinterpret_cast<uint2*>(vd + (2 * n + 1) * kValStride) =
          uint2{__builtin_amdgcn_perm(q[n][1], q[n][0], 0x07060302u),
                __builtin_amdgcn_perm(q[n][3], q[n][2], 0x07060302u)};
    }
  }
};

// One wave's rows: what it carries from tile to tile.
struct TileRows {
  u32x4_t qh[8], ql[8];   // query operands: dims 16 s + 8 h .. of row lane % 32
  f32x16_t o[4];          // outputs, in units of unit / 2^kUnitBits
  u32x4_t ph[2], pl[2];   // weights of a tile: hi and lo parts
  float m, l;             // reference (log2 units), this lane's share of the sum
  bool even;              // the wave's rows have one `down`, which the key scales carry
};

// The lowest n (clamped to 0 .. 32) of 32 bits.
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? ~0u : (n > 0 ? (1u << n) - 1 : 0u);
}

// a b, 0 where a or b is 0 whatever the other is (an intrinsic without a builtin;
// as inline assembly the wait states behind a transcendental would be missing).
__device__ float mul_or_zero(float a, float b) __asm("llvm.amdgcn.fmul.legacy");

// Scores of a tile's keys at k, before their scales.  kLo, here and below: operands
// are pairs of parts (otherwise one fp16 value each).
template <bool kLo = true>
__device__ __forceinline__ f32x16_t tile_scores(const TileRows& w, const char* k, int ql, int h) {
  const char* kp = k + ql * kKeyStride + 16 * h;
  u32x4_t f[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) f[s] = *reinterpret_cast<const u32x4_t*>(kp + 32 * s);
  f32x16_t x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    x = mfma32(f[s], w.qh[s], x);
    if constexpr (kLo) x = mfma32(f[s], w.ql[s], x);
  }
  return x;
}

// Outputs: the values at v by the weights.
template <bool kLo = true>
__device__ __forceinline__ void tile_values(TileRows& w, const char* v, int ql, int h) {
  const char* vp = v + ql * kValStride + 16 * value_slot(ql, h);
  const char* vq = v + ql * kValStride + 16 * value_slot(ql, 2 + h);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const u32x4_t f0 = *reinterpret_cast<const u32x4_t*>(vp + 32 * d * kValStride);
    const u32x4_t f1 = *reinterpret_cast<const u32x4_t*>(vq + 32 * d * kValStride);
    w.o[d] = mfma32(f0, w.ph[0], w.o[d]);
    w.o[d] = mfma32(f1, w.ph[1], w.o[d]);
    if constexpr (kLo) {
      w.o[d] = mfma32(f0, w.pl[0], w.o[d]);
      w.o[d] = mfma32(f1, w.pl[1], w.o[d]);
    }
  }
}

// Scores x become scores against the reference, rounded once; sc: key scales.
// row_down: the row's `down`, read where the wave's rows differ in it.  masked: the row sees only the keys whose bits of `see` (of keys 4 h ..) are set.
// Returns whether a row's reference has to be raised.
__device__ __forceinline__ bool tile_relative(const TileRows& w, f32x16_t& x, const float* sc,
                                              const float* row_down, int h,
                                              bool masked,
                                              uint32_t see, float& top) {
  if (!w.even) {
    const float down = *row_down;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= down;
  }
  const float ref = w.m == -INFINITY ? 0.f : w.m;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&sc[8 * c + 4 * h]);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * c + j] = __builtin_fmaf(x[4 * c + j], ks[j], -ref);
  }
  if (masked) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = see >> (8 * (i / 4) + i % 4) & 1 ? x[i] : -INFINITY;
  }
  top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  const f32x2_t tops = half_pair(top);
  top = fmaxf(tops[0], tops[1]);
  return __any(top > (w.m == -INFINITY ? -INFINITY : kSlack));
}

// Raises the reference to the tile's largest score.
__device__ __forceinline__ void tile_raise(TileRows& w, f32x16_t& x, float top) {
  const float ref = w.m == -INFINITY ? 0.f : w.m;
  const float m = fmaxf(w.m, ref + top);
  const float f = w.m == m ? 1.0f : (w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m - m));
  const float by = (m == -INFINITY ? 0.f : m) - ref;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] -= by;
  w.l *= f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] *= f;
  w.m = m;
}

// Weights of relative scores x as pairs; sc: value scales.  hi: cut to fp16; lo:
// the exact rest, to nearest.  (A scale that is not finite counts where the
// weight is not 0, so not in rows that do not see its key.)  Without lo parts the
// products are rounded to nearest: 2^-12 each, of which sums of many keep less.
// kTileSums: weights are added up over the tile first (pieces of thousands of tiles: beside
// one score far above the others each weight alone would be rounded away).
template <bool kLo = true, bool kTileSums = false>
__device__ __forceinline__ void tile_weights(TileRows& w, const f32x16_t& x, const float* sc,
                                             int h) {
  float minus_one = -1.0f;
  asm volatile("" : "+s"(minus_one));
  float sum = kTileSums ? 0.f : w.l;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&sc[8 * c + 4 * h]);
    float p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = __builtin_amdgcn_exp2f(x[4 * c + j]);
      sum += e;
      p[j] = mul_or_zero(e, vs[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      if constexpr (kLo) {
        const uint32_t hi = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_pkrtz(p[2 * j], p[2 * j + 1]));
        w.ph[c >> 1][2 * (c & 1) + j] = hi;
        w.pl[c >> 1][2 * (c & 1) + j] = rest_pair(hi, p[2 * j], p[2 * j + 1], minus_one);
      } else {
        w.ph[c >> 1][2 * (c & 1) + j] = __builtin_bit_cast(
            uint32_t, half2_t{static_cast<_Float16>(p[2 * j]), static_cast<_Float16>(p[2 * j + 1])});
      }
    }
  }
  w.l = kTileSums ? w.l + sum : sum;
}

}  // namespace
}  // namespace iq

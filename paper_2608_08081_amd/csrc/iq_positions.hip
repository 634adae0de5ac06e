// Rotary positions of queries and keys, gfx950.
//
// A pair (a, b) of dims is turned by the angle position * frequency.  Far positions
// turn millions of times, so the angle is reduced in 64 bits, to a quarter turn and
// the rest of it (|rest| <= 1/2), which fits 32.
//
// Bound by memory: every value is read and written once.  A workgroup takes kTokens
// tokens with all of their heads: it computes a token's angles once, into LDS, while
// its first values are on their way; then each thread turns 16 values at a time (8
// pairs, in either layout two 16-byte words of fp16 or four of fp32).  16384 tokens of 40
// heads in fp16 take 66 us, 5.1 TB/s (a large copy's rate); 4099 tokens of 18 heads in fp32
// 17.2 us, 4.4 TB/s; one token 4.0 us, a launch and its chain of loads.
#include <hip/hip_runtime.h>
#include <math.h>

#include "iq_g8_device.h"

namespace iq {
namespace {

constexpr int kRotThreadsPerGroup = 256;
constexpr int kTokens = 4;
constexpr int kUnit = 16;   // values of a thread's task

// 16 values at p0 (8 of them) and p1 (the others), as floats.
__device__ __forceinline__ void load_unit(const __half* p0, const __half* p1, u32x4_t (&w)[4]) {
  w[0] = *reinterpret_cast<const u32x4_t*>(p0);
  w[1] = *reinterpret_cast<const u32x4_t*>(p1);
}
__device__ __forceinline__ void load_unit(const float* p0, const float* p1, u32x4_t (&w)[4]) {
  w[0] = reinterpret_cast<const u32x4_t*>(p0)[0];
  w[1] = reinterpret_cast<const u32x4_t*>(p0)[1];
  w[2] = reinterpret_cast<const u32x4_t*>(p1)[0];
  w[3] = reinterpret_cast<const u32x4_t*>(p1)[1];
}
__device__ __forceinline__ void store_unit(__half* p0, __half* p1, const u32x4_t (&w)[4]) {
  *reinterpret_cast<u32x4_t*>(p0) = w[0];
  *reinterpret_cast<u32x4_t*>(p1) = w[1];
}
__device__ __forceinline__ void store_unit(float* p0, float* p1, const u32x4_t (&w)[4]) {
  reinterpret_cast<u32x4_t*>(p0)[0] = w[0];
  reinterpret_cast<u32x4_t*>(p0)[1] = w[1];
  reinterpret_cast<u32x4_t*>(p1)[0] = w[2];
  reinterpret_cast<u32x4_t*>(p1)[1] = w[3];
}
template <typename T>
__device__ __forceinline__ float get(const u32x4_t (&w)[4], int i) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(float, static_cast<uint32_t>(w[i / 4][i % 4]));
  } else {
    return static_cast<float>(__builtin_bit_cast(half2_t, static_cast<uint32_t>(w[i / 8][i / 2 % 4]))[i & 1]);
  }
}
// Values i and i + 1 of a unit.
template <typename T>
__device__ __forceinline__ void put(u32x4_t (&w)[4], int i, float a, float b) {
  if constexpr (sizeof(T) == 4) {
    w[i / 4][i % 4] = __builtin_bit_cast(uint32_t, a);
    w[i / 4][i % 4 + 1] = __builtin_bit_cast(uint32_t, b);
  } else {
    w[i / 8][i / 2 % 4] = __builtin_bit_cast(
        uint32_t, half2_t{static_cast<_Float16>(a), static_cast<_Float16>(b)});
  }
}

// cos and sin of a position's angle at freq radians per position.
__device__ __forceinline__ f32x2_t turn(int32_t position, double freq) {
  // quarter turns: whole ones and the rest (|position| freq loses nothing that
  // counts: 2^-52 of at most 2^31 turns)
  const double x = static_cast<double>(position) * freq * 0.63661977236758134308;   // 2 / pi
  const double whole = rint(x);
  float s, c;
  sincospif(0.5f * static_cast<float>(x - whole), &s, &c);
  const int quarter = static_cast<int>(whole - 4.0 * floor(0.25 * whole));
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return f32x2_t{quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss};
}

template <typename T, bool kHalf>
__global__ __launch_bounds__(kRotThreadsPerGroup) void rotate_positions_kernel(RotateArgs a) {
  __shared__ __attribute__((aligned(16))) f32x2_t turns[kTokens][kDim / 2];
  const int tid = threadIdx.x;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * kTokens;
  const int tokens = a.n_tokens - t0 < kTokens ? static_cast<int>(a.n_tokens - t0) : kTokens;
  const int pairs = a.rope_dim / 2;
  const int shift = a.head_shift - 4;            // a head's tasks are 2^shift
  const int heads = a.n_q_heads + a.n_kv_heads;
  const int per_token = heads << shift;
  const int n = tokens * per_token;
  // Task e: 16 values of a head of a token.
  struct Task {
    const T *p0, *p1;
    T *d0, *d1;
    int token, first;   // its first pair, or -1: values that are not turned
  };
  auto task = [&](int e) {
    Task x;
    x.token = e / per_token;
    const int r = e - x.token * per_token;
    const int head = r >> shift, u = r & ((1 << shift) - 1);
    const bool is_k = head >= a.n_q_heads;
    const int64_t t = t0 + x.token;
    const int64_t at = static_cast<int64_t>(is_k ? head - a.n_q_heads : head) << a.head_shift;
    const T* src = static_cast<const T*>(is_k ? a.k : a.q) + t * (is_k ? a.k_stride : a.q_stride) + at;
    T* dst = static_cast<T*>(is_k ? a.k_out : a.q_out) +
             t * (is_k ? a.k_out_stride : a.q_out_stride) + at;
    const bool turned = kUnit * u < a.rope_dim;
    const int i0 = kHalf && turned ? 8 * u : kUnit * u;
    const int i1 = kHalf && turned ? i0 + pairs : i0 + 8;
    x.p0 = src + i0;
    x.p1 = src + i1;
    x.d0 = dst + i0;
    x.d1 = dst + i1;
    x.first = turned ? 8 * u : -1;
    return x;
  };
  u32x4_t w[4];
  Task cur;
  if (tid < n) {
    cur = task(tid);
    load_unit(cur.p0, cur.p1, w);
  }
  for (int e = tid; e < tokens * pairs; e += kRotThreadsPerGroup) {
    const int t = e / pairs, i = e - t * pairs;
    turns[t][i] = turn(a.positions[t0 + t], a.freqs[i]) * a.amplitude;
  }
  lds_barrier();
  for (int e = tid; e < n; e += kRotThreadsPerGroup) {
    const Task now = cur;
    u32x4_t x[4] = {w[0], w[1], w[2], w[3]};
    if (e + kRotThreadsPerGroup < n) {
      cur = task(e + kRotThreadsPerGroup);
      load_unit(cur.p0, cur.p1, w);
    }
    if (now.first >= 0) {
      f32x2_t cs[8];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4_t*>(&cs[2 * i]) =
            *reinterpret_cast<const f32x4_t*>(&turns[now.token][now.first + 2 * i]);
      if constexpr (kHalf) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float lo[2], hi[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float p = get<T>(x, i + j), q = get<T>(x, 8 + i + j);
            lo[j] = __builtin_fmaf(p, cs[i + j][0], -(q * cs[i + j][1]));
            hi[j] = __builtin_fmaf(p, cs[i + j][1], q * cs[i + j][0]);
          }
          put<T>(x, i, lo[0], lo[1]);
          put<T>(x, 8 + i, hi[0], hi[1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = get<T>(x, 2 * i), q = get<T>(x, 2 * i + 1);
          put<T>(x, 2 * i, __builtin_fmaf(p, cs[i][0], -(q * cs[i][1])),
                 __builtin_fmaf(p, cs[i][1], q * cs[i][0]));
        }
      }
    }
    store_unit(now.d0, now.d1, x);
  }
}

}  // namespace

hipError_t launch_rotate_positions(const RotateArgs& a, int dtype, bool half_layout,
                                   hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.n_tokens + kTokens - 1) / kTokens));
#define IQ_LAUNCH_ROTATE(T_, HALF_)                                                        \
  hipLaunchKernelGGL((rotate_positions_kernel<T_, HALF_>), grid, dim3(kRotThreadsPerGroup), 0, \
                     stream, a)
  if (dtype == IQ_DTYPE_F16) {
    if (half_layout) IQ_LAUNCH_ROTATE(__half, true);
    else IQ_LAUNCH_ROTATE(__half, false);
  } else {
    if (half_layout) IQ_LAUNCH_ROTATE(float, true);
    else IQ_LAUNCH_ROTATE(float, false);
  }
#undef IQ_LAUNCH_ROTATE
  return hipGetLastError();
}

}  // namespace iq

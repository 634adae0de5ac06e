// Decode attention with a sliding window and sinks on the packed cache, gfx950:
// the query at the end of a row of L positions attends positions j >= L -
// window and the first n_sinks.  App. A / Table 2 on those positions; the same
// operands, products and softmax as the span kernel (iq_span_device.h), whose
// chunks walk the row as if the positions between the sinks and the window were
// not there.
//
// Work decomposition: a row (KV head x head group of 8 query heads) of a
// sequence sees at most ceil(sinks / 16) + ceil(window / 16) + 1 batches of 16
// positions, which the launch knows, so a fixed number of workgroups per row
// shares the batches that the row's length leaves, in equal parts; a second
// kernel merges the parts and applies the inverse rotation.  The fused step's
// new token goes with a row's first part.  Without a new token, rows of one part
// are rotated back by the workgroups that make them (kAlone): 64 sequences of 8 KV
// heads with a window of 4096 55.8 us, with a merge 58.3; the fused step's lengths
// advance behind all heads of a sequence, which the merge waits for.
//
// Measured: windows of 4096 + 16 of 64 sequences of 1000 to 16000 positions with 8
// KV heads on pools 55 to 57 us.  They see 204 MB; on pages of 16 positions 227 MB
// are fetched (a head's scales are half a 128-byte line there; pages of 32 and rows
// 1 % more than is seen), at 4.1 TB/s, as the span kernel does in the middle of long
// rows.  The fused step on the same rows: 58.8 us where the attention alone takes
// 53.3 (pools; rows 56.5 and 52.6, at 2 bits 51.0 and 46.3, at 4 bits 64.5 and
// 60.3).  One sequence with a window of 1024 9.4 us, two launches of 5.8 and 3.4
// us; its step 11.5.
#include <hip/hip_runtime.h>
#include <math.h>

#include "iq_span_device.h"

namespace iq {
namespace {

// A head's output of its unrotated sums O and the weights' sum L, 32 threads' 4 dims
// each.  (A row that sees nothing is zero; a sum that is NaN stays visible.)
__device__ __forceinline__ f32x4_t window_result(f32x4_t O, float L, f32x4_t ql, f32x4_t qr,
                                                 int blk) {
  return rotate_inverse(O * (L == 0.f ? 0.f : 1.0f / L), ql, qr, blk);
}

template <bool kAppend, bool kAlone, bool kPaged, int kBits>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(4)))
void decode_window_kernel(
    const float* __restrict__ q, uint8_t* __restrict__ k_codes, float* __restrict__ k_norms,
    uint8_t* __restrict__ v_codes, float* __restrict__ v_norms,
    const int32_t* __restrict__ seq_lens, const float* __restrict__ quats,
    float* __restrict__ partials, float* __restrict__ out, int64_t capacity, int max_seq_len,
    int window, int n_sinks, int n_kv_heads, int n_splits, float qscale, CodebookB<kBits> cb,
    const void* __restrict__ k_new, const void* __restrict__ v_new, int new_f16,
    int32_t* __restrict__ status, PageTable pages, int group, int batch) {
  const G8Args<kBits> a{q,        k_codes, k_norms, v_codes,  v_norms,     seq_lens,
                        quats,    partials, partials, capacity, max_seq_len, n_kv_heads,
                        n_splits, 0,       qscale,  cb,       k_new,       v_new,
                        new_f16,  status,  pages,   group,    batch,       nullptr};
  __shared__ __attribute__((aligned(16))) SpanSmem<kBits, false> sm;
  const int vshift = group > kHeads ? 1 : 0;
  const int n_rows = n_kv_heads << vshift;
  const int split = blockIdx.x, y = blockIdx.y, b = blockIdx.z;
  const int g = y >> vshift, vg = y & vshift;
  const int n_parts = kAppend ? n_splits + 1 : n_splits;
  const int seq0 = seq_lens[b];
  const int len = span_length(seq0, max_seq_len);   // cached positions that can be attended
  // the first position of the window: that of the row with its new token
  int end = len;
  if constexpr (kAppend) {
    if (new_token<kPaged>(a, g, b).written) end = span_length(seq0 + 1, max_seq_len);
  }
  const int lo = end > window ? end - window : 0;
  // batches of the sinks, and of the rest that lies before the window
  const int sink_end = n_sinks < len ? (n_sinks + 15) & ~15 : (len + 15) & ~15;
  const int skip = (lo & ~15) > sink_end ? (lo & ~15) - sink_end : 0;
  const SpanHole hole{sink_end, skip, n_sinks, lo - skip};
  const int vlen = len - skip;
  const int n_bat = (vlen + 15) >> 4;
  const int a0 = static_cast<int>(static_cast<int64_t>(n_bat) * split / n_splits);
  const int a1 = static_cast<int>(static_cast<int64_t>(n_bat) * (split + 1) / n_splits);
  float* row_parts = partials + (static_cast<int64_t>(b) * n_rows + y) * n_parts * (kHeads * kPart);
  float* part = row_parts + static_cast<int64_t>(split) * (kHeads * kPart);
  const bool append = kAppend && split == 0;
  const int blk = threadIdx.x & 31, hh = static_cast<int>(threadIdx.x) >> 5;
  float* const head_out =
      out + ((static_cast<int64_t>(b) * n_kv_heads + g) * group + kHeads * vg + hh) * kDim + 4 * blk;
  const bool mine = hh < kHeads && hh < group - kHeads * vg;   // of this row's heads
  if (a1 <= a0) {
    if constexpr (kAlone) {
      if (mine) *reinterpret_cast<f32x4_t*>(head_out) = f32x4_t{0.f, 0.f, 0.f, 0.f};
      return;
    }
    if (threadIdx.x < kHeads)
      *reinterpret_cast<f32x2_t*>(part + threadIdx.x * kPart) = f32x2_t{-INFINITY, 0.f};
    if (!append) return;
  }
  build_pair_table(sm, cb, threadIdx.x);   // before the span's barriers
  attend_span<kAppend, kPaged, kBits, false, true>(
      sm, a, group, g, vg, b, a0, a1, vlen, part, append,
      row_parts + static_cast<int64_t>(n_splits) * (kHeads * kPart), hole);
  if constexpr (!kAlone) return;
  __syncthreads();   // the part, written by this workgroup's other threads
  if (hh >= kHeads) return;
  const float* p = part + hh * kPart;
  const float m = p[0], L = p[1];
  f32x4_t O = *reinterpret_cast<const f32x4_t*>(p + 2 + 4 * blk);
  // (no maximum: nothing to attend, or only NaN scores, whose sum is NaN)
  if (m == -INFINITY) O = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t x = window_result(O, L, par[0], par[1], blk);
  if (mine) *reinterpret_cast<f32x4_t*>(head_out) = x;
}

// Merge of the parts of the rows, the inverse rotation, and (fused step) the
// advance of the lengths past the tokens that were written.  A head's 128 dims
// are 32 threads' (4 each); kShare groups of them share its parts.  Workgroup:
// 8 / kShare heads of a row.
constexpr int kWindowMergeThreads = 256;
template <bool kAppend, int kShare>
__global__ __launch_bounds__(kWindowMergeThreads) void merge_window_kernel(
    const float* __restrict__ partials, const float* __restrict__ quats, float* __restrict__ out,
    int n_kv_heads, int n_parts, int32_t* __restrict__ seq_lens, int64_t capacity, int group) {
  constexpr int kUnroll = 8;
  __shared__ __attribute__((aligned(16))) f32x4_t red_o[kHeads][32];
  __shared__ float red_m[kHeads], red_l[kHeads];
  const int tid = threadIdx.x;
  const int vshift = group > kHeads ? 1 : 0;
  const int n_rows = n_kv_heads << vshift;
  const int y = static_cast<int>(blockIdx.x) / kShare, b = blockIdx.y;
  const int g = y >> vshift, vg = y & vshift;
  const int nh = group - kHeads * vg < kHeads ? group - kHeads * vg : kHeads;
  const int blk = tid & 31, slot = tid >> 5;
  const int hh = (static_cast<int>(blockIdx.x) % kShare) * (kHeads / kShare) + slot / kShare;
  const float* base =
      partials + (static_cast<int64_t>(b) * n_rows + y) * n_parts * (kHeads * kPart) + hh * kPart;
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t ql = par[0], qr = par[1];
  float M = -INFINITY, L = 0.f;
  f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s0 = slot % kShare; s0 < n_parts; s0 += kShare * kUnroll) {
    f32x2_t ml[kUnroll];
    f32x4_t o[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int s = s0 + kShare * u < n_parts ? s0 + kShare * u : s0;
      const float* p = base + static_cast<int64_t>(s) * (kHeads * kPart);
      ml[u] = *reinterpret_cast<const f32x2_t*>(p);
      o[u] = *reinterpret_cast<const f32x4_t*>(p + 2 + 4 * blk);
      if (s0 + kShare * u >= n_parts) ml[u][0] = -INFINITY;
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) top = fmaxf(top, ml[u][0]);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - top);
    L *= f;
    O *= f;
    M = top;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      // (a part with nothing to attend has no outputs: select.  One whose
      // scores are all NaN has no maximum either, but a NaN sum.)
      const bool live = ml[u][0] != -INFINITY;
      const float c = live ? __builtin_amdgcn_exp2f(ml[u][0] - M) : 0.f;
      L += c * ml[u][1];
#pragma unroll
      for (int e = 0; e < 4; ++e) O[e] += live ? c * o[u][e] : 0.f;
    }
  }
  if constexpr (kShare > 1) {
    red_o[slot][blk] = O;
    if (blk == 0) {
      red_m[slot] = M;
      red_l[slot] = L;
    }
    lds_barrier();
    if (slot % kShare != 0) return;
    for (int u = 0; u < kShare; ++u) M = fmaxf(M, red_m[slot + u]);
    L = 0.f;
    O = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int u = 0; u < kShare; ++u) {
      const float m = red_m[slot + u];
      const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      L += c * red_l[slot + u];
      O += c * red_o[slot + u][blk];
    }
  }
  const f32x4_t x = window_result(O, L, ql, qr, blk);
  if (hh < nh)
    *reinterpret_cast<f32x4_t*>(
        out + ((static_cast<int64_t>(b) * n_kv_heads + g) * group + kHeads * vg + hh) * kDim +
        4 * blk) = x;
  if constexpr (kAppend) {
    if (blockIdx.x == 0 && tid == 0) {
      // the new token's l entry: 1 where it was written
      const int seq0 = seq_lens[b];
      if (base[static_cast<int64_t>(n_parts - 1) * (kHeads * kPart) + 1] > 0.f &&
          seq0 < capacity)
        seq_lens[b] = seq0 + 1;
    }
  }
}

}  // namespace

namespace {

constexpr int64_t kWorkgroups = 512;

// Parts of a row that leave a batch per wave, of the positions that it sees.
int64_t parts_by_batches(int64_t max_seq_len, int64_t window, int64_t n_sinks) {
  // positions that the batches of a row hold at most
  const int64_t seen = (n_sinks + 15) / 16 * 16 + window + 15;
  const int64_t n_bat = ((seen < max_seq_len ? seen : max_seq_len) + 15) / 16;
  return n_bat / kWaves > 1 ? n_bat / kWaves : 1;
}

}  // namespace

// Parts per row: as many as give the chip two workgroups per CU (64 sequences of
// 8 KV heads with one part per row and a merge, 58.4 us; two 62.3, four 71.8), and
// a batch per wave at least.
int64_t window_splits(int64_t batch, int64_t n_rows, int64_t max_seq_len, int64_t window,
                      int64_t n_sinks) {
  const int64_t rows = batch * n_rows, most = parts_by_batches(max_seq_len, window, n_sinks);
  const int64_t s = rows > 0 ? kWorkgroups / rows : 1;
  return s < 1 ? 1 : (s < most ? s : most);
}

// (A row of a larger batch has fewer parts, and the parts of all rows can be fewer;
// they are never more than one per workgroup or row.)
int64_t window_most_parts(int64_t batch, int64_t n_rows, int64_t max_seq_len, int64_t window,
                          int64_t n_sinks) {
  const int64_t rows = batch * n_rows;
  if (rows >= kWorkgroups) return rows;
  const int64_t by_batches = rows * parts_by_batches(max_seq_len, window, n_sinks);
  return by_batches < kWorkgroups ? by_batches : kWorkgroups;
}

hipError_t launch_decode_window(int64_t n_splits, const float* q, uint8_t* k_codes,
                                float* k_norms, uint8_t* v_codes, float* v_norms,
                                int32_t* seq_lens, int64_t capacity, int64_t max_seq_len,
                                int64_t window, int64_t n_sinks, const float* quats,
                                int64_t batch, int64_t n_kv_heads, int64_t group, float scale,
                                float* out, float* partials, const StepAppend* append,
                                const PageTable* pages, int bits, hipStream_t stream) {
  const int64_t n_rows = n_kv_heads * ((group + kHeads - 1) / kHeads);
  const dim3 grid(static_cast<unsigned>(n_splits), static_cast<unsigned>(n_rows),
                  static_cast<unsigned>(batch));
  const float qscale = scale * kLog2e;
  const PageTable pt = pages ? *pages : PageTable{nullptr, 0, 4, 1};
  // (a window or sinks past the longest row are the whole row)
  const int win = static_cast<int>(window < max_seq_len ? window : (max_seq_len > 0 ? max_seq_len : 1));
  const int sinks = static_cast<int>(n_sinks < max_seq_len ? n_sinks : max_seq_len);
#define IQ_LAUNCH_WINDOW(APP_, ALONE_, PAGED_, BITS_)                                              \
  hipLaunchKernelGGL((decode_window_kernel<APP_, ALONE_, PAGED_, BITS_>), grid, dim3(kThreads), 0, \
                     stream, q, k_codes, k_norms, v_codes, v_norms, seq_lens, quats, partials,     \
                     out, capacity, static_cast<int>(max_seq_len), win, sinks,                     \
                     static_cast<int>(n_kv_heads), static_cast<int>(n_splits), qscale,             \
                     codebook_for<BITS_>(nullptr), append ? append->k_new : nullptr,               \
                     append ? append->v_new : nullptr, append ? append->f16 : 0,                   \
                     append ? append->status : nullptr, pt, static_cast<int>(group),               \
                     static_cast<int>(batch))
#define IQ_LAUNCH_WINDOW_A(APP_, ALONE_)      \
  if (pages) {                                \
    IQ_LAUNCH_WINDOW(APP_, ALONE_, true, 3);  \
  } else if (bits == 2) {                     \
    IQ_LAUNCH_WINDOW(APP_, ALONE_, false, 2); \
  } else if (bits == 4) {                     \
    IQ_LAUNCH_WINDOW(APP_, ALONE_, false, 4); \
  } else {                                    \
    IQ_LAUNCH_WINDOW(APP_, ALONE_, false, 3); \
  }
  const bool alone = append == nullptr && n_splits == 1;
  if (append) {
    IQ_LAUNCH_WINDOW_A(true, false)
  } else if (alone) {
    IQ_LAUNCH_WINDOW_A(false, true)
  } else {
    IQ_LAUNCH_WINDOW_A(false, false)
  }
#undef IQ_LAUNCH_WINDOW_A
#undef IQ_LAUNCH_WINDOW
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || alone) return e;
  // the rows' parts (and the new token's) merged; the step's lengths advance here
  const int n_parts = static_cast<int>(append ? n_splits + 1 : n_splits);
  // (rows of many parts are read by 8 groups of threads per head)
#define IQ_LAUNCH_WINDOW_MERGE(APP_, SHARE_)                                                      \
  hipLaunchKernelGGL((merge_window_kernel<APP_, SHARE_>),                                         \
                     dim3(static_cast<unsigned>(n_rows * SHARE_), static_cast<unsigned>(batch)),  \
                     dim3(kWindowMergeThreads), 0, stream, partials, quats, out,                  \
                     static_cast<int>(n_kv_heads), n_parts, seq_lens, capacity,                   \
                     static_cast<int>(group))
#define IQ_LAUNCH_WINDOW_MERGE_A(APP_)   \
  if (n_parts > 16) {                    \
    IQ_LAUNCH_WINDOW_MERGE(APP_, 8);     \
  } else {                               \
    IQ_LAUNCH_WINDOW_MERGE(APP_, 1);     \
  }
  if (append) {
    IQ_LAUNCH_WINDOW_MERGE_A(true)
  } else {
    IQ_LAUNCH_WINDOW_MERGE_A(false)
  }
#undef IQ_LAUNCH_WINDOW_MERGE_A
#undef IQ_LAUNCH_WINDOW_MERGE
  return hipGetLastError();
}

}  // namespace iq

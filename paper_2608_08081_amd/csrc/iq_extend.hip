// Room for new tokens on page pools, gfx950: page tables, slots and positions of the
// new tokens of a batch of sequences, from their lengths (iq_pages.hip describes the
// pools; fresh pages are the free ones of lowest index, as there).
//
// Two launches: the free pages by chunk and what every sequence asks for; then, a sequence
// to a workgroup, who comes before it, and its entries, slots and positions.  Above
// kFewRows sequences (or kFewChunks chunks) a workgroup of its own, between the two, finds
// who comes before whom: the sums that every workgroup would make grow with the square of
// the sequences.
// Bound by launches and by the latency of loads that follow each other.  In a graph, with two
// launches and with three, timed in turn: 64 rows 8.3 and 11.8 us, 1000 rows of 50542 tokens on 100000 pages
// 11.2 and 14.8, 8192 rows 32 and 41, 16384 rows 74 and 73, 32768 rows 209 and 139.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iq_g8_device.h"

namespace iq {
namespace {

constexpr int kCopyThreads = 256;
constexpr int kCopyWaves = kCopyThreads / 64;
constexpr int kChunk = 2048;                // pages of one workgroup's count
constexpr int kChunkWords = kChunk / 64;
constexpr int kFewRows = 8192, kFewChunks = 2048;
constexpr int kWaveWords = kChunkWords / kCopyWaves;   // a wave's

__device__ __forceinline__ bool in_pool(int32_t p, int n_pages) {
  return static_cast<uint32_t>(p) < static_cast<uint32_t>(n_pages);
}

// What sequence b asks for.
struct ExtendRow {
  int len, n;        // as given, n at least 0
  int k0, k1;        // the entries that its new positions lie on
  bool sane, room;
};
__device__ __forceinline__ ExtendRow extend_row(const ExtendArgs& a, int len, int n) {
  ExtendRow r;
  r.len = len;
  r.sane = r.len >= 0 && n >= 0;
  r.n = n > 0 ? n : 0;
  const int64_t cap = static_cast<int64_t>(a.max_pages) << a.page_shift;
  const int64_t end = static_cast<int64_t>(r.len) + r.n;
  r.room = r.n == 0 || end <= cap;
  r.k0 = r.k1 = 0;
  if (r.sane && r.room && r.n > 0) {
    r.k0 = r.len >> a.page_shift;
    r.k1 = static_cast<int>((end + (int64_t{1} << a.page_shift) - 1) >> a.page_shift);
  }
  return r;
}

// Workgroup c < n_chunks: the free pages of a chunk, and the counts.  The others: a
// sequence per wave, its table copied and its unmapped entries counted.
__global__ __launch_bounds__(kCopyThreads) void extend_count_kernel(ExtendArgs a) {
  __shared__ int sums[kCopyWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (static_cast<int>(blockIdx.x) < a.n_chunks) {
    const int64_t word0 = static_cast<int64_t>(blockIdx.x) * kChunkWords + wave * kWaveWords;
    int32_t held[kWaveWords];   // loaded at once
#pragma unroll
    for (int i = 0; i < kWaveWords; ++i) {
      const int64_t p = (word0 + i) * 64 + lane;
      held[i] = a.refs[p < a.n_pages ? p : 0];
    }
    int n = 0;
    int32_t before[kWaveWords];
#pragma unroll
    for (int i = 0; i < kWaveWords; ++i) {
      const int64_t p = (word0 + i) * 64 + lane;
      const uint64_t w = __ballot(p < a.n_pages && held[i] <= 0);
      before[i] = n;
      n += __builtin_popcountll(w);
      if (p < a.n_pages) {
        if (lane == 0) a.words[word0 + i] = w;
        if (a.out_refs != a.refs) a.out_refs[p] = held[i];
      }
    }
    if (lane == 0) sums[wave] = n;
    __syncthreads();
    int base = 0, total = 0;
    for (int w = 0; w < kCopyWaves; ++w) {
      base += w < wave ? sums[w] : 0;
      total += sums[w];
    }
#pragma unroll
    for (int i = 0; i < kWaveWords; ++i)
      if (lane == 0 && (word0 + i) * 64 < a.n_pages) a.prefix[word0 + i] = base + before[i];
    if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
    return;
  }
  const int64_t b = (static_cast<int64_t>(blockIdx.x) - a.n_chunks) * kCopyWaves + wave;
  if (b >= a.batch) return;
  const ExtendRow r = extend_row(a, a.seq_lens[b], a.new_lens[b]);
  const int32_t* row = a.tables + b * a.max_pages;
  int32_t* out = a.out_tables + b * a.max_pages;
  const bool copy = a.out_tables != a.tables;
  int need = 0, first = -1, last = -1;
  for (int k0 = copy ? 0 : r.k0 & ~63; k0 < (copy ? a.max_pages : r.k1); k0 += 64) {
    const int k = k0 + lane;
    const int32_t e = k < a.max_pages ? row[k] : 0;
    if (copy && k < a.max_pages) out[k] = e;
    const uint64_t open = __ballot(k >= r.k0 && k < r.k1 && !in_pool(e, a.n_pages));
    if (open) {
      need += __builtin_popcountll(open);
      first = first < 0 ? k0 + __builtin_ctzll(open) : first;
      last = k0 + 63 - __builtin_clzll(open);
    }
  }
  if (lane == 0) {
    a.lens[b] = r.len;   // (out_lens may be seq_lens)
    a.need[b] = need;
    a.first[b] = need == 0 || last - first + 1 == need ? first : ~first;
  }
}

// Whether sequence b gets its pages and tokens; its first row, length and status (write: by
// the one thread that does).
__device__ __forceinline__ bool settle_row(const ExtendArgs& a, int b, const ExtendRow& r, int need,
                                           int64_t before, int64_t start, int64_t free_pages,
                                           bool write) {
  const bool held = start + r.n <= a.n_tokens;
  const bool served = need == 0 || before + need <= free_pages;
  const bool fits = r.sane && r.room && held && served;
  if (write) {
    a.row_starts[b] = static_cast<int32_t>(start < a.n_tokens ? start : a.n_tokens);
    a.out_lens[b] = fits ? r.len + r.n : r.len;
    const int flags = (!r.sane || !held ? IQ_ERR_INVALID_ARGUMENT : 0) |
                      (r.sane && (!r.room || !served) ? IQ_ERR_CAPACITY : 0);
    if (flags && a.status != nullptr) atomicOr(a.status, flags);
  }
  return fits;
}

// One workgroup: the fresh pages and tokens before each sequence, the free pages
// before each chunk, and which sequences get their pages.
constexpr int kScanThreads = 1024;
__global__ __launch_bounds__(kScanThreads) void extend_scan_kernel(ExtendArgs a) {
  __shared__ int64_t sums[kScanThreads / 64][2];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // (x, y) of every thread before this one, and of all
  auto scan = [&](int64_t x, int64_t y, int64_t& bx, int64_t& by, int64_t& tx, int64_t& ty) {
    int64_t ix = x, iy = y;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int64_t ox = __shfl_up(static_cast<long long>(ix), m);
      const int64_t oy = __shfl_up(static_cast<long long>(iy), m);
      ix += lane >= m ? ox : 0;
      iy += lane >= m ? oy : 0;
    }
    __syncthreads();
    if (lane == 63) {
      sums[wave][0] = ix;
      sums[wave][1] = iy;
    }
    __syncthreads();
    bx = ix - x;
    by = iy - y;
    tx = ty = 0;
    for (int w = 0; w < kScanThreads / 64; ++w) {
      bx += w < wave ? sums[w][0] : 0;
      by += w < wave ? sums[w][1] : 0;
      tx += sums[w][0];
      ty += sums[w][1];
    }
  };
  int64_t free_pages = 0;
  for (int c0 = 0; c0 < a.n_chunks; c0 += kScanThreads) {
    const int c = c0 + tid;
    const int n = c < a.n_chunks ? a.counts[c] : 0;
    int64_t at, none, total, no;
    scan(n, 0, at, none, total, no);
    if (c < a.n_chunks) a.counts[c] = static_cast<int32_t>(free_pages + at);
    free_pages += total;
  }
  int64_t pages = 0, tokens = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kScanThreads) {
    const int b = b0 + tid;
    const bool there = b < a.batch;
    ExtendRow r{0, 0, 0, 0, true, true};
    int need = 0;
    if (there) {
      r = extend_row(a, a.lens[b], a.new_lens[b]);
      need = a.need[b];
    }
    int64_t before, start, tp, tt;
    scan(need, r.n, before, start, tp, tt);
    before += pages;
    start += tokens;
    if (there) {
      const int64_t end = start + r.n;
      a.before[b] = before;
      a.starts[b] = start;
      a.fits[b] = settle_row(a, b, r, need, before, start, free_pages, true) ? 1 : 0;
      if (b == a.batch - 1)
        a.row_starts[a.batch] = static_cast<int32_t>(end < a.n_tokens ? end : a.n_tokens);
    }
    pages += tp;
    tokens += tt;
  }
}

// The free page of this rank (there are more than `rank` of them), by bisection
// over the chunks, the words of one, and the bits of one.
__device__ __forceinline__ int free_page(const ExtendArgs& a, const int32_t* counts, int rank) {
  int lo = 0, hi = a.n_chunks;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (counts[m] <= rank) lo = m; else hi = m;
  }
  int r = rank - counts[lo];
  const int w0 = lo * kChunkWords;
  const int words = (a.n_pages + 63) / 64 - w0;
  lo = 0;
  hi = words < kChunkWords ? words : kChunkWords;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a.prefix[w0 + m] <= r) lo = m; else hi = m;
  }
  r -= a.prefix[w0 + lo];
  const uint64_t w = a.words[w0 + lo];
  int bit = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) {
    const int n = __builtin_popcountll(w >> bit & ((uint64_t{1} << step) - 1));
    if (n <= r) {
      r -= n;
      bit += step;
    }
  }
  return (w0 + lo) * 64 + bit;
}

// Workgroup (b, y): sequence b's entries, slots and positions, 256 entries at a time;
// (batch, y): the padding behind the last sequence.
// kScanned: who comes before whom is known.
template <bool kScanned>
__global__ __launch_bounds__(kCopyThreads) void extend_fill_kernel(ExtendArgs a) {
  __shared__ int32_t entries[kCopyThreads];
  __shared__ int ranks[kCopyWaves];
  __shared__ int64_t sums[2][kCopyWaves];
  __shared__ int32_t chunk_at[kScanned ? 1 : kFewChunks];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int b = blockIdx.x;
  int64_t pages = 0, start = 0;   // of the sequences before this one
  if (!kScanned) {
    for (int i = tid; i < b; i += kCopyThreads) {
      const int n = a.new_lens[i];
      pages += a.need[i];
      start += n > 0 ? n : 0;
    }
    for (int m = 1; m < 64; m <<= 1) {
      pages += __shfl_xor(static_cast<long long>(pages), m);
      start += __shfl_xor(static_cast<long long>(start), m);
    }
    if (lane == 0) {
      sums[0][wave] = pages;
      sums[1][wave] = start;
    }
    __syncthreads();
    pages = start = 0;
#pragma unroll
    for (int w = 0; w < kCopyWaves; ++w) {
      pages += sums[0][w];
      start += sums[1][w];
    }
  }
  if (b == a.batch) {
    int64_t end = start < a.n_tokens ? start : a.n_tokens;
    if (kScanned) end = a.row_starts[b];
    else if (tid == 0 && blockIdx.y == 0) a.row_starts[b] = static_cast<int32_t>(end);
    for (int64_t t = end + static_cast<int64_t>(blockIdx.y) * kCopyThreads + tid; t < a.n_tokens;
         t += static_cast<int64_t>(gridDim.y) * kCopyThreads) {
      a.slots[t] = -1;
      a.positions[t] = 0;
    }
    return;
  }
  const int len = a.lens[b], n = a.new_lens[b] > 0 ? a.new_lens[b] : 0, need = a.need[b];
  bool fits;
  if (kScanned) {
    pages = a.before[b];
    start = a.starts[b];
    fits = a.fits[b] != 0;
  } else {
    int64_t free_pages = 0;
    if (need > 0) {
      // the free pages before each chunk
      constexpr int kEach = kFewChunks / kCopyThreads;
      int32_t x[kEach], sum = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int c = kEach * tid + i;
        x[i] = c < a.n_chunks ? a.counts[c] : 0;
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) sum += x[i];
      int incl = sum;
      for (int m = 1; m < 64; m <<= 1) {
        const int o = __shfl_up(incl, m);
        incl += lane >= m ? o : 0;
      }
      if (lane == 63) ranks[wave] = incl;
      __syncthreads();
      int32_t at = incl - sum;
#pragma unroll
      for (int w = 0; w < kCopyWaves; ++w) {
        at += w < wave ? ranks[w] : 0;
        free_pages += ranks[w];
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        chunk_at[kEach * tid + i] = at;
        at += x[i];
      }
      __syncthreads();
    }
    fits = settle_row(a, b, extend_row(a, len, a.new_lens[b]), need, pages, start, free_pages,
                      tid == 0 && blockIdx.y == 0);
  }
  const int32_t* const counts = kScanned ? a.counts : chunk_at;
  if (!fits) {
    for (int64_t i = static_cast<int64_t>(blockIdx.y) * kCopyThreads + tid;
         i < n && start + i < a.n_tokens; i += static_cast<int64_t>(gridDim.y) * kCopyThreads) {
      a.slots[start + i] = -1;
      a.positions[start + i] = static_cast<int32_t>(len + i);
    }
    return;
  }
  if (n == 0) return;
  const int page = 1 << a.page_shift;
  const int k0 = len >> a.page_shift;
  const int k1 = static_cast<int>((static_cast<int64_t>(len) + n + page - 1) >> a.page_shift);
  const int first = a.first[b], from = first < 0 ? ~first : first;
  const bool open = need > 0;
  // mapped entries among those that are not: one workgroup takes them in order
  const bool holes = open && first < 0;
  if (holes && blockIdx.y > 0) return;
  const int64_t step = static_cast<int64_t>(holes ? 1 : gridDim.y) * kCopyThreads;
  int before = static_cast<int>(pages);
  const int32_t* row = a.out_tables + static_cast<int64_t>(b) * a.max_pages;
  for (int64_t e0 = k0 + static_cast<int64_t>(blockIdx.y) * kCopyThreads; e0 < k1; e0 += step) {
    const int k = static_cast<int>(e0) + tid;
    int32_t e = -1;
    bool fresh = false;
    if (k < k1) {
      // (a fresh entry is written by this thread alone)
      e = row[k];
      fresh = open && k >= from && !in_pool(e, a.n_pages);
    }
    int rank = before + k - from;
    if (holes) {
      const uint64_t mine = __ballot(fresh);
      if (lane == 0) ranks[wave] = __builtin_popcountll(mine);
      __syncthreads();
      rank = before + __builtin_popcountll(mine & ((uint64_t{1} << lane) - 1));
      for (int w = 0; w < kCopyWaves; ++w) {
        rank += w < wave ? ranks[w] : 0;
        before += ranks[w];
      }
    }
    if (fresh) {
      e = free_page(a, counts, rank);
      a.out_tables[static_cast<int64_t>(b) * a.max_pages + k] = e;
      a.out_refs[e] = 1;
    }
    __syncthreads();
    entries[tid] = e;
    __syncthreads();
    // the tokens on these entries
    const int64_t p0 = e0 << a.page_shift, p1 = (e0 + kCopyThreads) << a.page_shift;
    const int64_t end = static_cast<int64_t>(len) + n;
    const int64_t hi = p1 < end ? p1 : end;
    for (int64_t p = (p0 > len ? p0 : len) + tid; p < hi; p += kCopyThreads) {
      const int64_t t = start + (p - len);
      const int32_t at = entries[(p >> a.page_shift) - e0];
      a.slots[t] = (static_cast<int64_t>(at) << a.page_shift) + (p & (page - 1));
      a.positions[t] = static_cast<int32_t>(p);
    }
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

ExtendPlan extend_plan(int64_t n_pages, int64_t batch) {
  ExtendPlan p;
  const size_t chunks = static_cast<size_t>((n_pages + kChunk - 1) / kChunk);
  const size_t rows = static_cast<size_t>(batch);
  p.n_chunks = static_cast<int64_t>(chunks);
  p.words = 0;
  p.counts = align256(p.words + chunks * kChunkWords * 8);
  p.prefix = align256(p.counts + chunks * 4);
  p.before = align256(p.prefix + chunks * kChunkWords * 4);
  p.starts = align256(p.before + rows * 8);
  p.need = align256(p.starts + rows * 8);
  p.first = align256(p.need + rows * 4);
  p.fits = align256(p.first + rows * 4);
  p.lens = align256(p.fits + rows * 4);
  p.total_bytes = align256(p.lens + rows * 4);
  return p;
}

hipError_t launch_extend_pages(ExtendArgs a, void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  const ExtendPlan p = extend_plan(a.n_pages, a.batch);
  a.words = reinterpret_cast<uint64_t*>(ws + p.words);
  a.counts = reinterpret_cast<int32_t*>(ws + p.counts);
  a.prefix = reinterpret_cast<int32_t*>(ws + p.prefix);
  a.before = reinterpret_cast<int64_t*>(ws + p.before);
  a.starts = reinterpret_cast<int64_t*>(ws + p.starts);
  a.need = reinterpret_cast<int32_t*>(ws + p.need);
  a.first = reinterpret_cast<int32_t*>(ws + p.first);
  a.fits = reinterpret_cast<int32_t*>(ws + p.fits);
  a.lens = reinterpret_cast<int32_t*>(ws + p.lens);
  a.n_chunks = static_cast<int32_t>(p.n_chunks);
  const unsigned rows = static_cast<unsigned>((a.batch + kCopyWaves - 1) / kCopyWaves);
  hipLaunchKernelGGL(extend_count_kernel, dim3(static_cast<unsigned>(p.n_chunks) + rows),
                     dim3(kCopyThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // workgroups enough for a few rounds of 256 tokens each
  int64_t shares = a.n_tokens / (int64_t{a.batch} * 1024) + 1;
  shares = shares < 64 ? shares : 64;
  const dim3 grid(static_cast<unsigned>(a.batch) + 1, static_cast<unsigned>(shares));
  if (a.batch <= kFewRows && a.n_chunks <= kFewChunks) {
    hipLaunchKernelGGL(extend_fill_kernel<false>, grid, dim3(kCopyThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(extend_scan_kernel, dim3(1), dim3(kScanThreads), 0, stream, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(extend_fill_kernel<true>, grid, dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace iq

// Records moved between caches, gfx950: acceptance of a path of drafted tokens
// into the cache, forking (reordering, freeing) of sequences on page pools, and
// compaction of the pools.  Everything moved is copied bit for bit.
//
// Pools are laid out [n_pages][n_kv_heads][page_size], so a page of one array is
// one stretch of memory.  page_refs[p] counts who holds page p (table entries,
// and whatever else the caller counts, a cache of prompts for one); a page with
// a count of 0 or less is free.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iq_g8_device.h"

namespace iq {
namespace {

constexpr int kCopyThreads = 256;
constexpr int kChunk = 2048;                // pages of one workgroup's scan
constexpr int kChunkWords = kChunk / 64;
constexpr int kCopyWaves = kCopyThreads / 64;
constexpr int kWaveWords = kChunkWords / kCopyWaves;   // a wave's
constexpr int64_t kPiece = 32 << 10;        // bytes of a page's records that one workgroup copies

// n 16-byte words by the workgroup, four loads in flight per thread.
__device__ __forceinline__ void copy_words(void* dst, const void* src, int64_t n) {
  u32x4_t* d = static_cast<u32x4_t*>(dst);
  const u32x4_t* s = static_cast<const u32x4_t*>(src);
  int64_t i = threadIdx.x;
  for (; i + 3 * kCopyThreads < n; i += 4 * kCopyThreads) {
    u32x4_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = s[i + j * kCopyThreads];
#pragma unroll
    for (int j = 0; j < 4; ++j) d[i + j * kCopyThreads] = v[j];
  }
  for (; i < n; i += kCopyThreads) d[i] = s[i];
}

__device__ __forceinline__ bool in_pool(int32_t p, int n_pages) {
  return static_cast<uint32_t>(p) < static_cast<uint32_t>(n_pages);
}

// ---- acceptance ---------------------------------------------------------------
// One workgroup per sequence (it alone reads and advances the sequence's
// length): all of its records, or none and a status.  4.6 us for one sequence or
// 64: the launch and three loads that wait for each other (length and path, page
// table, record).
constexpr int kAcceptThreads = 512;
template <bool kPaged>
__global__ __launch_bounds__(kAcceptThreads) void accept_kernel(
    Cache draft, Cache cache, int64_t draft_capacity, int64_t capacity, PageTable pages,
    const int32_t* __restrict__ path, const int32_t* __restrict__ n_accept, int max_path,
    const int32_t* seq_lens, int32_t* out_lens, int32_t* __restrict__ status, int n_kv_heads,
    int bits) {
  __shared__ int64_t src_at[64], dst_at[64];   // record of KV head 0
  __shared__ int outcome;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int len = seq_lens[b], n = n_accept[b];
  if (tid < 64) {
    const bool sane = n >= 0 && n <= max_path && len >= 0;
    const bool room = sane && len <= capacity && n <= capacity - len;
    bool bad = false, lost = false;
    if (room && tid < n) {
      const int node = path[static_cast<int64_t>(b) * max_path + tid];
      bad = node < 0 || node >= draft_capacity;
      src_at[tid] = static_cast<int64_t>(b) * n_kv_heads * draft_capacity + node;
      int64_t at = static_cast<int64_t>(b) * n_kv_heads * capacity + len + tid;
      if constexpr (kPaged) {
        at = paged_record(pages, n_kv_heads, b, 0, len + tid);
        lost = at < 0;
      }
      dst_at[tid] = at;
    }
    const int flags = (!sane || __any(bad) ? IQ_ERR_INVALID_ARGUMENT : 0) |
                      ((sane && !room) || __any(lost) ? IQ_ERR_CAPACITY : 0);
    if (tid == 0) {
      outcome = flags;
      if (flags && status != nullptr) atomicOr(status, flags);
      out_lens[b] = flags ? len : len + n;
    }
  }
  __syncthreads();
  if (outcome) return;
  const int64_t src_head = draft_capacity;
  const int64_t dst_head = kPaged ? int64_t{1} << pages.page_shift : capacity;
  // 16-byte pieces of the records: piece fastest, then token, KV head, side
  const int per_side = n * bits * n_kv_heads;
  for (int e = tid; e < 2 * per_side; e += kAcceptThreads) {
    const int side = e >= per_side;
    const int r = e - side * per_side;
    const int i = r / bits % n, g = r / bits / n, piece = r % bits;
    const u32x4_t* s = reinterpret_cast<const u32x4_t*>(side ? draft.v_codes : draft.k_codes);
    u32x4_t* d = reinterpret_cast<u32x4_t*>(side ? cache.v_codes : cache.k_codes);
    d[(dst_at[i] + g * dst_head) * bits + piece] = s[(src_at[i] + g * src_head) * bits + piece];
  }
  const int per_norm = n * n_kv_heads;
  for (int e = tid; e < 2 * per_norm; e += kAcceptThreads) {
    const int side = e >= per_norm;
    const int r = e - side * per_norm;
    const int i = r % n, g = r / n;
    const float* s = side ? draft.v_norms : draft.k_norms;
    float* d = side ? cache.v_norms : cache.k_norms;
    d[dst_at[i] + g * dst_head] = s[src_at[i] + g * src_head];
  }
}

// ---- scans over pages ---------------------------------------------------------
// Words of 64 flags, and their number per chunk of kChunk pages: the pages with
// refs > 0 (kLive) or the others.
template <bool kLive>
__global__ __launch_bounds__(kCopyThreads) void flag_pages_kernel(
    const int32_t* __restrict__ refs, int n_pages, uint64_t* __restrict__ words,
    int32_t* __restrict__ counts) {
  __shared__ int sums[kCopyThreads / 64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t word0 = static_cast<int64_t>(blockIdx.x) * kChunkWords + wave;
  int32_t held[kWaveWords];   // loaded at once
#pragma unroll
  for (int i = 0; i < kWaveWords; ++i) {
    const int64_t p = (word0 + i * kCopyWaves) * 64 + lane;
    held[i] = refs[p < n_pages ? p : 0];
  }
  int n = 0;
#pragma unroll
  for (int i = 0; i < kWaveWords; ++i) {
    const int64_t word = word0 + i * kCopyWaves;
    const uint64_t w = __ballot(word * 64 + lane < n_pages && (held[i] > 0) == kLive);
    n += __builtin_popcountll(w);
    if (lane == 0 && word * 64 < n_pages) words[word] = w;
  }
  if (lane == 0) sums[wave] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    int total = 0;
    for (int i = 0; i < kCopyThreads / 64; ++i) total += sums[i];
    counts[blockIdx.x] = total;
  }
}

// Sum of v[0 .. n - 1] over the workgroup, the same in every thread.
__device__ __forceinline__ int block_total(const int32_t* v, int n) {
  __shared__ int sums[kCopyThreads / 64];
  int x = 0;
  for (int i = threadIdx.x; i < n; i += kCopyThreads) x += v[i];
  x = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = x;
  __syncthreads();
  int total = 0;
  for (int i = 0; i < kCopyThreads / 64; ++i) total += sums[i];
  return total;
}

// The same of numbers whose sum needs 64 bits (a thread's share, at most 65535 /
// 256 of them, each below 2^22, does not): the low and high halves apart.
__device__ __forceinline__ int64_t block_total64(const int32_t* v, int n) {
  __shared__ int64_t sums[kCopyThreads / 64];
  int x = 0;
  for (int i = threadIdx.x; i < n; i += kCopyThreads) x += v[i];
  const int lo = wave_scan(x & 0xFFFF), hi = wave_scan(x >> 16);
  if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = lo + (static_cast<int64_t>(hi) << 16);
  __syncthreads();
  int64_t total = 0;
  for (int i = 0; i < kCopyThreads / 64; ++i) total += sums[i];
  return total;
}

// The page with flag number `rank` (from 0), -1 if there is none; one wave, the
// same in every lane.
__device__ __forceinline__ int nth_flag(const uint64_t* words, const int32_t* counts, int n_pages,
                                        int n_chunks, int64_t rank, int lane) {
  if (rank >= n_pages) return -1;
  int r = static_cast<int>(rank);
  for (int c0 = 0; c0 < n_chunks; c0 += 64) {
    const int c = c0 + lane < n_chunks ? counts[c0 + lane] : 0;
    const int incl = wave_scan(c);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (r >= total) {
      r -= total;
      continue;
    }
    const int i = __builtin_popcountll(__ballot(incl <= r));
    r -= __builtin_amdgcn_readlane(incl - c, i);
    const int64_t w0 = static_cast<int64_t>(c0 + i) * kChunkWords;
    uint64_t word = 0;
    if (lane < kChunkWords && (w0 + lane) * 64 < n_pages) word = words[w0 + lane];
    const int n = __builtin_popcountll(word);
    const int wincl = wave_scan(n);
    const int k = __builtin_popcountll(__ballot(wincl <= r));
    r -= __builtin_amdgcn_readlane(wincl - n, k);
    const uint64_t w =
        static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(word), k)) |
        static_cast<uint64_t>(static_cast<uint32_t>(
            __builtin_amdgcn_readlane(static_cast<int>(word >> 32), k)))
            << 32;
    const bool hit = (w >> lane & 1) &&
                     __builtin_popcountll(w & ((uint64_t{1} << lane) - 1)) == r;
    return static_cast<int>((w0 + k) * 64 + __builtin_ctzll(__ballot(hit)));
  }
  return -1;
}

// ---- forking --------------------------------------------------------------------
// Four launches, each of which has to see all of the one before: the counts, the
// rows, the free pages, the fresh pages and copies.  14.4 us for 32 rows as for
// 256 (2.0 + 4.1 + 2.7 + 5.5 and the gaps): latency, no memory rate.
__global__ __launch_bounds__(kCopyThreads) void copy_refs_kernel(const int32_t* __restrict__ src,
                                                                 int32_t* __restrict__ dst,
                                                                 int n) {
  const int i = blockIdx.x * kCopyThreads + threadIdx.x;
  if (i < n) dst[i] = src[i];
}

constexpr int kPending = -2;   // a table entry that takes a fresh page

// What row i becomes: its parent, its positions, the pages wholly used and the
// pages it needs.
struct ForkRow {
  int parent, len, full, need;
};
__device__ __forceinline__ ForkRow fork_row(const ForkArgs& a, int i) {
  ForkRow r{-1, 0, 0, 0};
  const int p = a.parents[i];
  if (p < 0 || p >= a.batch) return r;
  const int64_t cap = static_cast<int64_t>(a.max_pages) << a.page_shift;
  int64_t len = a.seq_lens[p];
  len = len < 0 ? 0 : (len > cap ? cap : len);
  const int64_t room = len + a.reserve < cap ? len + a.reserve : cap;
  const int64_t page = int64_t{1} << a.page_shift;
  r.parent = p;
  r.len = static_cast<int>(len);
  r.full = static_cast<int>(len >> a.page_shift);
  r.need = static_cast<int>((room + page - 1) >> a.page_shift);
  return r;
}

// Workgroup i: the pages of input row i are let go, output row i is laid out but
// for its fresh pages.  out_refs starts as page_refs.  The source of a copy is
// held once more until the copy is made, so that it counts as used.
__global__ __launch_bounds__(kCopyThreads) void fork_rows_kernel(ForkArgs a) {
  const int i = blockIdx.x;
  if (i < a.batch) {
    const int32_t* row = a.tables + static_cast<int64_t>(i) * a.max_pages;
    for (int k = threadIdx.x; k < a.max_pages; k += kCopyThreads)
      if (in_pool(row[k], a.n_pages)) atomicSub(&a.out_refs[row[k]], 1);
  }
  if (i >= a.out_batch) return;
  const ForkRow r = fork_row(a, i);
  // the first row of its parent keeps the pages behind the full ones
  int other = 0;
  for (int k = threadIdx.x; k < i; k += kCopyThreads) other |= a.parents[k] == r.parent;
  const bool first = !__syncthreads_or(other);
  const int32_t* src = a.tables + static_cast<int64_t>(r.parent < 0 ? 0 : r.parent) * a.max_pages;
  int32_t* dst = a.out_tables + static_cast<int64_t>(i) * a.max_pages;
  int fresh = 0, copy = 0;
  for (int k = threadIdx.x; k < a.max_pages; k += kCopyThreads) {
    int32_t e = -1;
    if (k < r.need) {
      const int32_t p = src[k];
      const bool there = in_pool(p, a.n_pages);
      if (k < r.full) {
        e = there ? p : -1;
      } else if (first && there && a.refs[p] == 1) {
        e = p;
      } else {
        e = kPending;
        ++fresh;
        if (there && k == r.full && (r.len & ((1 << a.page_shift) - 1)) != 0) {
          atomicAdd(&a.out_refs[p], 1);
          copy = 1;
        }
      }
      if (e >= 0) atomicAdd(&a.out_refs[e], 1);
    }
    dst[k] = e;
  }
  for (int m = 1; m < 64; m <<= 1) fresh += __shfl_xor(fresh, m);
  __shared__ int sums[kCopyThreads / 64];
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = fresh;
  copy = __syncthreads_or(copy);
  if (threadIdx.x == 0) {
    int total = 0;
    for (int w = 0; w < kCopyThreads / 64; ++w) total += sums[w];
    a.fresh[i] = total;
    a.copies[i] = copy ? 1 : 0;
    a.out_lens[i] = r.len;
    if (a.parents[i] >= a.batch && a.status != nullptr)
      atomicOr(a.status, static_cast<int32_t>(IQ_ERR_INVALID_ARGUMENT));
  }
}

// Workgroup (i, y): row i's fresh pages (the lowest free ones, in the order of
// rows and of a row's pages; y = 0 enters them, a wave each), and a share of the
// used part of the parent's last page, which goes to the first of them.
__global__ __launch_bounds__(kCopyThreads) void fork_pages_kernel(ForkArgs a) {
  const int i = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
  const bool copy = a.copies[i] != 0;
  if (a.fresh[i] == 0 || (blockIdx.y > 0 && !copy)) return;
  __shared__ int first_page;
  // (rows that ask for all of their pages: more than 2^31 in all)
  const int64_t before = block_total64(a.fresh, i);
  const ForkRow r = fork_row(a, i);
  auto free_page = [&](int64_t rank) {
    return nth_flag(a.words, a.counts, a.n_pages, a.n_chunks, rank, lane);
  };
  if (blockIdx.y == 0) {
    int32_t* dst = a.out_tables + static_cast<int64_t>(i) * a.max_pages;
    int n = 0;   // fresh pages so far
    bool short_of = false;
    for (int k0 = r.full; k0 < r.need; k0 += 64) {
      uint64_t pending = __ballot(k0 + lane < r.need && dst[k0 + lane] == kPending);
      __syncthreads();   // every wave has read them
      for (; pending; pending &= pending - 1, ++n) {
        if (n % kCopyWaves != wave) continue;
        const int k = k0 + __builtin_ctzll(pending);
        const int p = free_page(before + n);
        if (lane == 0) {
          if (n == 0) first_page = p;
          dst[k] = p;
          if (p >= 0) {
            a.out_refs[p] = 1;
          } else {
            short_of = true;
            // positions whose page has no place are lost
            if (k == r.full) a.out_lens[i] = r.full << a.page_shift;
          }
        }
      }
    }
    if (short_of && a.status != nullptr)
      atomicOr(a.status, static_cast<int32_t>(IQ_ERR_CAPACITY));
  } else if (wave == 0) {
    const int p = free_page(before);
    if (lane == 0) first_page = p;
  }
  __syncthreads();
  if (!copy) return;
  const int32_t from = a.tables[static_cast<int64_t>(r.parent) * a.max_pages + r.full];
  if (blockIdx.y == 0 && threadIdx.x == 0) atomicSub(&a.out_refs[from], 1);
  const int to = first_page;
  if (to < 0) return;
  // a wave's task: the used records' key codes, value codes or scales of a KV head
  constexpr int kWords = kRecordBytes / 16;
  const int used = r.len & ((1 << a.page_shift) - 1);
  const int n_tasks = 3 * a.n_kv_heads, step = kCopyWaves * static_cast<int>(gridDim.y);
  for (int t = static_cast<int>(blockIdx.y) * kCopyWaves + wave; t < n_tasks; t += step) {
    const int g = t / 3, what = t - 3 * g;
    const int64_t src = (static_cast<int64_t>(from) * a.n_kv_heads + g) << a.page_shift;
    const int64_t dst = (static_cast<int64_t>(to) * a.n_kv_heads + g) << a.page_shift;
    if (what < 2) {
      u32x4_t* codes = reinterpret_cast<u32x4_t*>(what ? a.pool.v_codes : a.pool.k_codes);
      const u32x4_t* s = codes + src * kWords;
      u32x4_t* d = codes + dst * kWords;
      for (int e = lane; e < used * kWords; e += 128) {
        const int f = e + 64 < used * kWords ? e + 64 : e;
        const u32x4_t x = s[e], y = s[f];
        d[e] = x;
        d[f] = y;
      }
    } else {
      for (int e = lane; e < used; e += 64) {
        const float k = a.pool.k_norms[src + e], v = a.pool.v_norms[src + e];
        a.pool.k_norms[dst + e] = k;
        a.pool.v_norms[dst + e] = v;
      }
    }
  }
}

// ---- compaction -------------------------------------------------------------------
// With n live pages, the live pages at or past n, in order, go to the free ones
// before n, in order.  8000 pages of 26 KB, a quarter of them moved, 28.5 us: the
// copy 19 of them, 100 MB at 5.3 TB/s, which is what a large copy reaches; 500
// pages 11 us, three launches.
//
// Workgroup c (a chunk of pages): the live pages before each word of its flags,
// the lists of pages that move and of the free pages that take them, and the
// entries of the pages that do not move.
__global__ __launch_bounds__(kCopyThreads) void compact_lists_kernel(CompactArgs a) {
  const int c = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t held[kWaveWords];   // the pages' counts, loaded at once
#pragma unroll
  for (int i = 0; i < kWaveWords; ++i) {
    const int p = c * kChunk + 64 * (wave + i * kCopyWaves) + lane;
    held[i] = a.refs[p < a.n_pages ? p : 0];
  }
  const int before = block_total(a.counts, c);
  const int n_live = block_total(a.counts, a.n_chunks);
  // live pages before page n_live: those before its chunk, and in it
  const int cn = n_live / kChunk;
  int low = block_total(a.counts, cn < a.n_chunks ? cn : a.n_chunks);
  if (cn < a.n_chunks) {
    const int64_t w = static_cast<int64_t>(cn) * kChunkWords + lane;
    const int rest = n_live - cn * kChunk - 64 * lane;   // pages of the lane's word before n_live
    int n = 0;
    if (lane < kChunkWords && w * 64 < a.n_pages && rest > 0)
      n = __builtin_popcountll(a.words[w] &
                               (rest >= 64 ? ~uint64_t{0} : (uint64_t{1} << rest) - 1));
    for (int m = 1; m < 64; m <<= 1) n += __shfl_xor(n, m);
    low += n;
  }
  if (c == 0 && tid == 0) {
    a.n_live[0] = n_live;
    a.summary[0] = n_live;
    a.summary[1] = low;
  }
  // the words' prefixes, by every wave for itself
  const int64_t w = static_cast<int64_t>(c) * kChunkWords + lane;
  uint64_t word = 0;
  if (lane < kChunkWords && w * 64 < a.n_pages) word = a.words[w];
  const int n = __builtin_popcountll(word);
  const int start = before + wave_scan(n) - n;
  if (tid < kChunkWords && w * 64 < a.n_pages) a.prefix[w] = start;
#pragma unroll
  for (int j = 0; j < kWaveWords; ++j) {
    const int i = wave + j * kCopyWaves;
    const uint64_t f = static_cast<uint64_t>(__shfl(static_cast<unsigned long long>(word), i));
    const int s = __shfl(start, i);
    const int p = c * kChunk + 64 * i + lane;
    if (p >= a.n_pages) continue;
    const bool live = f >> lane & 1;
    const int rank = s + __builtin_popcountll(f & ((uint64_t{1} << lane) - 1));
    if (live && p >= n_live) {
      a.movers[rank - low] = p;
      continue;   // entered by the copy
    }
    if (!live && p < n_live) {
      a.takers[p - rank] = p;
      continue;   // likewise; its map entry is that of a free page
    }
    a.out_refs[p] = held[j];
    a.page_map[p] = live ? p : -1;
  }
}

// Workgroups 0 .. map_blocks - 1: the tables renamed.  The others: the pages'
// records, a piece at a time; the first piece also enters the page.
__global__ __launch_bounds__(kCopyThreads) void compact_move_kernel(CompactArgs a, int map_blocks) {
  const int n_live = a.summary[0], low = a.summary[1];
  if (static_cast<int>(blockIdx.x) < map_blocks) {
    const int64_t n = static_cast<int64_t>(a.batch) * a.max_pages;
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * kCopyThreads + threadIdx.x; e < n;
         e += static_cast<int64_t>(map_blocks) * kCopyThreads) {
      const int32_t p = a.tables[e];
      int32_t to = p;
      if (in_pool(p, a.n_pages)) {
        const uint64_t f = a.words[p >> 6];
        if (!(f >> (p & 63) & 1)) {
          to = -1;
        } else if (p >= n_live) {
          const int rank =
              a.prefix[p >> 6] + __builtin_popcountll(f & ((uint64_t{1} << (p & 63)) - 1));
          to = a.takers[rank - low];
        }
      }
      a.out_tables[e] = to;
    }
    return;
  }
  const int moves = n_live - low;
  const int64_t bytes = (static_cast<int64_t>(a.n_kv_heads) << a.page_shift) * kRecordBytes;
  const int pieces = static_cast<int>((bytes + kPiece - 1) / kPiece);
  const int64_t per = (bytes / 16 + pieces - 1) / pieces;   // 16-byte words of a piece
  const int64_t n_words = bytes / 16, n_norms = bytes / kRecordBytes / 4;
  const int64_t n_items = static_cast<int64_t>(moves) * pieces;
  for (int64_t e = blockIdx.x - map_blocks; e < n_items; e += gridDim.x - map_blocks) {
    const int i = static_cast<int>(e / pieces), piece = static_cast<int>(e % pieces);
    const int from = a.movers[i], to = a.takers[i];
    const int64_t w0 = piece * per, w1 = w0 + per < n_words ? w0 + per : n_words;
    if (w1 > w0) {
      const int64_t s = from * n_words + w0, d = to * n_words + w0;
      copy_words(a.pool.k_codes + 16 * d, a.pool.k_codes + 16 * s, w1 - w0);
      copy_words(a.pool.v_codes + 16 * d, a.pool.v_codes + 16 * s, w1 - w0);
    }
    if (piece == 0) {
      copy_words(a.pool.k_norms + 4 * to * n_norms, a.pool.k_norms + 4 * from * n_norms, n_norms);
      copy_words(a.pool.v_norms + 4 * to * n_norms, a.pool.v_norms + 4 * from * n_norms, n_norms);
      if (threadIdx.x == 0) {
        // (refs may be out_refs: a page that takes another was free, one that
        // moves is free afterwards)
        a.out_refs[to] = a.refs[from];
        a.out_refs[from] = 0;
        a.page_map[from] = to;
        a.page_map[to] = -1;
      }
    }
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

hipError_t launch_accept(const Cache& draft, int64_t draft_capacity, const Cache& cache,
                         int64_t capacity, const PageTable* pages, const int32_t* path,
                         int64_t max_path, const int32_t* n_accept, const int32_t* seq_lens,
                         int32_t* out_lens, int32_t* status, int64_t batch, int64_t n_kv_heads,
                         int bits, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(batch));
  const PageTable pt = pages ? *pages : PageTable{nullptr, 0, 4, 1};
#define IQ_LAUNCH_ACCEPT(PAGED_)                                                             \
  hipLaunchKernelGGL(accept_kernel<PAGED_>, grid, dim3(kAcceptThreads), 0, stream, draft, cache, \
                     draft_capacity, capacity, pt, path, n_accept, static_cast<int>(max_path),   \
                     seq_lens, out_lens, status, static_cast<int>(n_kv_heads), bits)
  if (pages) {
    IQ_LAUNCH_ACCEPT(true);
  } else {
    IQ_LAUNCH_ACCEPT(false);
  }
#undef IQ_LAUNCH_ACCEPT
  return hipGetLastError();
}

PagesPlan pages_plan(int64_t n_pages, int64_t rows) {
  PagesPlan p;
  const size_t chunks = static_cast<size_t>((n_pages + kChunk - 1) / kChunk);
  p.n_chunks = static_cast<int64_t>(chunks);
  p.words = 0;
  p.counts = align256(p.words + chunks * kChunkWords * 8);
  p.prefix = align256(p.counts + chunks * 4);            // compaction: live pages before a word
  p.pages0 = align256(p.prefix + chunks * kChunkWords * 4);
  p.pages1 = align256(p.pages0 + static_cast<size_t>(n_pages) * 4);
  p.rows0 = align256(p.pages1 + static_cast<size_t>(n_pages) * 4);
  p.rows1 = align256(p.rows0 + static_cast<size_t>(rows) * 4);
  p.summary = align256(p.rows1 + static_cast<size_t>(rows) * 4);
  p.total_bytes = p.summary + 256;
  return p;
}

hipError_t launch_fork_pages(ForkArgs a, const int32_t* page_refs, void* workspace,
                             hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  const PagesPlan p = pages_plan(a.n_pages, a.out_batch);
  a.words = reinterpret_cast<uint64_t*>(ws + p.words);
  a.counts = reinterpret_cast<int32_t*>(ws + p.counts);
  a.fresh = reinterpret_cast<int32_t*>(ws + p.rows0);
  a.copies = reinterpret_cast<int32_t*>(ws + p.rows1);
  a.n_chunks = static_cast<int>(p.n_chunks);
  // the counts as they are now, beside those that change: in place, a copy of
  // them is kept
  a.refs = page_refs;
  int32_t* copy = a.out_refs;
  if (a.out_refs == page_refs) {
    copy = reinterpret_cast<int32_t*>(ws + p.pages0);
    a.refs = copy;
  }
  hipLaunchKernelGGL(copy_refs_kernel,
                     dim3(static_cast<unsigned>((a.n_pages + int64_t{kCopyThreads} - 1) / kCopyThreads)),
                     dim3(kCopyThreads), 0, stream, page_refs, copy, a.n_pages);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = a.batch > a.out_batch ? a.batch : a.out_batch;
  hipLaunchKernelGGL(fork_rows_kernel, dim3(static_cast<unsigned>(rows)), dim3(kCopyThreads), 0,
                     stream, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.out_batch == 0) return hipSuccess;
  hipLaunchKernelGGL(flag_pages_kernel<false>, dim3(static_cast<unsigned>(p.n_chunks)),
                     dim3(kCopyThreads), 0, stream, a.out_refs, a.n_pages, a.words, a.counts);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  // a task per wave, to a limit
  int64_t shares = (3 * int64_t{a.n_kv_heads} + kCopyThreads / 64 - 1) / (kCopyThreads / 64);
  shares = shares < 64 ? shares : 64;
  hipLaunchKernelGGL(fork_pages_kernel,
                     dim3(static_cast<unsigned>(a.out_batch), static_cast<unsigned>(shares)),
                     dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_compact_pages(CompactArgs a, void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  const PagesPlan p = pages_plan(a.n_pages, a.batch);
  a.words = reinterpret_cast<uint64_t*>(ws + p.words);
  a.counts = reinterpret_cast<int32_t*>(ws + p.counts);
  a.prefix = reinterpret_cast<int32_t*>(ws + p.prefix);
  a.movers = reinterpret_cast<int32_t*>(ws + p.pages0);
  a.takers = reinterpret_cast<int32_t*>(ws + p.pages1);
  a.summary = reinterpret_cast<int32_t*>(ws + p.summary);
  a.n_chunks = static_cast<int>(p.n_chunks);
  const dim3 chunks(static_cast<unsigned>(p.n_chunks));
  hipLaunchKernelGGL(flag_pages_kernel<true>, chunks, dim3(kCopyThreads), 0, stream, a.refs,
                     a.n_pages, a.words, a.counts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(compact_lists_kernel, chunks, dim3(kCopyThreads), 0, stream, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int64_t entries = static_cast<int64_t>(a.batch) * a.max_pages;
  int64_t map_blocks = (entries + 4 * kCopyThreads - 1) / (4 * kCopyThreads);
  map_blocks = map_blocks < 256 ? map_blocks : 256;
  int64_t move_blocks = (static_cast<int64_t>(a.n_pages) + 1) / 2;
  move_blocks = move_blocks < 2048 ? move_blocks : 2048;
  hipLaunchKernelGGL(compact_move_kernel, dim3(static_cast<unsigned>(map_blocks + move_blocks)),
                     dim3(kCopyThreads), 0, stream, a, static_cast<int>(map_blocks));
  return hipGetLastError();
}

}  // namespace iq

// Attention of chunks of new tokens over packed page pools (App. A per token; Table 2
// A-D), gfx950: sequences of a batch bring any number of tokens each, packed one after
// the other, whose records the pools already hold at the sequences' last positions;
// every token sees the positions up to its own (or a window of them, and sinks).
//
// For a KV head the rows (token, query head of the group) of a sequence share every key
// and value.  A workgroup takes a block of consecutive rows, decodes each tile of 32
// records that they see once into fp16 in LDS and multiplies it with all of the rows
// on the matrix cores: the products, layouts and softmax of iq_decode_tree.hip.  Queries
// are pairs of fp16 parts; so are, for fp32 queries (kLo), the products of weights and
// value scales.  With fp16 queries, whose outputs are rounded to fp16 again, these are
// one fp16 each, off by at most 2^-11, independently over the positions: an output is
// off by less than by its own rounding.
//
// Work decomposition: a kernel of its own rotates the queries and lists the pieces, a
// block of rows and a stretch of the tiles that it sees.  Blocks are cut where they have
// more than an even share of all tiles, so few rows over long contexts fill the chip;
// the parts of a block that is cut are merged and rotated back by a third kernel, a
// block in one piece is rotated back where it is made.  Consecutive workgroups are of
// different KV heads: with 8 of them each XCD's cache holds the records of one.
#include <hip/hip_runtime.h>
#include <math.h>

#include "iq_tile_device.h"

namespace iq {
namespace {

// Rows row0 .. of sequence b, tiles t0 .. t1 - 1 of those that they see (row0 < 0: no
// piece); part: where its results go, -1 for the output; start, n, len: the sequence's
// first token, tokens and length.
struct PrefillPiece {
  int32_t b, row0, t0, t1, part, start, n, len;
};
// A block of rows in several parts.
struct PrefillSplit {
  int32_t b, row0, part0, parts;
};

constexpr int kQBytes = 4 * kDim;   // of a rotated query: two fp16 parts of every entry

struct PrefillArgs {
  const void* q;
  const uint8_t* k_codes;
  const float* k_norms;
  const uint8_t* v_codes;
  const float* v_norms;
  const int32_t* row_starts;
  const int32_t* seq_lens;
  const float* quats;
  void* out;
  int64_t q_stride, out_stride;
  int32_t n_tokens, n_rows;   // rows of a KV head: n_tokens * group
  int32_t max_seq_len, batch, n_kv_heads, group, window, n_sinks;
  int32_t block_rows, shares, round_tiles, max_pieces, max_parts, max_splits;
  uint32_t group_magic;       // 2^32 / group rounded up (a group of 1: 0)
  int32_t unit_chunks, unit_len;   // a sequence's stretches of value scales, 0: none
  float qscale;
  PageTable pages;
  // workspace
  char* q_op;             // [n_kv_heads][n_rows][2 parts][128] fp16
  float* q_down;          // [n_kv_heads][n_rows]: 2^-(exponent of the parts)
  PrefillPiece* pieces;   // [max_pieces]
  PrefillSplit* splits;   // [max_splits]
  int32_t* n_splits;
  float* units;           // [batch][n_kv_heads][unit_chunks]: a stretch's largest value scale
  float* part_ml;         // [max_parts][n_kv_heads][block_rows][2]
  float* part_o;          // [max_parts][n_kv_heads][block_rows][128]
};

// r / group for r < 2^27 (the error of r magic / 2^32 is below 2^27 16 / 2^32 < 1).
__device__ __forceinline__ int row_token(const PrefillArgs& a, int r) {
  const uint32_t x = static_cast<uint32_t>(r);
  return static_cast<int>(a.group_magic ? __umulhi(x, a.group_magic) : x);
}

// A sequence: its first token, its tokens, its length.
struct PrefillSequence {
  int start, n, len;
};
__device__ __forceinline__ PrefillSequence prefill_sequence(const PrefillArgs& a, int b) {
  auto clamped = [&](int x) { return x < 0 ? 0 : (x > a.n_tokens ? a.n_tokens : x); };
  const int s = clamped(a.row_starts[b]), e = clamped(a.row_starts[b + 1]);
  return PrefillSequence{s, e > s ? e - s : 0, span_length(a.seq_lens[b], a.max_seq_len)};
}

// The first position of the window of a token at p.
__device__ __forceinline__ int window_start(const PrefillArgs& a, int p) {
  return a.window > 0 && p - a.window + 1 > 0 ? p - a.window + 1 : 0;
}

// The tiles that a block of rows sees: those of the sinks (n_sink of them), then, `skip`
// tiles on, those from its first token's window to its last token.
struct PrefillTiles {
  int n_sink, skip, n;
  int lo, end;   // first position of the first token's window, behind the last token
};
__device__ __forceinline__ PrefillTiles prefill_tiles(const PrefillArgs& a,
                                                      const PrefillSequence& s, int row0) {
  const int rows = s.n * a.group;
  const int last = row0 + a.block_rows < rows ? row0 + a.block_rows : rows;
  const int i0 = row_token(a, row0), i1 = row_token(a, last - 1);
  PrefillTiles t;
  const int p0 = s.len - s.n + i0;
  t.end = s.len - s.n + i1 + 1;
  t.end = t.end > 0 ? t.end : 0;
  t.lo = window_start(a, p0);
  const int seen = a.n_sinks < t.end ? a.n_sinks : t.end;
  t.n_sink = (seen + kTile - 1) / kTile;
  t.skip = t.lo / kTile > t.n_sink ? t.lo / kTile - t.n_sink : 0;
  t.n = (t.end + kTile - 1) / kTile - t.skip;
  return t;
}

// ---- the pieces and the rotated queries ------------------------------------------
constexpr int kPrepThreads = 256;
constexpr int kPrepRows = kPrepThreads / 32;
constexpr int kPlanChunk = 1024;   // sequences whose blocks are listed together

// The plan counts in the time of an eighth of a tile of a full block, and its figures only choose
// among ways to cut.  A tile takes a workgroup 1.3 us (2048 tokens of 32768), a piece's start and
// end 5 each: 8 tiles.  The others were set by trial.  Times in us with what is here and with
// other values (32 query heads, fp16, unless said; one of 14 kinds of batches that a value is
// not named with moved by less than 4 %):
//   kPieceWork 8 tiles; 4; 16       4 chunks, 16 single tokens 227; 227; 236
//   kMergeWork 18 tiles; 9; 36      2048 of 32768 1395; 1418; 1398; 512 of 8192 with a window 57;
//                                   57; 75; 64 of 32768 with a window 40; 40; 42; three short
//                                   prompts 54; 50; 61; fp32 chunks with a window 175; 175; 158
//   tiles of few rows cheaper; not  4 chunks, 16 single tokens 227; 222
//   their pieces finer (0.35); not  the same 227; 249; 64 single tokens 124; 136; 256 of 8000 beside
//                                   32 single tokens 168; 158, in fp32 beside 3 141; 107; three
//                                   short prompts 54; 50
//   0.7 of the longest; 0.5; 1      512 of 8192 with a window 57; 62; 57; fp32 with a window 175;
//                                   157; 175
//   an eighth more; 0; a quarter    256 of 8000 beside 32 168; 230; 168; 64 single tokens 124; 119;
//                                   127; 4 chunks, 16 single tokens 227; 223; 218; three short
//                                   prompts 54; 50; 53
constexpr int kWays = 8, kBuckets = 16;
constexpr float kTileWork = 8.0f;
// What a piece takes besides its tiles; a part of 256 rows, which is written and read again.
constexpr float kPieceWork = 8 * kTileWork, kMergeWork = 18 * kTileWork;

// A block of rows that a wave of eight has little of: seven waves only decode.
__device__ __forceinline__ float tile_work(const PrefillArgs& a, int rows) {
  return a.block_rows < 256 || rows >= a.block_rows ? kTileWork
         : rows <= kTile && a.unit_chunks > 0       ? 2.0f
                                                    : 4.0f + static_cast<float>((rows + 63) / 64);
}

// The pieces of a block of n tiles at about tau of work to a piece (an eighth more does; 0:
// one piece).
__device__ __forceinline__ int pieces_of(int n, float work, float tau) {
  const int p = static_cast<int>(
      ceilf(static_cast<float>(n) * work * __builtin_amdgcn_rcpf(tau) - 0.125f));
  return tau > 0.f && p > 1 ? (p < n ? p : n) : 1;
}

// One workgroup lists the pieces, in four passes over the blocks of rows: their work; what
// the ways to cut them would take; how many pieces there are of each size; the pieces.
// (One loop for all passes: the code of a pass is short, and a call of a few blocks spends
// most of its time on fetching it.)
__device__ __forceinline__ void plan_pieces(const PrefillArgs& a) {
  constexpr int kWaves = kPrepThreads / 64, kEach = kPlanChunk / kPrepThreads;
  __shared__ PrefillSequence seqs[kPlanChunk];
  __shared__ int starts[kPlanChunk];   // blocks of the chunk before each sequence's
  __shared__ int sums[2][kWaves];
  __shared__ float ways[kWaves][kWays][4];
  __shared__ int buckets[kBuckets];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  // x and y of the threads before this one; their sums over all
  auto scan = [&](int (&v)[2], int (&total)[2]) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int incl = wave_scan(v[i]);
      if (lane == 63) sums[i][wave] = incl;
      v[i] = incl - v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      total[i] = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        v[i] += w < wave ? sums[i][w] : 0;
        total[i] += sums[i][w];
      }
    }
  };
  const int block_shift = 31 - __builtin_clz(a.block_rows);
  auto blocks_of = [&](const PrefillSequence& s) {
    return (s.n * a.group + a.block_rows - 1) >> block_shift;
  };
  // the time of a piece of n tiles
  const float shares = static_cast<float>(a.shares);
  const float round = static_cast<float>(a.round_tiles), by_round = 1.0f / round;
  auto piece_work = [&](float n, float work) {
    return ceilf(n * by_round) * round * work + kPieceWork;
  };
  // a row of a part, written and read again by all of the chip
  const float merge = kMergeWork / 65536.0f * static_cast<float>(a.n_kv_heads) * shares;
  int chunk = -1, blocks = 0;      // the chunk of sequences that is loaded, its blocks
  float total = 0.f, tau = 0.f, largest = 1.f;
  int base[2] = {0, 0};            // parts and splits so far
  const int way = tid & (kWays - 1);
  if (tid < kBuckets) buckets[tid] = 0;
  for (int pass = 0; pass < 4; ++pass) {
    // of pass 0 the work and the blocks; of pass 1 this lane's way's pieces, parts, time of
    // all and of the longest
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < a.batch; c0 += kPlanChunk) {
      if (chunk != c0) {
        chunk = c0;
        __syncthreads();
        int v[2] = {0, 0}, sum[2];
        PrefillSequence s[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          const int b = c0 + kEach * tid + i;
          s[i] = b < a.batch ? prefill_sequence(a, b) : PrefillSequence{0, 0, 0};
          v[0] += blocks_of(s[i]);
        }
        scan(v, sum);
        blocks = sum[0];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          seqs[kEach * tid + i] = s[i];
          starts[kEach * tid + i] = v[0];
          v[0] += blocks_of(s[i]);
        }
        __syncthreads();
      }
      const int shift = pass == 1 ? 3 : 0;   // threads of a block: one for each way
      for (int i0 = 0; i0 < blocks; i0 += kPrepThreads >> shift) {
        const int i = i0 + (tid >> shift);
        const bool there = i < blocks;
        // block i: its sequence (those without blocks share their start with the next one:
        // the last of them has it), its first row, its tiles and their work
        int j = 0;
        const int rows_here = a.batch - c0 < kPlanChunk ? a.batch - c0 : kPlanChunk;
        for (int step = 1 << (31 - __builtin_clz(rows_here)); step > 0; step >>= 1)
          if (j + step < kPlanChunk && starts[j + step] <= i) j += step;
        const PrefillSequence s = seqs[there ? j : 0];
        const int row0 = there ? (i - starts[j]) << block_shift : 0;
        const int n = there ? prefill_tiles(a, s, row0).n : 0;
        const float nf = static_cast<float>(n), work = tile_work(a, s.n * a.group - row0);
        if (pass == 0) {
          f[0] += nf * work;
          f[1] += there ? 1.f : 0.f;
          continue;
        }
        // (blocks of few rows are cut finer, their parts are small)
        const float rows_f = fminf(static_cast<float>(s.n * a.group - row0),
                                   static_cast<float>(a.block_rows));
        const float small = rows_f * 8.0f <= static_cast<float>(a.block_rows) ? 0.35f : 1.0f;
        const int pieces = there ? pieces_of(n, work, tau * small) : 0;
        const float p = static_cast<float>(pieces);
        const float w = piece_work(ceilf(nf * __builtin_amdgcn_rcpf(fmaxf(p, 1.f)) - 0.01f), work);
        if (pass == 1) {
          f[0] += p;
          f[1] += pieces > 1 ? p : 0.f;
          f[2] += p * w + (pieces > 1 ? p * merge * rows_f : 0.f);
          f[3] = there ? fmaxf(f[3], w) : f[3];
          continue;
        }
        // the longest pieces first, by sixteenths of the longest
        int k = static_cast<int>((1.0f - w / largest) * static_cast<float>(kBuckets));
        k = k < 0 ? 0 : (k < kBuckets ? k : kBuckets - 1);
        if (pass == 2) {
          if (there) atomicAdd(&buckets[k], pieces);
          continue;
        }
        int v[2] = {pieces > 1 ? pieces : 0, pieces > 1 ? 1 : 0}, sum[2];
        scan(v, sum);
        const int part = base[0] + v[0], at = base[1] + v[1];
        base[0] += sum[0];
        base[1] += sum[1];
        if (!there) continue;
        // (there is room for all of them where row_starts is as it should be; where its rows
        // overlap, what does not fit is left out)
        const int b = c0 + j;
        const int to = atomicAdd(&buckets[k], pieces);
        const bool cut = pieces > 1 && part + pieces <= a.max_parts && at < a.max_splits;
        if (cut) a.splits[at] = PrefillSplit{b, row0, part, pieces};
        const int each = n / pieces, more = n - each * pieces;
        int t = 0;
        for (int q = 0; q < pieces && to + q < a.max_pieces; ++q) {
          const int t1 = t + each + (q < more ? 1 : 0);
          a.pieces[to + q] =
              pieces == 1 || cut
                  ? PrefillPiece{b, row0, t, t1, cut ? part + q : -1, s.start, s.n, s.len}
                  : PrefillPiece{0, -1, 0, 0, -1, 0, 0, 0};
          t = t1;
        }
      }
    }
    if (pass < 2) {
      // over the lanes of a way (pass 0: over all)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = f[e];
        for (int m = pass == 0 ? 1 : kWays; m < 64; m <<= 1) {
          const float o = __shfl_xor(x, m);
          x = e < 3 ? x + o : fmaxf(x, o);
        }
        if (lane < kWays) ways[wave][lane][e] = x;
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v)
          f[e] = e < 3 ? f[e] + ways[v][way][e] : fmaxf(f[e], ways[v][way][e]);
      }
      __syncthreads();
    }
    if (pass == 0) {
      // This lane's way to cut, by the work of a piece (0: none are cut): what makes at most
      // one round of the chip's workgroups, or an eighth to three times as many pieces.
      total = f[0];
      const float lone = shares - f[1];
      const float by = way == 0   ? 0.f
                       : way == 1 ? (lone > 0.f ? __builtin_amdgcn_rcpf(lone) * shares : 0.f)
                       : way < 7  ? static_cast<float>(1 << (6 - way)) * 0.5f
                                  : 0.33333334f;
      tau = total / shares * by;
    } else if (pass == 1) {
      // The least time: the longest piece, or the rounds of the pieces at their mean, and the
      // parts.  (A way that needs more room than there is: none.  Not cutting always fits;
      // splits are at most half of the parts.)
      const float rounds = ceilf(f[0] / shares) / fmaxf(f[0], 1.f) * f[2];
      const bool fits = way == 0 || (tau > 0.f && f[0] <= static_cast<float>(a.max_pieces) &&
                                     f[1] <= static_cast<float>(a.max_parts));
      float cost = fits ? fmaxf(fminf(rounds, f[2] / shares + 0.7f * f[3]), f[3]) : INFINITY;
      largest = f[3];
      for (int m = 1; m < kWays; m <<= 1) {
        const float oc = __shfl_xor(cost, m), ot = __shfl_xor(tau, m), ol = __shfl_xor(largest, m);
        // (both lanes of a pair choose alike: the lower way where the costs are equal)
        const bool other = oc < cost || (oc == cost && (way & m));
        cost = other ? oc : cost;
        tau = other ? ot : tau;
        largest = other ? ol : largest;
      }
    } else if (pass == 2) {
      __syncthreads();
      int from = 0;
      for (int k = 0; k < kBuckets; ++k) from += k < tid ? buckets[k] : 0;
      __syncthreads();
      if (tid < kBuckets) buckets[tid] = from;
      __syncthreads();
    }
  }
  __syncthreads();
  // (the last bucket ends where all pieces do)
  const int pieces = buckets[kBuckets - 1];
  if (tid == 0) a.n_splits[0] = base[1] < a.max_splits ? base[1] : a.max_splits;
  for (int p = pieces + tid; p < a.max_pieces; p += kPrepThreads)
    a.pieces[p] = PrefillPiece{0, -1, 0, 0, -1, 0, 0, 0};
}

__device__ __forceinline__ f32x4_t load4(const float* p) {
  return *reinterpret_cast<const f32x4_t*>(p);
}
__device__ __forceinline__ f32x4_t load4(const _Float16* p) {
  typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
  const half4_t h = *reinterpret_cast<const half4_t*>(p);
  return f32x4_t{static_cast<float>(h[0]), static_cast<float>(h[1]), static_cast<float>(h[2]),
                 static_cast<float>(h[3])};
}
__device__ __forceinline__ void store4(float* p, f32x4_t x) {
  *reinterpret_cast<f32x4_t*>(p) = x;
}
__device__ __forceinline__ void store4(_Float16* p, f32x4_t x) {
  typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
  *reinterpret_cast<half4_t*>(p) =
      half4_t{static_cast<_Float16>(x[0]), static_cast<_Float16>(x[1]),
              static_cast<_Float16>(x[2]), static_cast<_Float16>(x[3])};
}

// The largest finite value scale of a stretch of a sequence, of those that some new token sees:
// the sinks, and from the first token's window on.  (What lies between may be anything, on pages
// that are not mapped too: they would read another sequence's.)
__device__ __forceinline__ void largest_scale(const PrefillArgs& a, int stretch, int g) {
  __shared__ float red[kPrepThreads / 64];
  const int tid = threadIdx.x;
  const int b = stretch / a.unit_chunks, c = stretch - b * a.unit_chunks;
  const PrefillSequence s = prefill_sequence(a, b);
  const int p0 = c * a.unit_len, p1 = s.n > 0 ? (p0 + a.unit_len < s.len ? p0 + a.unit_len : s.len) : 0;
  // the stretch's first n_sink positions, then `skip` positions on those of windows, n in all
  const int ends = a.n_sinks < p1 ? a.n_sinks : p1, n_sink = ends > p0 ? ends - p0 : 0;
  const int lo = window_start(a, s.len - s.n);
  const int skip = lo > p0 + n_sink ? lo - p0 - n_sink : 0;
  const int n = p1 - p0 - skip > n_sink ? p1 - p0 - skip : n_sink;
  float largest = 0.f;
  constexpr int kAhead = 16;
  const int32_t* const table = a.pages.tables + static_cast<int64_t>(b) * a.pages.max_pages;
  for (int q0 = tid; q0 < n; q0 += kAhead * kPrepThreads) {
    int32_t entry[kAhead];
    float v[kAhead];
    auto position = [&](int u) {
      const int q = q0 + u * kPrepThreads < n ? q0 + u * kPrepThreads : q0;
      return p0 + (q < n_sink ? q : q + skip);
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) entry[u] = table[position(u) >> a.pages.page_shift];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int p = position(u);
      const int64_t page = static_cast<uint32_t>(entry[u]) < static_cast<uint32_t>(a.pages.n_pages)
                               ? entry[u]
                               : 0;
      v[u] = a.v_norms[((page * a.n_kv_heads + g) << a.pages.page_shift) +
                       (p & ((1 << a.pages.page_shift) - 1))];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      largest = fabsf(v[u]) < INFINITY ? fmaxf(largest, fabsf(v[u])) : largest;
  }
  largest = wave64_max(largest);
  if ((tid & 63) == 0) red[tid >> 6] = largest;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kPrepThreads / 64; ++w) largest = fmaxf(largest, red[w]);
    a.units[(static_cast<int64_t>(b) * a.n_kv_heads + g) * a.unit_chunks + c] = largest;
  }
}

// Grid (1 + batch * unit_chunks + blocks of 32 rows, n_kv_heads): the pieces, the largest
// value scales, and the rotated queries of 32 rows of a KV head, each by 32 lanes, lane blk
// its dims 4 blk .. 4 blk + 3.
template <typename T>
__global__ __launch_bounds__(kPrepThreads) void prefill_prep_kernel(PrefillArgs a) {
  const int tid = threadIdx.x, g = blockIdx.y;
  if (blockIdx.x == 0) {
    if (g == 0) plan_pieces(a);
    return;
  }
  const int stretches = a.batch * a.unit_chunks;
  if (static_cast<int>(blockIdx.x) <= stretches) {
    largest_scale(a, static_cast<int>(blockIdx.x) - 1, g);
    return;
  }
  const int blk = tid & 31;
  const int r0 = (static_cast<int>(blockIdx.x) - 1 - stretches) * kTile;
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t ql = par[0], qr = par[1];
  constexpr int kEach = kTile / kPrepRows;
  f32x4_t y[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = r0 + (tid >> 5) + kPrepRows * i;
    const int rc = r < a.n_rows ? r : a.n_rows - 1;   // every lane takes part
    const int t = row_token(a, rc), h = rc - t * a.group;
    y[i] = load4(static_cast<const T*>(a.q) + static_cast<int64_t>(t) * a.q_stride +
                 (static_cast<int64_t>(g) * a.group + h) * kDim + 4 * blk);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = r0 + (tid >> 5) + kPrepRows * i;
    y[i] = rotate_forward(y[i], ql, qr, blk, kInvSqrtDim * a.qscale);
    const float am = group32_max(fmaxf(fmaxf(fabsf(y[i][0]), fabsf(y[i][1])),
                                       fmaxf(fabsf(y[i][2]), fabsf(y[i][3]))));
    // an exact power of two brings the row's largest entry below 2^14
    int e = 0;
    if (am > 0.f && am < INFINITY) {
      frexpf(am, &e);
      e = 14 - e;
      e = e > 100 ? 100 : (e < -100 ? -100 : e);
    }
    const float up = ldexpf(1.0f, e);
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float x0 = y[i][2 * j] * up, x1 = y[i][2 * j + 1] * up;
      const _Float16 h0 = static_cast<_Float16>(x0), h1 = static_cast<_Float16>(x1);
      hi[j] = __builtin_bit_cast(uint32_t, half2_t{h0, h1});
      lo[j] = __builtin_bit_cast(uint32_t,
                                 half2_t{static_cast<_Float16>(x0 - static_cast<float>(h0)),
                                         static_cast<_Float16>(x1 - static_cast<float>(h1))});
    }
    if (r < a.n_rows) {
      const int64_t row = static_cast<int64_t>(g) * a.n_rows + r;
      uint2* dst = reinterpret_cast<uint2*>(a.q_op + row * kQBytes + 8 * blk);
      dst[0] = uint2{hi[0], hi[1]};
      dst[32] = uint2{lo[0], lo[1]};
      // (0 for a row of zeros, infinities or NaN: it does not count for the exponent that a
      // block shares, and stays what it is)
      if (blk == 0) a.q_down[row] = am > 0.f && am < INFINITY ? ldexpf(1.0f, -e) : 0.f;
    }
  }
}

// ---- the attention -----------------------------------------------------------------
// What a row sees: positions below end, from lo on or below the sinks' end.
struct PrefillView {
  int32_t end, lo;
  float down;   // 2^-(exponent of the query parts)
  int32_t pad;
};

template <int kRows>
constexpr int prefill_waves() {
  return kRows == 8 ? 8 : 4;
}

// Grid (pieces * KV heads + KV head).  kRows: waves of 32 rows; below four, groups of waves share the tiles of the piece.
// The loops are those of iq_decode_tree.hip: with few rows a tile after the other; with
// four or eight waves of rows a tile's scores are multiplied while the next tile is
// decoded, and the tile before multiplied with its values while its weights are computed.
template <int kRows, typename T>
__global__ __launch_bounds__(64 * prefill_waves<kRows>()) __attribute__((amdgpu_waves_per_eu(2)))
void prefill_kernel(PrefillArgs a, Codebook cb) {
  constexpr bool kLo = sizeof(T) == 4;
  constexpr int kWavesHere = prefill_waves<kRows>(), kThreadsHere = 64 * kWavesHere;
  constexpr int kRB = kRecordBytes;
  constexpr int kGroups = kWavesHere / kRows;
  constexpr int kPair = kRows == 8 ? 2 : 1;   // tiles of a barrier, decoded by four waves each
  using Decode = TileDecode<(kRows == 8 ? 4 : kRows), 3>;
  constexpr int kKeyBufs = kRows == 1 ? 1 : 2 * kPair;
  constexpr int kValueBufs = kRows >= 4 ? 3 * kPair : kKeyBufs;
  struct Smem {
    uint32_t lut[64];
    union {
      PrefillView view[kTile];   // what the wave's rows see,
      float ml[kTile][2];        // in the end their references and sums
    } rows[kWavesHere];
    float red[kWavesHere];
    union {
      struct {
        char k[kGroups][kKeyBufs][kKeyBytes];
        char v[kGroups][kValueBufs][kValueBytes];
        float sc[kWavesHere][kKeyBufs][2 * kTile];   // a wave's: key scales, value scales
      } t;
      float o[kWavesHere][kTile][kORow];
    };
  };
  __shared__ __attribute__((aligned(16))) Smem sm;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ql = lane & 31, h = lane >> 5;
  const int kg = wave / kRows, rw = wave % kRows;
  const uint32_t heads = static_cast<uint32_t>(a.n_kv_heads), at = blockIdx.x / heads;
  const int g = static_cast<int>(blockIdx.x - at * heads);
  const PrefillPiece piece = a.pieces[at];
  if (piece.row0 < 0) return;
  const int t0 = piece.t0, t1 = piece.t1, b = piece.b;
  const PrefillSequence seq{piece.start, piece.n, piece.len};
  const int n_rows = seq.n * a.group;
  const PrefillTiles tiles = prefill_tiles(a, seq, piece.row0);
  const int n_sink = tiles.n_sink, skip = tiles.skip;
  // the row of the wave's first row, of this lane's, and of the wave's last that is there
  const int wave_row = piece.row0 + rw * kTile;
  const int row = wave_row + ql, rc = row < n_rows ? row : n_rows - 1;
  auto first = [&](int j) { return (j < n_sink ? j : j + skip) * kTile; };
  // is position p seen by some row of the block?
  auto counts = [&](int p) { return p < tiles.end && (p >= tiles.lo || p < a.n_sinks); };

  // ---- loads of a tile -------------------------------------------------------------
  struct Source {
    global_bytes_t keys, values;
    global_floats_t k_norms, v_norms;
  };
  Source cache{(global_bytes_t)a.k_codes, (global_bytes_t)a.v_codes, (global_floats_t)a.k_norms,
               (global_floats_t)a.v_norms};
  asm volatile("" : "+s"(cache.keys), "+s"(cache.values));
  asm volatile("" : "+s"(cache.k_norms), "+s"(cache.v_norms));
  const int32_t* const table = a.pages.tables + static_cast<int64_t>(b) * a.pages.max_pages;
  auto pool_record = [&](int p, int32_t entry) {
    const int64_t page =
        static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.pages.n_pages) ? entry : 0;
    return ((page * a.n_kv_heads + g) << a.pages.page_shift) +
           (p & ((1 << a.pages.page_shift) - 1));
  };
  // the last position that the block sees
  const int seen_last = tiles.end - 1;
  // the page entry of this lane's position of the next tile (a pair: of its first tile in
  // the lanes below 32, of its second above), read a tile (pair) ahead
  int32_t next_page = 0;
  auto load_pages = [&](int j) {
    const int jt = kPair == 2 && h && j + 1 < tiles.n ? j + 1 : j;
    const int p = first(jt) + ql;
    next_page = table[(p < seen_last ? p : seen_last) >> a.pages.page_shift];
  };
  Decode dec;
  dec.setup(kRows == 8 ? rw & 3 : rw, lane);
  const int own = kRows == 8 ? rw >> 2 : 0;   // which tile of a pair this wave decodes
  float raw_scale[kPair];
  bool live[kPair];   // raw_scale is that of a position that some row sees
  auto half_of = [&](int i) { return kRows == 1 ? i : rw & 1; };
  auto load_scale = [&](int j, int32_t entry, float& raw, bool& counted) {
    const int p0 = first(j);
    const int p = p0 + ql < seen_last ? p0 + ql : seen_last;
    // (this lane's: a key's scale in half 0, a value's in half 1)
    raw = (h ? cache.v_norms : cache.k_norms)[pool_record(p, entry)];
    counted = counts(p0 + ql);
  };
  auto load_records = [&](int j, int32_t entry) {
    const int p0 = first(j);
    const bool whole = p0 + kTile - 1 <= seen_last;
#pragma unroll
    for (int i = 0; i < Decode::kTasks; ++i) {
      // the half's first position, or the last one there is
      const int at = p0 + 16 * half_of(i), p = at < seen_last ? at : seen_last;
      const int64_t r = pool_record(p, __builtin_amdgcn_readlane(entry, 16 * half_of(i)));
      dec.load(i, cache.keys + r * kRB, cache.values + r * kRB, seen_last - p, whole);
    }
  };
  auto ahead = [&](int jt) { return jt < t1 ? jt : t1 - 1; };   // (past the end: the last tile)
  auto load = [&](int j) {
    if constexpr (kPair == 2) {
      const int j1 = ahead(j + 1);
      int32_t e0 = next_page, e1 = next_page;
      const auto both = __builtin_amdgcn_permlane32_swap(e0, e0, false, false);
      e0 = both[0];                       // the lower lanes' in both halves
      e1 = j1 == j ? e0 : both[1];        // the upper lanes'
      load_scale(j, e0, raw_scale[0], live[0]);
      load_scale(j1, e1, raw_scale[1], live[1]);
      load_records(own ? j1 : j, own ? e1 : e0);
    } else {
      load_scale(j, next_page, raw_scale[0], live[0]);
      load_records(j, next_page);
    }
  };

  int j = t0 + kg;
  if (j < t1) {
    load_pages(j);
    load(j);
    load_pages(ahead(j + (kRows >= 4 ? kPair : kGroups)));
  }
  // ---- the wave's rows ---------------------------------------------------------------
  TileRows w;
  float down;
  {
    const int64_t qrow =
        static_cast<int64_t>(g) * a.n_rows + static_cast<int64_t>(seq.start) * a.group + rc;
    const char* src = a.q_op + qrow * kQBytes + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      w.qh[s] = *reinterpret_cast<const u32x4_t*>(src + 32 * s);
      w.ql[s] = *reinterpret_cast<const u32x4_t*>(src + 256 + 32 * s);
    }
    down = a.q_down[qrow];
  }
  PrefillView mine;
  mine.end = seq.len - seq.n + row_token(a, rc) + 1;
  mine.lo = a.window > 0 ? mine.end - a.window : 0;
  mine.pad = 0;
  // a tile that the wave's first row sees to its end and its last from its start on is
  // seen by all of them
  const int all_end = __builtin_amdgcn_readfirstlane(mine.end);
  const int all_lo = __builtin_amdgcn_readlane(mine.lo, 31);
  // ---- the unit of the value scales: the exponent of the largest finite one that some
  // row sees in this piece ---------------------------------------------------------------
  float largest = 0.f;
  {
    constexpr int kAhead = 8, kStep = kThreadsHere / kTile;
    for (int jt = t0 + (tid >> 5); jt < t1; jt += kAhead * kStep) {
      float v[kAhead];
      int64_t r[kAhead];
      bool in[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int je = jt + u * kStep < t1 ? jt + u * kStep : t1 - 1;
        const int p = first(je) + ql;
        in[u] = counts(p);
        // (a position that does not count: the last one's scale is read instead)
        const int pc = in[u] ? p : seen_last;
        r[u] = pool_record(pc, table[pc >> a.pages.page_shift]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = a.v_norms[r[u]];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        largest = in[u] && fabsf(v[u]) < INFINITY ? fmaxf(largest, fabsf(v[u])) : largest;
    }
    largest = wave64_max(largest);
    if (lane == 0) sm.red[wave] = largest;
  }
  // ---- one exponent for the wave's rows where they lie within 2^15 of each other (the
  // smallest still has its bits down to 2^-24): exact but for those ----------------------
  const float down_max = wave64_max(down), down_min = -wave64_max(-down);
  w.even = down_min * 32768.0f >= down_max;
  if (w.even && down_min != down_max) {
    const _Float16 f = static_cast<_Float16>(down / down_max);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      w.qh[s] = __builtin_bit_cast(u32x4_t, __builtin_bit_cast(half8_t, w.qh[s]) * f);
      w.ql[s] = __builtin_bit_cast(u32x4_t, __builtin_bit_cast(half8_t, w.ql[s]) * f);
    }
  }
  const float down0 = w.even ? down_max : 1.0f;
  mine.down = down;
  // (in LDS: read where a tile is masked, and in the end)
  const PrefillView* const view = &sm.rows[wave].view[ql];
  if (h == 0) sm.rows[wave].view[ql] = mine;
  // (arrived before the loop: a wait for them inside it would be one for the next tile's
  // records as well)
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    asm volatile("" : "+v"(w.qh[s]));
    asm volatile("" : "+v"(w.ql[s]));
  }
  w.m = -INFINITY;
  w.l = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] = 0.f;
  build_pair_table(sm, cb, tid);
  lds_barrier();   // the pair table, red
#pragma unroll
  for (int i = 0; i < kWavesHere; ++i) largest = fmaxf(largest, sm.red[i]);
  uint32_t unit = __builtin_amdgcn_readfirstlane(
      static_cast<int>(__builtin_bit_cast(uint32_t, largest) & 0x7F800000u));
  unit = unit > kMinScaleBits ? unit : kMinScaleBits;
  // what this lane's scale is staged times
  const float factor =
      h ? __builtin_bit_cast(float, ((127u + 127u + kUnitBits) << 23) - unit) : down0;
  auto store = [&](char* k, char* v, float* sc) {
#pragma unroll
    for (int i = 0; i < kPair; ++i) sc[2 * kTile * i + lane] = live[i] ? raw_scale[i] * factor : 0.f;
#pragma unroll
    for (int i = 0; i < Decode::kTasks; ++i) dec.store(sm.lut, i, half_of(i), k, v);
  };
  // bits of the keys of tile j that this lane's row sees; false: all rows all
  auto see = [&](int jt, uint32_t& bits) {
    const int p0 = first(jt);
    bits = 0;
    if (p0 + kTile <= all_end && (p0 >= all_lo || p0 + kTile <= a.n_sinks)) return false;
    bits = low_bits(view->end - p0) & (~low_bits(view->lo - p0) | low_bits(a.n_sinks - p0));
    bits >>= 4 * h;
    return true;
  };

  if constexpr (kRows >= 4) {
    if (t0 < t1) {
      constexpr int kKeyStep = kPair * kKeyBytes;
      constexpr int kScaleStep = kPair * 2 * kTile;
      char* const kbuf = sm.t.k[0][0];
      char* vfree = sm.t.v[0][2 * kPair];
      char* vcur = sm.t.v[0][0];
      char* vnext = sm.t.v[0][kPair];
      char* vlast = vfree;   // the tile whose weights are ready
      float* const sc = sm.t.sc[wave][0];
      const int own_k = own * kKeyBytes, own_v = own * kValueBytes;
      // before the first tile: weights of nothing, times values of nothing
      for (int e = tid; e < kValueBytes / 16; e += kThreadsHere)
        reinterpret_cast<u32x4_t*>(vlast)[e] = u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < 2; ++s) w.ph[s] = w.pl[s] = u32x4_t{0, 0, 0, 0};
      store(kbuf + own_k, vcur + own_v, sc);
      load(ahead(j + kPair));
      load_pages(ahead(j + 2 * kPair));
      lds_barrier();
      // scores x of tile jt to weights, those of the tile before to outputs
      auto finish = [&](f32x16_t& x, int jt, const float* scales) {
        uint32_t bits = 0;
        const bool masked = jt >= t1 || see(jt, bits);
        float top;
        if (tile_relative(w, x, scales, &view->down, h, masked, bits, top)) {
          tile_values<kLo>(w, vlast, ql, h);
#pragma unroll
          for (int s = 0; s < 2; ++s) w.ph[s] = w.pl[s] = u32x4_t{0, 0, 0, 0};
          tile_raise(w, x, top);
        }
        tile_values<kLo>(w, vlast, ql, h);
        tile_weights<kLo, true>(w, x, scales + kTile, h);
      };
      // (a wave without rows only decodes)
      if (wave_row >= n_rows) {
        for (int it = 0; j < t1; ++it, j += kPair) {
          const int next = (it & 1) ^ 1;
          store(kbuf + next * kKeyStep + own_k, vnext + own_v, sc + next * kScaleStep);
          load(ahead(j + 2 * kPair));
          load_pages(ahead(j + 3 * kPair));
          char* const was = vcur;
          vcur = vnext;
          vnext = vfree;
          vfree = was;
          lds_barrier();
        }
      }
      for (int it = 0; j < t1; ++it, j += kPair) {
        const int cur = it & 1;
        const char* const k = kbuf + cur * kKeyStep;
        const float* const scales = sc + cur * kScaleStep;
        // (past the end: the last tile once more, into buffers that are free)
        f32x16_t x = tile_scores(w, k, ql, h);
        store(kbuf + (cur ^ 1) * kKeyStep + own_k, vnext + own_v, sc + (cur ^ 1) * kScaleStep);
        load(ahead(j + 2 * kPair));
        load_pages(ahead(j + 3 * kPair));
        finish(x, j, scales);
        vlast = vcur;
        if constexpr (kPair == 2) {
          x = tile_scores(w, k + kKeyBytes, ql, h);
          finish(x, j + 1, scales + 2 * kTile);
          vlast = vcur + kValueBytes;
        }
        char* const was = vcur;
        vcur = vnext;
        vnext = vfree;
        vfree = was;
        lds_barrier();
      }
      tile_values<kLo>(w, vlast, ql, h);
    }
  } else {
    const int n_iter = (t1 - t0 + kGroups - 1) / kGroups;
    for (int it = 0; it < n_iter; ++it, j += kGroups) {
      const int cur = it % kKeyBufs;
      char* const k = sm.t.k[kg][cur];
      char* const v = sm.t.v[kg][cur];
      float* const sc = sm.t.sc[wave][cur];
      if (j < t1) store(k, v, sc);
      if (j + kGroups < t1) {
        load(j + kGroups);
        load_pages(ahead(j + 2 * kGroups));
      }
      if constexpr (kRows == 1)
        wave_lds_fence();
      else
        lds_barrier();
      if (j < t1) {
        uint32_t bits;
        const bool masked = see(j, bits);
        f32x16_t x = tile_scores(w, k, ql, h);
        float top;
        if (tile_relative(w, x, sc, &view->down, h, masked, bits, top)) tile_raise(w, x, top);
        tile_weights<kLo, true>(w, x, sc + kTile, h);
        tile_values<kLo>(w, v, ql, h);
      }
      if constexpr (kRows == 1) wave_lds_fence();   // the next tile behind this one's reads
    }
  }

  // ---- the groups' results joined, by row ----------------------------------------------
  lds_barrier();   // every wave is done with the tiles
  const f32x2_t ls = half_pair(w.l);
  wave_lds_fence();   // every lane has read its row's view
  if (h == 0) {
    sm.rows[wave].ml[ql][0] = w.m;
    sm.rows[wave].ml[ql][1] = ls[0] + ls[1];
  }
  const float oscale = __builtin_bit_cast(float, unit) * (1.0f / (1 << kUnitBits));
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<f32x4_t*>(&sm.o[wave][ql][32 * d + 8 * c + 4 * h]) =
          f32x4_t{w.o[d][4 * c], w.o[d][4 * c + 1], w.o[d][4 * c + 2], w.o[d][4 * c + 3]} * oscale;
  lds_barrier();
  const int blk = tid & 31;
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t qleft = par[0], qright = par[1];
  for (int r = tid >> 5; r < kRows * kTile; r += kThreadsHere / 32) {
    if (piece.row0 + r >= n_rows) break;   // (the row's 32 lanes alike)
    float M = -INFINITY, L = 0.f;
    f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGroups; ++k) M = fmaxf(M, sm.rows[k * kRows + r / kTile].ml[r % kTile][0]);
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const int wv = k * kRows + r / kTile;
      const float m = sm.rows[wv].ml[r % kTile][0];
      // (without a maximum: nothing seen, a sum of 0, or only NaN scores)
      const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      L += c * sm.rows[wv].ml[r % kTile][1];
      if (m != -INFINITY)
        O += c * *reinterpret_cast<const f32x4_t*>(&sm.o[wv][r % kTile][4 * blk]);
    }
    if (piece.part < 0) {
      // (a row that sees nothing is zero; a sum that is NaN stays visible)
      const f32x4_t x = rotate_inverse(O * (L == 0.f ? 0.f : 1.0f / L), qleft, qright, blk);
      const int i = row_token(a, piece.row0 + r), hh = piece.row0 + r - i * a.group;
      store4(static_cast<T*>(a.out) + (seq.start + static_cast<int64_t>(i)) * a.out_stride +
                 (static_cast<int64_t>(g) * a.group + hh) * kDim + 4 * blk,
             x);
    } else {
      const int64_t at =
          (static_cast<int64_t>(piece.part) * a.n_kv_heads + g) * a.block_rows + r;
      if (blk == 0) *reinterpret_cast<f32x2_t*>(&a.part_ml[2 * at]) = f32x2_t{M, L};
      *reinterpret_cast<f32x4_t*>(&a.part_o[kDim * at + 4 * blk]) = O;
    }
  }
}

// ---- blocks of 256 rows of fp16 queries ------------------------------------------------
// Eight waves of 32 rows, two on each SIMD (four of 64 rows, one on each, took 2.0 times as
// long).  2048 tokens of 32 query and 4 KV heads at the end of 32768 take 1.31 to 1.40 ms (by the
// card's clock), 760 to 814 TFLOP/s of products counted once; 4096 tokens by themselves 226 to
// 242 us.  The matrix cores are busy for 44 % of the cycles, vector instructions for 52 %: what a
// wave does besides the products bounds it (where it took 1.32 ms, decoding took 0.28, the 6-bit
// products 0.15, exponentials 0.10, as the kernel without them shows), so that is kept small: 128
// records are decoded at a time, 16 by a wave; weights are exp2 of their scores with no search
// for a maximum, times the value scales, rounded once; scales are staged once for all waves.
//
// A turn of 128 records has four steps, a tile each: scores, weights, outputs.  A step's value
// operands come from LDS while its weights are made, the next step's key operands while its
// outputs are.  The next turn's keys are decoded in step 0, its values in step 2, with a
// barrier behind step 1 and one behind step 3; two buffers of each do.
constexpr int kWideWaves = 8, kWideThreads = 64 * kWideWaves;
constexpr int kTurn = 4;                      // tiles of a turn
// Weights are 2^kLift at the reference, which is raised only when a lane's share of a tile's
// sum passes 2^15 (times a value scale, below 1 in its units, they are in fp16's range then): a
// wave that raises its rows keeps the others waiting.  (Raised from 2^4 above the reference on: 233
// instead of 218 us for 4096 tokens, then.  2^2, 2^4, 2^6 and 2^8 at the reference: 241, 237,
// 240 and 247 us; a batch of chunks and single tokens 224, 230, 229 and 234.)  Times the value
// scale, weights below 2^-14 lose bits, at 2^-25 the last: 2^-29 of the largest each.
constexpr float kLift = 4.0f;

typedef TileDecode<2, 3> WideDecode;          // 16 records by a wave

// (called from several places: otherwise functions of their own, their state in memory)
#define IQ_INLINE __attribute__((always_inline))

// A place that is the same in every lane, kept in scalar registers.
__device__ __forceinline__ global_bytes_t scalar_place(global_bytes_t p) {
  const uint64_t x = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return (global_bytes_t)(static_cast<uint64_t>(hi) << 32 | lo);
}

// What fp16 leaves of a query (lo parts) counts by 1 / 8 of it or so: 32 values of 6 bits
// (sign, 2 of exponent, 3 of mantissa) to six registers, products of 64 of them in the time
// of 16 of fp16.
typedef _Float16 half32_t __attribute__((ext_vector_type(32)));
typedef uint32_t u32x6_t __attribute__((ext_vector_type(6)));
typedef int32_t i32x8_t __attribute__((ext_vector_type(8)));

// 32 values divided by `scale` (a power of two), in 6 bits.
__device__ __forceinline__ i32x8_t six_bits(const u32x4_t* f, float scale) {
  struct Four {
    u32x4_t v[4];
  };
  const u32x6_t x = __builtin_amdgcn_cvt_scalef32_pk32_fp6_f16(
      __builtin_bit_cast(half32_t, Four{{f[0], f[1], f[2], f[3]}}), scale);
  return i32x8_t{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]),
                 static_cast<int>(x[3]), static_cast<int>(x[4]), static_cast<int>(x[5]), 0, 0};
}
__device__ __forceinline__ f32x16_t mfma_six(i32x8_t a, i32x8_t b, f32x16_t c) {
  // (formats 2: 6 bits of which 2 exponent; the operands' scales 2^-5 and 1, by their exponents)
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 2, 2, 0, 127 - 5, 0, 127);
}

// A wave's 32 rows: operands, outputs, the weights of a tile.
struct WideRows {
  u32x4_t q[8];
  i32x8_t rest[2];
  f32x16_t o[4];
  u32x4_t p[2];
  float m, l;          // reference, less kLift (log2 units); this lane's share of the sum
  float ref;           // m, 0 before there is one
  int32_t end, lo;     // what the row sees
};

__global__ __launch_bounds__(kWideThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void prefill_wide_kernel(PrefillArgs a, Codebook cb) {
  constexpr int kRB = kRecordBytes;
  struct Smem {
    uint32_t lut[64];
    float red[kWideWaves];
    float ks[2][kTurn * kTile], vs[2][kTurn * kTile];   // scales of keys and of values
    f32x2_t ml[kTurn][kTile];   // few rows: the waves' references and sums
    f32x4_t rot[4 * kNumBlocks];
    union {
      struct {
        char k[2][kTurn][kKeyBytes];
        char v[2][kTurn][kValueBytes];
      } t;
      float o[kWideWaves][kTile][kORow];
    };
  };
  __shared__ __attribute__((aligned(16))) Smem sm;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ql = lane & 31, h = lane >> 5;
  const uint32_t heads = static_cast<uint32_t>(a.n_kv_heads), at = blockIdx.x / heads;
  const int g = static_cast<int>(blockIdx.x - at * heads);
  const PrefillPiece piece = a.pieces[at];
  if (piece.row0 < 0) return;
  const int t0 = piece.t0, t1 = piece.t1, b = piece.b;
  const PrefillSequence seq{piece.start, piece.n, piece.len};
  const int n_rows = seq.n * a.group;
  const PrefillTiles tiles = prefill_tiles(a, seq, piece.row0);
  const int n_sink = tiles.n_sink, skip = tiles.skip;
  // a block of at most 32 rows: four waves take one tile of a turn each
  const bool few = n_rows - piece.row0 <= kTile;
  const int wave_row = few ? (wave < kTurn ? piece.row0 : n_rows) : piece.row0 + wave * kTile;
  auto first = [&](int j) { return (j < n_sink ? j : j + skip) * kTile; };
  // (no branches: each would end the stretch of code that products are spread over)
  auto counts = [&](int p) {
    return static_cast<bool>((p < tiles.end) & ((p >= tiles.lo) | (p < a.n_sinks)));
  };

  // ---- loads of a turn: this wave's 16 records, half `half` of tile `own` ------
  const global_bytes_t keys = (global_bytes_t)a.k_codes, values = (global_bytes_t)a.v_codes;
  const global_floats_t k_norms = (global_floats_t)a.k_norms, v_norms = (global_floats_t)a.v_norms;
  const int32_t* const table = a.pages.tables + static_cast<int64_t>(b) * a.pages.max_pages;
  const int seen_last = tiles.end - 1;   // the last position that the block sees
  const int own = wave >> 1, half = wave & 1;
  WideDecode dec;
  dec.setup(0, lane);
  auto ahead = [&](int jt) { return jt < t1 ? jt : t1 - 1; };   // (past the end: the last tile)
  auto position = [&](int j) { return first(ahead(j + own)) + 16 * half; };
  auto clamped = [&](int p) { return p < seen_last ? p : seen_last; };
  int32_t next_page = 0;   // of the records that are loaded next, read a turn ahead
  auto load_page = [&](int j) { next_page = table[clamped(position(j)) >> a.pages.page_shift]; };
  float raw_ks = 0.f, raw_vs = 0.f;
  int pos = 0;   // where the loaded records begin
  // (16 positions are in one page; those behind the last that is seen are read as well, and
  // count for nothing.  The arrays' places go through scalar registers, with the lane's
  // offsets beside them: a few instructions for a turn, and no others to multiply with.)
  const uint32_t koff = dec.koff, soff = 4 * (lane & 15);
  auto load_keys = [&](int j) IQ_INLINE -> int64_t {
    pos = position(j);
    const int32_t entry = __builtin_amdgcn_readfirstlane(next_page);
    const int64_t page =
        static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.pages.n_pages) ? entry : 0;
    const int at16 = clamped(pos) & ((1 << a.pages.page_shift) - 1) & ~15;
    const int64_t record = ((page * a.n_kv_heads + g) << a.pages.page_shift) +
                           __builtin_amdgcn_readfirstlane(at16);
    const global_bytes_t kp = scalar_place(keys + record * kRB);
    const global_bytes_t ks = scalar_place((global_bytes_t)(k_norms + record));
    const global_bytes_t vs = scalar_place((global_bytes_t)(v_norms + record));
#pragma unroll
    for (int e = 0; e < 3; ++e)
      dec.raw_k[0][e] = *(const IQ_GLOBAL uint32_t*)(kp + koff + 4 * e);
    raw_ks = *(const IQ_GLOBAL float*)(ks + soff);
    raw_vs = *(const IQ_GLOBAL float*)(vs + soff);
    return record;
  };
  auto load_values = [&](int64_t record) IQ_INLINE {
    const global_bytes_t vp = scalar_place(values + record * kRB);
#pragma unroll
    for (int e = 0; e < 4; ++e) dec.raw_v[0][e] = *(const IQ_GLOBAL u32_a1_t*)(vp + dec.voff + e * kRB);
  };
  if (t0 < t1) {
    load_page(t0);
    load_values(load_keys(t0));
    load_page(t0 + kTurn);
  }
  // ---- the wave's rows ---------------------------------------------------------------------
  WideRows w;
  u32x4_t rest[8];
  float down;
  {
    const int row = wave_row + ql, rc = row < n_rows ? row : n_rows - 1;
    const int64_t qrow =
        static_cast<int64_t>(g) * a.n_rows + static_cast<int64_t>(seq.start) * a.group + rc;
    const char* src = a.q_op + qrow * kQBytes + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      w.q[s] = *reinterpret_cast<const u32x4_t*>(src + 32 * s);
      rest[s] = *reinterpret_cast<const u32x4_t*>(src + 256 + 32 * s);
    }
    down = a.q_down[qrow];
    w.end = seq.len - seq.n + row_token(a, rc) + 1;
    w.lo = a.window > 0 ? w.end - a.window : 0;
    w.m = -INFINITY;
    w.l = w.ref = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[d][i] = 0.f;
#pragma unroll
    for (int s = 0; s < 2; ++s) w.p[s] = u32x4_t{0, 0, 0, 0};
  }
  // a tile that the wave's first row sees to its end and its last from its start on is
  // seen by all of them
  const int all_end = __builtin_amdgcn_readfirstlane(w.end);
  const int all_lo = __builtin_amdgcn_readlane(w.lo, 31);
  // ---- the unit of the value scales: the exponent of the largest finite one that the
  // sequence's tokens see ---------------------------------------------------------------------
  float largest = 0.f;
  const float* const units = a.units + (static_cast<int64_t>(b) * a.n_kv_heads + g) * a.unit_chunks;
  for (int i = lane; i < a.unit_chunks; i += 64) largest = fmaxf(largest, units[i]);
  largest = wave64_max(largest);
  const float top = wave64_max(down);
  if (lane == 0) sm.red[wave] = top;
  build_pair_table(sm, cb, tid);
  // the head's blocks M_i H_4, for the outputs
  if (tid < kNumBlocks) {
    float m[4][4];
    so4_matrix_h4(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * tid, m);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      sm.rot[4 * tid + r] = f32x4_t{m[r][0], m[r][1], m[r][2], m[r][3]} * kInvSqrtDim;
  }
  lds_barrier();   // the pair table, red, rot
  float down_max = 0.f;
#pragma unroll
  for (int i = 0; i < kWideWaves; ++i) {
    down_max = fmaxf(down_max, sm.red[i]);
  }
  down_max = fmaxf(down_max, 0x1p-120f);   // (rows of zeros)
  down_max = __builtin_bit_cast(
      float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, down_max)));
  // One exponent for the block's rows, exact powers of two.  (A row far smaller than the
  // largest loses bits below 2^-24 of the unit: rows of fp16 are at most 2^17 by entry, so
  // the scores of ordinary ones, about 1, move by less than 2^-13 beside the largest that
  // there can be.)
  {
    const _Float16 f = static_cast<_Float16>(down / down_max);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      w.q[s] = __builtin_bit_cast(u32x4_t, __builtin_bit_cast(half8_t, w.q[s]) * f);
      rest[s] = __builtin_bit_cast(u32x4_t, __builtin_bit_cast(half8_t, rest[s]) * f);
    }
    // (rests are at most 4)
    w.rest[0] = six_bits(rest, 1.0f);
    w.rest[1] = six_bits(rest + 4, 1.0f);
  }
  uint32_t unit = __builtin_amdgcn_readfirstlane(
      static_cast<int>(__builtin_bit_cast(uint32_t, largest) & 0x7F800000u));
  unit = unit > kMinScaleBits ? unit : kMinScaleBits;
  // (2^125 at most: of larger ones neither 1 / 2 unit nor 2 unit is a normal number.  Scales are up
  // to 4 times 2 unit then; a row whose weight for one of them, times it, fp16 cannot hold has an
  // output beyond fp16.)
  constexpr uint32_t kMaxUnitBits = (127u + 125u) << 23;
  unit = unit < kMaxUnitBits ? unit : kMaxUnitBits;
  const float v_factor = __builtin_bit_cast(float, ((127u + 126u) << 23) - unit);   // 1 / 2 unit

  // ---- decoding ----------------------------------------------------------------------------------
  // (A value scale that is not finite: 0, so that rows that do not see the key stay as they
  // are, and its key's scale is NaN for those that do.)
  // all: every position of the turn counts.
  auto store_keys = [&](bool all, char* k, float* sc, float* sv) IQ_INLINE {
    uint32_t x[3];
#pragma unroll
    for (int e = 0; e < 3; ++e) x[e] = dec.raw_k[0][e];
    u32x4_t p[4];
    key_pairs<3>(sm.lut, x, p);
    char* kd = k + (dec.key + 16 * half) * kKeyStride + 64 * dec.chunk;
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<u32x4_t*>(kd + 16 * e) = p[e];
    float ks = fabsf(raw_vs) < INFINITY ? raw_ks * down_max : NAN;
    float vs = fabsf(raw_vs) < INFINITY ? raw_vs * v_factor : 0.f;
    if (!all) {
      const bool in = counts(pos + (lane & 15));
      ks = in ? ks : 0.f;
      vs = in ? vs : 0.f;
    }
    sc[kTile * own + 16 * half + (lane & 15)] = ks;
    sv[kTile * own + 16 * half + (lane & 15)] = vs;
  };
  // Values lie in LDS by dimension, dim 8 v + m in row 16 m + 2 (v % 8) + v / 8: rows of 80
  // bytes are read 32 in a row without bank conflicts, and a wave's write of dim m of 16 v's
  // and 4 quads of records meets no other in its bank either (the 8 dims of a lane in
  // consecutive rows: writes 4 times as long).
  const int value_row = 2 * (dec.vdim & 7) + (dec.vdim >> 3);
  auto store_values = [&](char* v) IQ_INLINE {
    u32x4_t q[4];
    window_pairs<3>(sm.lut, dec.raw_v[0], dec.vshift, q);
    // a dim's 4 records are 8 bytes, in the order of the weights; dim m of the 8 in row
    // 16 m + value_row
    char* vd = v + value_row * kValStride + 16 * (2 * half + (dec.quad & 1)) + 8 * (dec.quad >> 1);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      *reinterpret_cast<uint2*>(vd + 32 * n * kValStride) =
          uint2{__builtin_amdgcn_perm(q[n][1], q[n][0], 0x05040100u),
                __builtin_amdgcn_perm(q[n][3], q[n][2], 0x05040100u)};
      *reinterpret_cast<uint2*>(vd + (32 * n + 16) * kValStride) =
          uint2{__builtin_amdgcn_perm(q[n][1], q[n][0], 0x07060302u),
                __builtin_amdgcn_perm(q[n][3], q[n][2], 0x07060302u)};
    }
  };

  // ---- a tile's products and weights ------------------------------------------------------------
  // Operands from LDS, loaded while the products before theirs are under way.
  u32x4_t kf[8], vf[8];
  auto load_key_operands = [&](const char* k) IQ_INLINE {
    const char* kp = k + ql * kKeyStride + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) kf[s] = *reinterpret_cast<const u32x4_t*>(kp + 32 * s);
  };
  auto load_value_operands = [&](const char* v) IQ_INLINE {
    const char* vp = v + ql * kValStride + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s)
      vf[s] = *reinterpret_cast<const u32x4_t*>(vp + 32 * (s >> 1) * kValStride + 32 * (s & 1));
  };
  auto scores = [&]() IQ_INLINE {
    f32x16_t x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) x = mfma32(kf[s], w.q[s], x);
    // (levels are at most 6.03 times 2^-5)
    x = mfma_six(six_bits(kf, 0.03125f), w.rest[0], x);
    x = mfma_six(six_bits(kf + 4, 0.03125f), w.rest[1], x);
    return x;
  };
  auto outputs = [&]() IQ_INLINE {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      w.o[d] = mfma32(vf[2 * d], w.p[0], w.o[d]);
      w.o[d] = mfma32(vf[2 * d + 1], w.p[1], w.o[d]);
    }
  };
  // Scores x of tile jt against the reference.  all: the wave's rows see all of the tile.
  auto relative = [&](bool all, f32x16_t& x, const float* sc, int jt) IQ_INLINE {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&sc[8 * e + 4 * h]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * e + i] = __builtin_fmaf(x[4 * e + i], ks[i], -w.ref);
    }
    if (!all) {
      const int p0 = first(ahead(jt));
      uint32_t see =
          low_bits(w.end - p0) & (~low_bits(w.lo - p0) | low_bits(a.n_sinks - p0));
      see = jt < t1 ? see >> (4 * h) : 0u;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[i] = see >> (8 * (i / 4) + i % 4) & 1 ? x[i] : -INFINITY;
    }
  };
  // The reference raised to the tile's largest score, where that is above it.
  bool open = true;   // some row has none yet
  auto raise = [&](f32x16_t& x) IQ_INLINE {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
    const f32x2_t tops = half_pair(top);
    top = fmaxf(tops[0], tops[1]);
    const float m = fmaxf(w.m, w.ref + top - kLift);
    const float f = w.m == m ? 1.0f : (w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.m - m));
    const float ref = m == -INFINITY ? 0.f : m, by = ref - w.ref;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] -= by;
    w.l *= f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[d][i] *= f;
    w.m = m;
    w.ref = ref;
    open = __any(m == -INFINITY);
  };
  // The weights of relative scores, times the value scales sv; this lane's sum of them.
  auto weights = [&](const f32x16_t& x, const float* sv) IQ_INLINE {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&sv[8 * e + 4 * h]);
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const float p0 = __builtin_amdgcn_exp2f(x[4 * e + i]), p1 = __builtin_amdgcn_exp2f(x[4 * e + i + 1]);
        sum += p0;
        sum += p1;
        // (a mixed-precision multiply-add rounds its result and places it)
        w.p[e >> 1][2 * (e & 1) + (i >> 1)] = __builtin_bit_cast(
            uint32_t, half2_t{static_cast<_Float16>(__builtin_fmaf(p0, vs[i], 0.f)),
                              static_cast<_Float16>(__builtin_fmaf(p1, vs[i + 1], 0.f))});
      }
    }
    return sum;
  };
  // A step: tile jt, whose keys are loaded; its values at v, the next tile's keys at k.
  // decode: what is decoded meanwhile.
  auto step = [&](bool all, const float* sc, const float* sv, int jt, const char* v, const char* k,
                  auto decode) IQ_INLINE {
    f32x16_t x = scores();
    decode();
    relative(all, x, sc, jt);
    if (open) raise(x);
    load_value_operands(v);
    float sum = weights(x, sv);
    // Above 2^15 fp16 may not hold a weight: then, seldom, the reference is raised and the
    // weights are made again.  (Rows of NaN: once.)
    if (__any(!(sum < 32768.0f) & (w.l < INFINITY))) {
      raise(x);
      sum = weights(x, sv);
    }
    w.l += sum;
    load_key_operands(k);
    outputs();
  };
  // Tiles j .. j + 3 are all there, next to each other, before end, and within the window (from
  // lo on) or the sinks.  (There may be more sinks than positions before end.)
  auto whole = [&](int j, int lo, int end) {
    const int p = first(j);
    return j + kTurn <= t1 && (skip == 0 || j >= n_sink || j + kTurn <= n_sink) &&
           p + kTurn * kTile <= end && (p >= lo || p + kTurn * kTile <= a.n_sinks);
  };

  if (t0 < t1) {
    store_keys(false, sm.t.k[0][own], sm.ks[0], sm.vs[0]);
    store_values(sm.t.v[0][own]);
    load_values(load_keys(t0 + kTurn));
    load_page(t0 + 2 * kTurn);
    lds_barrier();
    int cur = 0;   // buffers of the present turn
    if (wave_row >= n_rows) {
      // (a wave without rows only decodes)
      for (int j = t0; j < t1; j += kTurn, cur ^= 1) {
        store_keys(false, sm.t.k[cur ^ 1][own], sm.ks[cur ^ 1], sm.vs[cur ^ 1]);
        lds_barrier();
        store_values(sm.t.v[cur ^ 1][own]);
        load_values(load_keys(j + 2 * kTurn));
        load_page(j + 3 * kTurn);
        lds_barrier();
      }
    } else if (few) {
      for (int j = t0; j < t1; j += kTurn, cur ^= 1) {
        const bool all = whole(j, all_lo, all_end);
        const bool next = whole(j + kTurn, tiles.lo, tiles.end);
        const char* const k = sm.t.k[cur][wave];
        load_key_operands(k);
        step(all, sm.ks[cur] + kTile * wave, sm.vs[cur] + kTile * wave, j + wave, sm.t.v[cur][wave], k,
             [&]() IQ_INLINE { store_keys(next, sm.t.k[cur ^ 1][own], sm.ks[cur ^ 1], sm.vs[cur ^ 1]); });
        lds_barrier();
        store_values(sm.t.v[cur ^ 1][own]);
        load_values(load_keys(j + 2 * kTurn));
        load_page(j + 3 * kTurn);
        lds_barrier();
      }
    } else {
      load_key_operands(sm.t.k[0][0]);
      for (int j = t0; j < t1; j += kTurn, cur ^= 1) {
        const char(*k)[kKeyBytes] = sm.t.k[cur];
        const char(*v)[kValueBytes] = sm.t.v[cur];
        const float *const sc = sm.ks[cur], *const sv = sm.vs[cur];
        // no masks in this turn; every record of the next one counts
        const bool all = whole(j, all_lo, all_end);
        const bool next = whole(j + kTurn, tiles.lo, tiles.end);
        step(all, sc, sv, j, v[0], k[1],
             [&]() IQ_INLINE { store_keys(next, sm.t.k[cur ^ 1][own], sm.ks[cur ^ 1], sm.vs[cur ^ 1]); });
        step(all, sc + kTile, sv + kTile, j + 1, v[1], k[2], [&]() IQ_INLINE {});
        lds_barrier();
        step(all, sc + 2 * kTile, sv + 2 * kTile, j + 2, v[2], k[3], [&]() IQ_INLINE {
          store_values(sm.t.v[cur ^ 1][own]);
          load_values(load_keys(j + 2 * kTurn));
          load_page(j + 3 * kTurn);
        });
        step(all, sc + 3 * kTile, sv + 3 * kTile, j + 3, v[3], sm.t.k[cur ^ 1][0], [&]() IQ_INLINE {});
        lds_barrier();
      }
    }
  }

  // ---- the wave's results ------------------------------------------------------------------
  // 16 rows at a time, each by four lanes of 32 dims (8 blocks): R^T o = H_128 M^T o /
  // sqrt(128) = (H_32 (x) I_4)(M H_4)^T o / sqrt(128), the blocks and three of the five
  // butterflies in the lane, the others between the four.
  lds_barrier();   // every wave is done with the tiles
  // (the lane's row and half from the thread's number again, not kept over the tiles)
  int again = tid;
  asm volatile("" : "+v"(again));
  const int row_at = again & 31, half_at = again >> 5 & 1;
  const float oscale = 2.0f * __builtin_bit_cast(float, unit);
  const f32x2_t ls = half_pair(w.l);
  float m = w.m, l = ls[0] + ls[1], joined = 1.0f;
  if (few) {
    if (wave < kTurn && half_at == 0) sm.ml[wave][row_at] = f32x2_t{m, l};
    lds_barrier();
    float all_l = 0.f, most = -INFINITY;
#pragma unroll
    for (int i = 0; i < kTurn; ++i) most = fmaxf(most, sm.ml[i][row_at][0]);
#pragma unroll
    for (int i = 0; i < kTurn; ++i) {
      const f32x2_t other = sm.ml[i][row_at];
      // (without a maximum: nothing seen, a sum of 0, or only NaN scores)
      const float c = other[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(other[0] - most);
      all_l += c * other[1];
    }
    joined = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - most);
    m = most;
    l = all_l;
  }
  // (a row that sees nothing is zero; a sum that is NaN stays visible)
  const float scale = joined * (piece.part >= 0 ? oscale : oscale * (l == 0.f ? 0.f : 1.0f / l));
  if (wave_row < n_rows) {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4_t*>(&sm.o[wave][row_at][32 * d + 8 * e + 4 * half_at]) =
            f32x4_t{w.o[d][4 * e], w.o[d][4 * e + 1], w.o[d][4 * e + 2], w.o[d][4 * e + 3]} * scale;
    if (piece.part >= 0 && half_at == 0 && wave_row + row_at < n_rows && !(few && wave))
      *reinterpret_cast<f32x2_t*>(
          &a.part_ml[2 * ((static_cast<int64_t>(piece.part) * a.n_kv_heads + g) * a.block_rows +
                          (wave_row + row_at - piece.row0))]) = f32x2_t{m, l};
  }
  if (few)
    lds_barrier();
  else
    wave_lds_fence();
  // (of few rows, two waves join 16 each)
  if (few ? wave > 1 : wave_row >= n_rows) return;
  const int quarter = again & 3;
#pragma unroll 1
  for (int i = few ? 16 * wave : 0; i < (few ? 16 * wave + 16 : kTile); i += 16) {
    const int r = i + (again >> 2 & 15), row = (few ? piece.row0 : wave_row) + r;
    // dims 32 quarter + 4 b + e, in the values' order
    float x[32];
#pragma unroll
    for (int d = 0; d < 32; ++d)
      x[d] = sm.o[few ? 0 : wave][r]
                 [16 * (d & 7) + 8 * (quarter & 1) + 2 * (d >> 3) + (quarter >> 1)];
    if (few) {
#pragma unroll 1
      for (int k = 1; k < kTurn; ++k)
#pragma unroll
        for (int d = 0; d < 32; ++d)
          x[d] += sm.o[k][r][16 * (d & 7) + 8 * (quarter & 1) + 2 * (d >> 3) + (quarter >> 1)];
    }
    if (piece.part >= 0) {
      if (row < n_rows) {
        const int64_t to = (static_cast<int64_t>(piece.part) * a.n_kv_heads + g) * a.block_rows +
                           (row - piece.row0);
        f32x4_t* dst = reinterpret_cast<f32x4_t*>(&a.part_o[kDim * to + 32 * quarter]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dst[e] = f32x4_t{x[4 * e], x[4 * e + 1], x[4 * e + 2], x[4 * e + 3]};
      }
      continue;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f32x4_t z = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x4_t m = sm.rot[4 * (8 * quarter + e) + k];
#pragma unroll
        for (int c = 0; c < 4; ++c) z[c] = __builtin_fmaf(m[c], x[4 * e + k], z[c]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) x[4 * e + c] = z[c];
    }
#pragma unroll
    for (int st = 4; st < 32; st <<= 1)
#pragma unroll
      for (int d = 0; d < 32; ++d)
        if (!(d & st)) {
          const float p = x[d], q = x[d + st];
          x[d] = p + q;
          x[d + st] = p - q;
        }
    const float s0 = quarter & 1 ? -1.0f : 1.0f, s1 = quarter & 2 ? -1.0f : 1.0f;
#pragma unroll
    for (int d = 0; d < 32; ++d) x[d] = __builtin_fmaf(s0, x[d], xor_lane<1>(x[d]));
#pragma unroll
    for (int d = 0; d < 32; ++d) x[d] = __builtin_fmaf(s1, x[d], xor_lane<2>(x[d]));
    if (row < n_rows) {
      const int t = row_token(a, row), hh = row - t * a.group;
      u32x4_t* dst = reinterpret_cast<u32x4_t*>(
          static_cast<_Float16*>(a.out) + (seq.start + static_cast<int64_t>(t)) * a.out_stride +
          (static_cast<int64_t>(g) * a.group + hh) * kDim + 32 * quarter);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u32x4_t y;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          y[c] = __builtin_bit_cast(uint32_t,
                                    half2_t{static_cast<_Float16>(x[8 * e + 2 * c]),
                                            static_cast<_Float16>(x[8 * e + 2 * c + 1])});
        dst[e] = y;
      }
    }
  }
}

// ---- merge of the parts, inverse rotation ------------------------------------------------
// A row's 128 dims are 32 threads'.  The workgroups, as many as the chip holds at once, take
// 8 rows of a KV head of a split at a time: most calls cut few blocks or none.
template <typename T>
__global__ __launch_bounds__(kPrepThreads) void prefill_merge_kernel(PrefillArgs a) {
  constexpr int kUnroll = 8;
  const int blk = threadIdx.x & 31;
  const uint32_t per_head = a.block_rows / kPrepRows, heads = a.n_kv_heads;
  const uint32_t tasks = static_cast<uint32_t>(a.n_splits[0]) * heads * per_head;
  for (uint32_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const uint32_t rest = task / per_head, at_split = rest / heads;
    const int g = static_cast<int>(rest - at_split * heads);
    const int r = static_cast<int>(task - rest * per_head) * kPrepRows +
                  (static_cast<int>(threadIdx.x) >> 5);
    const PrefillSplit split = a.splits[at_split];
    const PrefillSequence seq = prefill_sequence(a, split.b);
    if (split.row0 + r >= seq.n * a.group) continue;   // (the row's 32 lanes alike)
    const f32x4_t* par =
        reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
    const f32x4_t qleft = par[0], qright = par[1];
    float M = -INFINITY, L = 0.f;
    f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int p1 = split.part0 + split.parts;
    for (int s0 = split.part0; s0 < p1; s0 += kUnroll) {
      f32x2_t ml[kUnroll];
      f32x4_t o[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int s = s0 + u < p1 ? s0 + u : s0;
        const int64_t at = (static_cast<int64_t>(s) * a.n_kv_heads + g) * a.block_rows + r;
        ml[u] = *reinterpret_cast<const f32x2_t*>(&a.part_ml[2 * at]);
        o[u] = *reinterpret_cast<const f32x4_t*>(&a.part_o[kDim * at + 4 * blk]);
        if (s0 + u >= p1) ml[u] = f32x2_t{-INFINITY, 0.f};
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
        // (a part without anything seen has no outputs: select)
        const bool live = ml[u][0] != -INFINITY;
        const float c = live ? __builtin_amdgcn_exp2f(ml[u][0] - M) : 0.f;
        L += c * ml[u][1];
#pragma unroll
        for (int e = 0; e < 4; ++e) O[e] += live ? c * o[u][e] : 0.f;
      }
    }
    const f32x4_t x = rotate_inverse(O * (L == 0.f ? 0.f : 1.0f / L), qleft, qright, blk);
    const int i = row_token(a, split.row0 + r), hh = split.row0 + r - i * a.group;
    store4(static_cast<T*>(a.out) + (seq.start + static_cast<int64_t>(i)) * a.out_stride +
               (static_cast<int64_t>(g) * a.group + hh) * kDim + 4 * blk,
           x);
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Waves of rows: the fewest that hold the rows of a sequence on average, four above 64,
// eight above 128.  Over 4000 positions and 4 KV heads, fp16 and fp32 queries: 64 sequences
// of 32 rows 77 and 78 us (by two waves 102 and 106), 32 of 64 rows 65 and 70 (by four 79 and
// 91), 16 of 128 rows 67 and 74 (by eight 65 and 78).
int prefill_row_waves(int64_t rows) {
  return rows <= 32 ? 1 : (rows <= 64 ? 2 : (rows <= 128 ? 4 : 8));
}

}  // namespace

void prefill_plan(int64_t batch, int64_t n_tokens, int64_t n_kv_heads, int64_t group,
                  int64_t max_seq_len, bool f16, PrefillPlan* plan) {
  const int64_t n_rows = n_tokens * group;
  const int64_t with_rows = batch < n_tokens ? batch : n_tokens;   // sequences, at most
  const int rows = prefill_row_waves(batch > 0 ? n_rows / batch : 0);
  const int64_t block = 32 * rows;
  // the chip holds 512 workgroups of four waves, 256 of eight
  const int64_t workgroups = rows == 8 ? 256 : 512;
  int64_t shares = workgroups / n_kv_heads;
  shares = shares > 1 ? shares : 1;
  plan->row_waves = rows;
  plan->shares = shares;
  plan->max_pieces = n_rows / block + with_rows + 2 * shares;
  const size_t all = static_cast<size_t>(n_kv_heads) * n_rows;
  const size_t parts = static_cast<size_t>(2 * shares) * n_kv_heads * block;
  plan->q_op = 0;
  plan->q_down = align256(plan->q_op + all * kQBytes);
  plan->n_splits = align256(plan->q_down + all * 4);
  plan->splits = plan->n_splits + 256;
  plan->pieces = align256(plan->splits + static_cast<size_t>(shares) * sizeof(PrefillSplit));
  // the value scales' stretches: of 4096 positions, as few as keep the grid small
  plan->unit_chunks = 0;
  plan->unit_len = 0;
  if (rows == 8 && f16) {
    const int64_t most = batch < 4096 ? 4096 / batch : 1;
    const int64_t want = (max_seq_len + 4095) / 4096 > 1 ? (max_seq_len + 4095) / 4096 : 1;
    plan->unit_chunks = want < most ? want : most;
    plan->unit_len = (max_seq_len + plan->unit_chunks - 1) / plan->unit_chunks;
  }
  plan->units =
      align256(plan->pieces + static_cast<size_t>(plan->max_pieces) * sizeof(PrefillPiece));
  plan->part_ml = align256(
      plan->units + static_cast<size_t>(batch) * n_kv_heads * plan->unit_chunks * 4);
  plan->part_o = align256(plan->part_ml + parts * 8);
  plan->total_bytes = align256(plan->part_o + parts * 4 * kDim);
  // Of blocks of every size: fp32 queries, pieces of the smallest blocks, and the parts of
  // twice the chip's workgroups, of 128 rows or 256 (for one KV head at least).
  const size_t most_pieces = static_cast<size_t>(n_rows / 32 + with_rows + 1024);
  const size_t heads = static_cast<size_t>(n_kv_heads);
  size_t most_parts = 2 * 512 * 128;
  most_parts = most_parts > 2 * heads * 256 ? most_parts : 2 * heads * 256;
  size_t n = align256(all * kQBytes);
  n = align256(n + all * 4) + 256;
  n = align256(n + 512 * sizeof(PrefillSplit));
  n = align256(n + most_pieces * sizeof(PrefillPiece));
  n = align256(n + static_cast<size_t>(batch > 4096 ? batch : 4096) * heads * 4);
  n = align256(n + most_parts * 8);
  plan->bound_bytes = align256(n + most_parts * 4 * kDim);
}

hipError_t launch_prefill(const PrefillPlan& plan, const PrefillCall& c, const PageTable& pages,
                          void* workspace, hipStream_t stream) {
  PrefillArgs a;
  a.q = c.q;
  a.k_codes = c.k_codes;
  a.k_norms = c.k_norms;
  a.v_codes = c.v_codes;
  a.v_norms = c.v_norms;
  a.row_starts = c.row_starts;
  a.seq_lens = c.seq_lens;
  a.quats = c.quats;
  a.out = c.out;
  a.q_stride = c.q_stride;
  a.out_stride = c.out_stride;
  a.n_tokens = static_cast<int32_t>(c.n_tokens);
  a.n_rows = static_cast<int32_t>(c.n_tokens * c.group);
  a.max_seq_len = static_cast<int32_t>(c.max_seq_len);
  a.batch = static_cast<int32_t>(c.batch);
  a.n_kv_heads = static_cast<int32_t>(c.n_kv_heads);
  a.group = static_cast<int32_t>(c.group);
  // a window that no position of a row lies before sees everything
  a.window = c.window > c.max_seq_len ? 0 : static_cast<int32_t>(c.window);
  a.n_sinks = a.window == 0 ? 0
                            : static_cast<int32_t>(c.n_sinks < c.max_seq_len ? c.n_sinks
                                                                             : c.max_seq_len);
  a.block_rows = 32 * plan.row_waves;
  a.shares = static_cast<int32_t>(plan.shares);
  // tiles that a workgroup takes together
  a.round_tiles = plan.row_waves < 4 ? 4 / plan.row_waves
                  : plan.row_waves == 4 ? 1
                                        : (c.f16 ? kTurn : 2);
  a.group_magic = c.group == 1 ? 0 : static_cast<uint32_t>(((uint64_t{1} << 32) + c.group - 1) / c.group);
  a.unit_chunks = static_cast<int32_t>(plan.unit_chunks);
  a.unit_len = static_cast<int32_t>(plan.unit_len);
  a.max_pieces = static_cast<int32_t>(plan.max_pieces);
  a.max_parts = static_cast<int32_t>(2 * plan.shares);
  a.max_splits = static_cast<int32_t>(plan.shares);
  a.qscale = c.scale * kLog2e;
  a.pages = pages;
  char* ws = static_cast<char*>(workspace);
  a.q_op = ws + plan.q_op;
  a.q_down = reinterpret_cast<float*>(ws + plan.q_down);
  a.n_splits = reinterpret_cast<int32_t*>(ws + plan.n_splits);
  a.splits = reinterpret_cast<PrefillSplit*>(ws + plan.splits);
  a.pieces = reinterpret_cast<PrefillPiece*>(ws + plan.pieces);
  a.units = reinterpret_cast<float*>(ws + plan.units);
  a.part_ml = reinterpret_cast<float*>(ws + plan.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
  const unsigned heads = static_cast<unsigned>(c.n_kv_heads);
  const dim3 prep(static_cast<unsigned>(1 + c.batch * plan.unit_chunks + (a.n_rows + kTile - 1) / kTile),
                  heads);
  const dim3 grid(heads * static_cast<unsigned>(plan.max_pieces));
  const dim3 merge(1024);
  const Codebook cb = codebook_for<3>(nullptr);
#define IQ_LAUNCH_PREFILL(ROWS_, T_)                                                          \
  hipLaunchKernelGGL((prefill_kernel<ROWS_, T_>), grid, dim3(64 * prefill_waves<ROWS_>()), 0, \
                     stream, a, cb)
#define IQ_LAUNCH_PREFILL_T(T_)                                                               \
  do {                                                                                        \
    hipLaunchKernelGGL(prefill_prep_kernel<T_>, prep, dim3(kPrepThreads), 0, stream, a);      \
    hipError_t e = hipGetLastError();                                                         \
    if (e != hipSuccess) return e;                                                            \
    switch (plan.row_waves) {                                                                 \
      case 1: IQ_LAUNCH_PREFILL(1, T_); break;                                                \
      case 2: IQ_LAUNCH_PREFILL(2, T_); break;                                                \
      case 4: IQ_LAUNCH_PREFILL(4, T_); break;                                                \
      default:                                                                                \
        if (c.f16)                                                                            \
          hipLaunchKernelGGL(prefill_wide_kernel, grid, dim3(kWideThreads), 0, stream, a, cb); \
        else                                                                                  \
          IQ_LAUNCH_PREFILL(8, float);                                                        \
        break;                                                                                \
    }                                                                                         \
    if ((e = hipGetLastError()) != hipSuccess) return e;                                      \
    hipLaunchKernelGGL(prefill_merge_kernel<T_>, merge, dim3(kPrepThreads), 0, stream, a);    \
  } while (0)
  if (c.f16) {
    IQ_LAUNCH_PREFILL_T(_Float16);
  } else {
    IQ_LAUNCH_PREFILL_T(float);
  }
#undef IQ_LAUNCH_PREFILL_T
#undef IQ_LAUNCH_PREFILL
  return hipGetLastError();
}

}  // namespace iq

// Attention of a tree of drafted tokens over the packed cache (App. A per
// node; Table 2 A-D), gfx950: up to 64 nodes per sequence, whose records lie in
// a draft cache of their own, see the cached positions (all, or a window and
// sinks) and the nodes that their mask words name.
//
// For a KV head the rows (node, query head of the group) share every key and
// value, so a workgroup decodes each tile of 32 records once into fp16 in LDS
// and multiplies it with all of its rows on the matrix cores
// (v_mfma_f32_32x32x16_f16):
//
//  QK: S[key][row] = sum_d Khat[key][d] Qt[row][d].  A: 32 keys of the tile; B:
//    the wave's 32 rows, kept in registers as fp16 hi + lo parts (two products,
//    ~22 bits).  A lane ends up with 16 keys of one row.
//  PV: O[d][row] = sum_key Vhat[key][d] P[key][row].  The weights are B
//    operands as they stand: k index 8 h + j of product s' is the key 16 s' + 8
//    (j / 4) + 4 h + j % 4 that register 8 s' + j of the score accumulator holds
//    in half h of the wave, and the tile's values are stored in LDS by
//    dimension with the keys in that order.  Weights as fp16 hi + lo parts.
//
// One pass over the positions: each row keeps a reference maximum, raised (and
// the sums rescaled) when a score exceeds it by more than 2^kSlack, the sum of
// its weights and its outputs.  Value scales enter the weights in units of the
// largest exponent so far, as in the span kernel.
//
// Work decomposition: the waves of a workgroup (4, two workgroups per CU; or 8,
// one) are kRows waves of 32 rows times 4 / kRows groups of keys, each group with
// tiles of its own.  The tiles of a sequence are cut into pieces, as many as its share of
// all sequences' tiles; a workgroup takes one piece of a KV head and block of
// rows, so ragged batches fill the chip evenly.  The rotated queries and the
// pieces are prepared by a kernel of its own (a workgroup of many rows would
// spend more on its queries than on a short piece), the pieces' results are
// merged and rotated back by a third.
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

// What a node sees, by the prep kernel: the nodes (bits), cached positions from
// lo on (kBlind: it sees nothing) and the sinks.  In the attention's LDS `down`
// is the row's 2^-(exponent of the query parts).
struct TreeNode {
  uint64_t nodes;
  int32_t lo;
  float down;
};
constexpr int kBlind = 0x7fffffff;

// What the nodes of a sequence see together: the nodes, and the largest `lo` of
// a node that sees anything.
struct TreeSequence {
  uint64_t nodes;
  int32_t lo_max, pad;
};

// A piece: tiles t0 .. t1 - 1 of sequence b, whose length is len.
struct TreePiece {
  int32_t b, t0, t1, len;
};

struct TreeArgs {
  const float* q;
  const uint8_t* k_codes;
  const float* k_norms;
  const uint8_t* v_codes;
  const float* v_norms;
  const uint8_t* dk_codes;
  const float* dk_norms;
  const uint8_t* dv_codes;
  const float* dv_norms;
  const int32_t* seq_lens;
  const int64_t* tree_mask;
  const float* quats;
  float* out;
  int64_t capacity, draft_capacity;
  int32_t max_seq_len, batch, n_tok, n_kv_heads, group, n_rows, window, n_sinks;
  int32_t row_blocks;
  int32_t shares;     // pieces that the sequences share in proportion to their tiles
  int32_t min_tiles;  // tiles of a piece at least
  int32_t max_pieces;
  float qscale;
  PageTable pages;
  // workspace
  char* q_op;          // [batch][n_kv_heads][n_rows][2][128] fp16: hi and lo parts
  float* q_down;       // [batch][n_kv_heads][n_rows]: 2^-(exponent of the parts)
  TreeNode* nodes;     // [batch][n_tok]
  TreeSequence* seqs;  // [batch]
  TreePiece* pieces;   // [max_pieces], no tiles: none
  int32_t* first;      // [batch + 1]: each sequence's first piece
  float* part_ml;      // [max_pieces][n_kv_heads][n_rows][2]
  float* part_o;       // [max_pieces][n_kv_heads][n_rows][128]
};

__device__ __forceinline__ int tree_length(const TreeArgs& a, int b) {
  return span_length(a.seq_lens[b], a.max_seq_len);
}

// The tiles of a sequence: those of its cached positions, without the `skip`
// between the sinks' (n_sink of them) and the window's, then the drafts'.
struct TreeTiles {
  uint32_t n_sink, skip, n_cache, n;
  int lo;   // first position of a root's window
};
__device__ __forceinline__ TreeTiles tree_tiles(const TreeArgs& a, int len) {
  TreeTiles t;
  t.lo = a.window > 0 && len >= a.window ? len - a.window + 1 : 0;
  const uint32_t lo = t.lo, seen = a.n_sinks < len ? a.n_sinks : len;
  t.n_sink = (seen + kTile - 1) / kTile;
  t.skip = lo / kTile > t.n_sink ? lo / kTile - t.n_sink : 0;
  t.n_cache = (static_cast<uint32_t>(len) + kTile - 1) / kTile - t.skip;
  t.n = t.n_cache + (static_cast<uint32_t>(a.n_tok) + kTile - 1) / kTile;
  return t;
}

// ---- the rotated queries and the nodes' views --------------------------------
// (Short calls spend much of their time on fetching instructions: whole-number
// divisions, tens of instructions each, are kept out of these kernels.)
constexpr int kPrepThreads = 256;
constexpr int kPrepRows = kPrepThreads / 32;

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

// The row of a node: r / group, r < 2^13.  (The quotient in floats is off by less
// than 2^-9, and (r + 1/2) / group is at least 1 / (2 group) >= 2^-7 off an integer.)
static_assert(kMaxGroup <= 64 && IQ_MAX_TREE_NODES * kMaxGroup < (1 << 13), "");
__device__ __forceinline__ int row_node(int r, float inv_group) {
  return static_cast<int>((static_cast<float>(r) + 0.5f) * inv_group);
}

// The pieces: with `per` tiles of all sequences to a share, a sequence of n tiles
// gets the next whole number above n / per of them.  A little more than the even
// share of `shares` makes shares + batch pieces at most; where their rounding
// allows, more shares still fit into max_pieces (even sequences: all of them), so
// a few numbers between are tried.  One workgroup.
__device__ __forceinline__ void plan_pieces(const TreeArgs& a) {
  constexpr int kPlanWaves = kPrepThreads / 64, kTries = 4;
  __shared__ float sums[kPlanWaves];
  __shared__ int tried[kPlanWaves][kTries];
  __shared__ int starts[kPrepThreads], lens[kPrepThreads], counts[kPlanWaves];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int my_len = tid < a.batch ? tree_length(a, tid) : 0;   // of the first round
  const int my_n = tid < a.batch ? static_cast<int>(tree_tiles(a, my_len).n) : 0;
  auto tiles_of = [&](int b) { return static_cast<int>(tree_tiles(a, tree_length(a, b)).n); };
  int64_t all = my_n;
  for (int b = tid + kPrepThreads; b < a.batch; b += kPrepThreads) all += tiles_of(b);
  const float wave_total = wave64_sum(static_cast<float>(all));
  if (lane == 0) sums[wave] = wave_total;
  __syncthreads();
  float total = 0.f;
  for (int w = 0; w < kPlanWaves; ++w) total += sums[w];
  total *= 1.0001f;   // (above the exact sum, whatever the roundings)
  auto share_of = [&](int shares) {   // 1 / per
    const float per =
        floorf(total * __builtin_amdgcn_rcpf(static_cast<float>(shares)) + 1.0f);
    return __builtin_amdgcn_rcpf(fmaxf(per, static_cast<float>(a.min_tiles)));
  };
  auto pieces_of = [&](int n, float share) {
    return static_cast<int>(ceilf(static_cast<float>(n) * share));
  };
  float shares[kTries];
#pragma unroll
  for (int i = 0; i < kTries; ++i) {
    shares[i] = share_of(a.max_pieces - ((a.max_pieces - a.shares) * i >> 2));
    int n = pieces_of(my_n, shares[i]);
    for (int b = tid + kPrepThreads; b < a.batch; b += kPrepThreads)
      n += pieces_of(tiles_of(b), shares[i]);
    n = __builtin_amdgcn_readlane(wave_scan(n), 63);
    if (lane == 0) tried[wave][i] = n;
  }
  __syncthreads();
  float share = share_of(a.shares);
#pragma unroll
  for (int i = kTries - 1; i >= 0; --i) {
    int n = 0;
    for (int w = 0; w < kPlanWaves; ++w) n += tried[w][i];
    share = n <= a.max_pieces ? shares[i] : share;
  }
  int base = 0;   // pieces of the sequences before this round's
  for (int c0 = 0; c0 < a.batch; c0 += kPrepThreads) {
    const int b = c0 + tid;
    const int len = c0 == 0 ? my_len : (b < a.batch ? tree_length(a, b) : 0);
    const int n = c0 == 0 ? my_n : (b < a.batch ? static_cast<int>(tree_tiles(a, len).n) : 0);
    const int mine = pieces_of(n, share);
    const int incl = wave_scan(mine);
    if (lane == 63) counts[wave] = incl;
    __syncthreads();
    int start = base + incl - mine, end = base;
    for (int w = 0; w < kPlanWaves; ++w) {
      start += w < wave ? counts[w] : 0;
      end += counts[w];
    }
    starts[tid] = start;
    lens[tid] = len;
    if (b < a.batch) a.first[b] = start;
    __syncthreads();
    // the round's pieces, each with its sequence by bisection
    const int rows = a.batch - c0 < kPrepThreads ? a.batch - c0 : kPrepThreads;
    for (int p = base + tid; p < end; p += kPrepThreads) {
      int i = 0;
      for (int step = kPrepThreads / 2; step > 0; step >>= 1)
        if (i + step < rows && starts[i + step] <= p) i += step;
      const uint32_t of = (i + 1 < rows ? starts[i + 1] : end) - starts[i], at = p - starts[i];
      // even parts, of a tile at least (see pieces_of: per is)
      const uint32_t n = tree_tiles(a, lens[i]).n, each = n / of, more = n - each * of;
      const uint32_t t0 = at * each + (at < more ? at : more);
      a.pieces[p] = TreePiece{c0 + i, static_cast<int>(t0),
                              static_cast<int>(t0 + each + (at < more ? 1 : 0)), lens[i]};
    }
    base = end;
    __syncthreads();
  }
  if (tid == 0) a.first[a.batch] = base;
  for (int p = base + tid; p < a.max_pieces; p += kPrepThreads)
    a.pieces[p] = TreePiece{0, 0, 0, 0};
}

// Grid (1 + batch, n_kv_heads, 1 + blocks of 32 rows): the pieces, the nodes of a
// sequence, and the rotated queries of 32 rows of a KV head.
__global__ __launch_bounds__(kPrepThreads) void tree_prep_kernel(TreeArgs a) {
  const int tid = threadIdx.x;
  const int b = static_cast<int>(blockIdx.x) - 1, g = blockIdx.y;
  if (b < 0) {
    if (g == 0 && blockIdx.z == 0) plan_pieces(a);
    return;
  }
  if (blockIdx.z == 0) {
    // a wave, lane u the sequence's node u
    const int u = tid;
    if (g != 0 || u >= 64) return;
    const int len = tree_length(a, b);
    const uint64_t all = a.n_tok == 64 ? ~uint64_t{0} : (uint64_t{1} << a.n_tok) - 1;
    const uint64_t word =
        u < a.n_tok ? static_cast<uint64_t>(a.tree_mask[static_cast<int64_t>(b) * a.n_tok + u]) & all
                    : 0;
    const int pos = len + __builtin_popcountll(word & ~(uint64_t{1} << u));
    // (window 0: everything; positions are below 2^31, windows clamped to it)
    const int lo = a.window > 0 ? pos - a.window + 1 : 0;
    uint64_t mine = word;
    // (a window of n_tok positions holds every node of a path)
    for (int t = a.window > 0 && a.window < a.n_tok ? 0 : a.n_tok; t < a.n_tok; ++t) {
      const uint64_t wt =
          static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(
              static_cast<int>(word), t))) |
          (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(
               static_cast<int>(word >> 32), t)))
           << 32);
      const int lt = __builtin_amdgcn_readlane(lo, t);
      const bool in = (wt >> u & 1) && (pos >= lt || pos < a.n_sinks);
      const uint64_t view = __ballot(in);
      mine = u == t ? view : mine;
    }
    if (u < a.n_tok)
      a.nodes[static_cast<int64_t>(b) * a.n_tok + u] =
          TreeNode{mine, word ? lo : kBlind, 0.f};
    int top = word ? lo : INT32_MIN;
    uint64_t any = mine;
    for (int m = 1; m < 64; m <<= 1) {
      const int o = __shfl_xor(top, m);
      top = o > top ? o : top;
      any |= static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(any), m));
    }
    if (u == 0) a.seqs[b] = TreeSequence{any, top, 0};
    return;
  }
  // 32 rows of a KV head (those of one wave of the attention), each by 32 lanes,
  // lane blk its dims 4 blk .. 4 blk + 3
  __shared__ float row_max[kTile];
  const int blk = tid & 31;
  const int r0 = (static_cast<int>(blockIdx.z) - 1) * kTile;
  const int64_t bg = static_cast<int64_t>(b) * a.n_kv_heads + g;
  const float inv_group = __builtin_amdgcn_rcpf(static_cast<float>(a.group));
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t ql = par[0], qr = par[1];
  constexpr int kEach = kTile / kPrepRows;
  f32x4_t y[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = r0 + (tid >> 5) + kPrepRows * i;
    const int rc = r < a.n_rows ? r : a.n_rows - 1;   // every lane takes part
    const int t = row_node(rc, inv_group), h = rc - t * a.group;
    y[i] = *reinterpret_cast<const f32x4_t*>(
        a.q + (((static_cast<int64_t>(b) * a.n_tok + t) * a.n_kv_heads + g) * a.group + h) * kDim +
        4 * blk);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    y[i] = rotate_forward(y[i], ql, qr, blk, kInvSqrtDim * a.qscale);
    const float am = group32_max(fmaxf(fmaxf(fabsf(y[i][0]), fabsf(y[i][1])),
                                       fmaxf(fabsf(y[i][2]), fabsf(y[i][3]))));
    if (blk == 0) row_max[(tid >> 5) + kPrepRows * i] = am;
  }
  __syncthreads();
  // An exact power of two brings the largest entry below 2^14 (see attend_split):
  // one for the 32 rows where their largest entries are within 2^15 of each other
  // (the smallest still has its bits down to 2^-24), otherwise each row's own.
  const float mine = row_max[blk];
  const bool counts = mine > 0.f && mine < INFINITY;
  float most = group32_max(counts ? mine : 0.f);
  const float least = -group32_max(counts ? -mine : -INFINITY);
  const bool even = most == 0.f || least * 32768.0f >= most;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = r0 + (tid >> 5) + kPrepRows * i;
    const float am = even ? most : row_max[(tid >> 5) + kPrepRows * i];
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
      const int64_t row = bg * a.n_rows + r;
      uint2* dst = reinterpret_cast<uint2*>(a.q_op + row * 512 + 8 * blk);
      dst[0] = uint2{hi[0], hi[1]};
      dst[32] = uint2{lo[0], lo[1]};
      if (blk == 0) a.q_down[row] = ldexpf(1.0f, -e);
    }
  }
}

// ---- the attention -----------------------------------------------------------
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
struct TreeDecode {
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
struct TreeRows {
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

// Scores of a tile's keys at k, before their scales.
__device__ __forceinline__ f32x16_t tree_scores(const TreeRows& w, const char* k, int ql, int h) {
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
    x = mfma32(f[s], w.ql[s], x);
  }
  return x;
}

// Outputs: the values at v by the weights.
__device__ __forceinline__ void tree_values(TreeRows& w, const char* v, int ql, int h) {
  const char* vp = v + ql * kValStride + 16 * value_slot(ql, h);
  const char* vq = v + ql * kValStride + 16 * value_slot(ql, 2 + h);
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const u32x4_t f0 = *reinterpret_cast<const u32x4_t*>(vp + 32 * d * kValStride);
    const u32x4_t f1 = *reinterpret_cast<const u32x4_t*>(vq + 32 * d * kValStride);
    w.o[d] = mfma32(f0, w.ph[0], w.o[d]);
    w.o[d] = mfma32(f1, w.ph[1], w.o[d]);
    w.o[d] = mfma32(f0, w.pl[0], w.o[d]);
    w.o[d] = mfma32(f1, w.pl[1], w.o[d]);
  }
}

// Scores x become scores against the reference, rounded once; sc: key scales.
// view: the row's.  masked: the row sees only the keys whose bits of `see` (of keys 4 h ..) are set.
// Returns whether a row's reference has to be raised.
__device__ __forceinline__ bool tree_relative(const TreeRows& w, f32x16_t& x, const float* sc,
                                              const TreeNode* view, int h, bool masked,
                                              uint32_t see, float& top) {
  if (!w.even) {
    const float down = view->down;
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
__device__ __forceinline__ void tree_raise(TreeRows& w, f32x16_t& x, float top) {
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
// weight is not 0, so not in rows that do not see its key.)
__device__ __forceinline__ void tree_weights(TreeRows& w, const f32x16_t& x, const float* sc,
                                             int h) {
  float minus_one = -1.0f;
  asm volatile("" : "+s"(minus_one));
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&sc[8 * c + 4 * h]);
    float p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = __builtin_amdgcn_exp2f(x[4 * c + j]);
      w.l += e;
      p[j] = mul_or_zero(e, vs[j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t hi = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_pkrtz(p[2 * j], p[2 * j + 1]));
      w.ph[c >> 1][2 * (c & 1) + j] = hi;
      w.pl[c >> 1][2 * (c & 1) + j] = rest_pair(hi, p[2 * j], p[2 * j + 1], minus_one);
    }
  }
}

// kRows: waves of rows.  Groups of one or two of them (few rows) take a tile
// after the other.  Four and eight, where the matrix cores have most to do, are
// pipelined: while a tile's scores are multiplied the next tile is decoded, and
// while its weights are computed the tile before is multiplied with its values; a
// barrier, two buffers of keys and three of values per tile (four waves) or pair
// of tiles (eight, four of which decode each).
//
// What bounds it: with many rows the power of the products, most of the rest is
// decoding.  512 rows over 32K (two sequences, 4 KV heads) take 146 to 152 us in
// calls back to back, 0.90 to 0.94 PFLOP/s of fp16 products (159 in a profile of
// single calls, at 1.8 GHz; by four waves 179 there, of which 117 are left without
// the products and 123 without the decoding), and a loop of nothing but products of
// such data runs at 1.3 PFLOP/s (its clock falls to 1.3 GHz).  96 rows by four waves
// (16 sequences of 500 to 8191 on pools) keep the matrix cores busy for 29 % of the
// cycles and wait for 44 % of their waves': a barrier per tile, and one wave of four
// only decodes.  With few rows it is decoding
// through LDS, which is busy 58 % of the cycles: 32 rows over 8 sequences of 8192
// read 1.2 TB/s of records (records fetched two tiles ahead instead of one: the
// same time).
template <int kRows>
constexpr int tree_waves() {
  return kRows == 8 ? 8 : 4;
}
template <int kRows, bool kPaged, int kBits>
__global__ __launch_bounds__(64 * tree_waves<kRows>()) __attribute__((amdgpu_waves_per_eu(2)))
void tree_kernel(TreeArgs a, CodebookB<kBits> cb) {
  constexpr int kTreeWaves = tree_waves<kRows>(), kTreeThreads = 64 * kTreeWaves;
  constexpr int kRB = record_bytes<kBits>();
  constexpr int kGroups = kTreeWaves / kRows;
  // tiles of a barrier, decoded by four waves each
  constexpr int kPair = kRows == 8 ? 2 : 1;
  using Decode = TreeDecode<(kRows == 8 ? 4 : kRows), kBits>;
  constexpr int kKeyBufs = kRows == 1 ? 1 : 2 * kPair;
  constexpr int kValueBufs = kRows >= 4 ? 3 * kPair : kKeyBufs;
  struct Smem {
    uint32_t lut[1 << (2 * kBits)];
    union {
      TreeNode view[kTile];   // what the wave's rows see,
      float ml[kTile][2];     // in the end their references and sums
    } rows[kTreeWaves];
    float red[kTreeWaves];
    union {
      struct {
        char k[kGroups][kKeyBufs][kKeyBytes];
        char v[kGroups][kValueBufs][kValueBytes];
        float sc[kTreeWaves][kKeyBufs][2 * kTile];   // a wave's: key scales, value scales
      } t;
      float o[kTreeWaves][kTile][kORow];
    };
  };
  __shared__ __attribute__((aligned(16))) Smem sm;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ql = lane & 31, h = lane >> 5;
  const int kg = wave / kRows, rw = wave % kRows;
  const TreePiece piece = a.pieces[blockIdx.x];
  const int t0 = piece.t0, t1 = piece.t1, len = piece.len;
  if (t0 == t1) return;
  const int g = blockIdx.y, b = piece.b, bg = b * a.n_kv_heads + g;
  const int row0 = static_cast<int>(blockIdx.z) * (kRows * kTile);
  // rows of this piece
  const int64_t part = (static_cast<int64_t>(blockIdx.x) * a.n_kv_heads + g) * a.n_rows;
  const TreeTiles tiles = tree_tiles(a, len);
  const int n_sink = tiles.n_sink, skip = tiles.skip, n_cache = tiles.n_cache;
  const TreeSequence all = a.seqs[b];
  // positions of tile j start at first(j)
  auto first = [&](int j) {
    return j >= n_cache ? (j - n_cache) * kTile : (j < n_sink ? j : j + skip) * kTile;
  };
  // is position p of a tile (of drafts or not) there, and seen by some node?
  auto counts = [&](bool draft, int p) {
    return draft ? p < a.n_tok && (all.nodes >> p & 1)
                 : p < len && (p >= tiles.lo || p < a.n_sinks);
  };

  // ---- loads of a tile -----------------------------------------------------
  // The arrays as this wave needs them, kept in registers (selected where they
  // are used, their addresses come out of memory for every tile).
  struct Source {
    global_bytes_t keys, values;
    global_floats_t k_norms, v_norms;
    int64_t row;               // the first record (pools: of the pool)
  };
  Source cache{(global_bytes_t)a.k_codes, (global_bytes_t)a.v_codes,
               (global_floats_t)a.k_norms, (global_floats_t)a.v_norms,
               kPaged ? 0 : static_cast<int64_t>(bg) * a.capacity};
  Source drafts{(global_bytes_t)a.dk_codes, (global_bytes_t)a.dv_codes,
                (global_floats_t)a.dk_norms, (global_floats_t)a.dv_norms,
                static_cast<int64_t>(bg) * a.draft_capacity};
  for (Source* s : {&cache, &drafts}) {
    asm volatile("" : "+s"(s->keys), "+s"(s->values), "+s"(s->row));
    asm volatile("" : "+s"(s->k_norms), "+s"(s->v_norms));
  }
  // pools: the record of position p, whose page entry is given
  auto pool_record = [&](int p, int32_t entry) {
    const int64_t page =
        static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.pages.n_pages) ? entry : 0;
    return ((page * a.n_kv_heads + g) << a.pages.page_shift) +
           (p & ((1 << a.pages.page_shift) - 1));
  };
  // pools: the page entry of this lane's position of the next tile (a pair: of its
  // first tile in the lanes below 32, of its second above), read a tile (pair) ahead
  int32_t next_page = 0;
  auto load_pages = [&](int j) {
    if (!kPaged || j >= n_cache) return;
    const int jt = kPair == 2 && h && j + 1 < n_cache ? j + 1 : j;
    const int p = first(jt) + ql;
    next_page = a.pages.tables[static_cast<int64_t>(b) * a.pages.max_pages +
                               ((p < len ? p : len - 1) >> a.pages.page_shift)];
  };
  Decode dec;
  dec.setup(kRows == 8 ? rw & 3 : rw, lane);
  const int own = kRows == 8 ? rw >> 2 : 0;   // which tile of a pair this wave decodes
  float raw_scale[kPair];
  bool live[kPair];   // raw_scale is that of a position that somebody sees
  auto half_of = [&](int i) { return kRows == 1 ? i : rw & 1; };
  // Tile j's scale of this lane.
  auto load_scale = [&](int j, int32_t entry, float& raw, bool& counted) {
    const bool draft = j >= n_cache;
    const int p0 = first(j), last = (draft ? a.n_tok : len) - 1;
    const int p = p0 + ql < last ? p0 + ql : last;
    const int64_t r =
        kPaged && !draft ? pool_record(p, entry) : (draft ? drafts.row : cache.row) + p;
    // (this lane's: a key's scale in half 0, a value's in half 1)
    const global_floats_t kn = draft ? drafts.k_norms : cache.k_norms;
    const global_floats_t vn = draft ? drafts.v_norms : cache.v_norms;
    raw = (h ? vn : kn)[r];
    counted = counts(draft, p0 + ql);
  };
  // Tile j's records that this wave decodes.
  auto load_records = [&](int j, int32_t entry) {
    const bool draft = j >= n_cache;
    const int p0 = first(j);
    const int last = (draft ? a.n_tok : len) - 1;
    const bool whole = p0 + kTile - 1 <= last;
    const int64_t row = draft ? drafts.row : cache.row;
    const global_bytes_t keys = draft ? drafts.keys : cache.keys;
    const global_bytes_t values = draft ? drafts.values : cache.values;
#pragma unroll
    for (int i = 0; i < Decode::kTasks; ++i) {
      // the half's first position, or the last one there is
      const int at = p0 + 16 * half_of(i), p = at < last ? at : last;
      const int64_t r = kPaged && !draft
                            ? pool_record(p, __builtin_amdgcn_readlane(entry, 16 * half_of(i)))
                            : row + p;
      dec.load(i, keys + r * kRB, values + r * kRB, last - p, whole);
    }
  };
  auto ahead = [&](int jt) { return jt < t1 ? jt : t1 - 1; };   // (past the end: the last tile)
  // Tile j, or the pair from j on.
  auto load = [&](int j) {
    if constexpr (kPair == 2) {
      const int j1 = ahead(j + 1);
      int32_t e0 = next_page, e1 = next_page;
      if constexpr (kPaged) {
        const auto both = __builtin_amdgcn_permlane32_swap(e0, e0, false, false);
        e0 = both[0];                       // the lower lanes' in both halves
        e1 = j1 == j ? e0 : both[1];        // the upper lanes'
      }
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
    load_pages(kRows >= 4 ? ahead(j + kPair) : j + kGroups);
  }
  // ---- the wave's rows --------------------------------------------------------
  TreeRows w;
  float down;
  const int row = row0 + rw * kTile + ql;
  const int rc = row < a.n_rows ? row : a.n_rows - 1;
  {
    const int64_t qrow = static_cast<int64_t>(bg) * a.n_rows + rc;
    const char* src = a.q_op + qrow * 512 + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      w.qh[s] = *reinterpret_cast<const u32x4_t*>(src + 32 * s);
      w.ql[s] = *reinterpret_cast<const u32x4_t*>(src + 256 + 32 * s);
    }
    down = a.q_down[qrow];
  }
  TreeNode node =
      a.nodes[static_cast<int64_t>(b) * a.n_tok +
              row_node(rc, __builtin_amdgcn_rcpf(static_cast<float>(a.group)))];
  // ---- the unit of the value scales: the exponent of the largest finite one
  // that somebody sees in this piece ------------------------------------------
  float largest = 0.f;
  {
    constexpr int kAhead = 4, kStep = kTreeThreads / kTile;
    for (int jt = t0 + (tid >> 5); jt < t1; jt += kAhead * kStep) {
      float v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int je = jt + u * kStep < t1 ? jt + u * kStep : t1 - 1;
        const bool draft = je >= n_cache;
        const int p = first(je) + ql;
        const bool in = counts(draft, p);
        // (a position that does not count: the first one's scale is read instead)
        int64_t r = (draft ? drafts.row : cache.row) + (in ? p : 0);
        if (kPaged && !draft)
          r = pool_record(in ? p : 0,
                          a.pages.tables[static_cast<int64_t>(b) * a.pages.max_pages +
                                         (in ? p >> a.pages.page_shift : 0)]);
        const float s = (draft ? a.dv_norms : a.v_norms)[r];
        v[u] = in ? s : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        largest = fabsf(v[u]) < INFINITY ? fmaxf(largest, fabsf(v[u])) : largest;
    }
    largest = wave64_max(largest);
    if (lane == 0) sm.red[wave] = largest;
  }
  // (in LDS: read where a tile is masked, and in the end)
  node.down = down;
  const TreeNode* const view = &sm.rows[wave].view[ql];
  if (h == 0) sm.rows[wave].view[ql] = node;
  // (arrived before the loop: a wait for them inside it would be one for the next
  // tile's records as well)
#pragma unroll
  for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(w.qh[s]), "+v"(w.ql[s]));
  w.m = -INFINITY;
  w.l = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] = 0.f;
  const float down0 =
      __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, down)));
  w.even = __all(down == down0);
  build_pair_table(sm, cb, tid);
  lds_barrier();   // the pair table, red
#pragma unroll
  for (int i = 0; i < kTreeWaves; ++i) largest = fmaxf(largest, sm.red[i]);
  uint32_t unit = __builtin_amdgcn_readfirstlane(
      static_cast<int>(__builtin_bit_cast(uint32_t, largest) & 0x7F800000u));
  unit = unit > kMinScaleBits ? unit : kMinScaleBits;
  // what this lane's scale is staged times
  const float factor =
      h ? __builtin_bit_cast(float, ((127u + 127u + kUnitBits) << 23) - unit)
        : (w.even ? down0 : 1.0f);
  auto store = [&](char* k, char* v, float* sc) {
#pragma unroll
    for (int i = 0; i < kPair; ++i) sc[2 * kTile * i + lane] = live[i] ? raw_scale[i] * factor : 0.f;
#pragma unroll
    for (int i = 0; i < Decode::kTasks; ++i) dec.store(sm.lut, i, half_of(i), k, v);
  };
  // bits of the keys of tile j that this lane's row sees; false: all rows all
  auto see = [&](int jt, uint32_t& bits) {
    const int p0 = first(jt);
    const bool draft = jt >= n_cache;
    bits = 0;
    if (!draft && p0 + kTile <= len && (p0 >= all.lo_max || p0 + kTile <= a.n_sinks)) return false;
    bits = draft ? static_cast<uint32_t>(view->nodes >> p0)
                 : low_bits(len - p0) & (~low_bits(view->lo - p0) | low_bits(a.n_sinks - p0));
    bits >>= 4 * h;
    return true;
  };

  if constexpr (kRows >= 4) {
    constexpr int kKeyStep = kPair * kKeyBytes, kValueStep = kPair * kValueBytes;
    constexpr int kScaleStep = kPair * 2 * kTile;
    char* const kbuf = sm.t.k[0][0];
    char* vfree = sm.t.v[0][2 * kPair];
    char* vcur = sm.t.v[0][0];
    char* vnext = sm.t.v[0][kPair];
    char* vlast = vfree;   // the tile whose weights are ready
    float* const sc = sm.t.sc[wave][0];
    const int own_k = own * kKeyBytes, own_v = own * kValueBytes;
    // before the first tile: weights of nothing, times values of nothing
    for (int e = tid; e < kValueBytes / 16; e += kTreeThreads)
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
      if (tree_relative(w, x, scales, view, h, masked, bits, top)) {
        tree_values(w, vlast, ql, h);
#pragma unroll
        for (int s = 0; s < 2; ++s) w.ph[s] = w.pl[s] = u32x4_t{0, 0, 0, 0};
        tree_raise(w, x, top);
      }
      tree_values(w, vlast, ql, h);
      tree_weights(w, x, scales + kTile, h);
      // the products one by one between the weights' instructions (24 nodes of 16
      // paged sequences: 115 us, in the compiler's own order 119.5)
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x402, 5, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    };
    // (a wave without rows only decodes)
    if (row0 + rw * kTile >= a.n_rows) {
      for (int it = 0; j < t1; ++it, j += kPair) {
        const int next = it & 1 ^ 1;
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
      f32x16_t x = tree_scores(w, k, ql, h);
      store(kbuf + (cur ^ 1) * kKeyStep + own_k, vnext + own_v, sc + (cur ^ 1) * kScaleStep);
      load(ahead(j + 2 * kPair));
      load_pages(ahead(j + 3 * kPair));
      finish(x, j, scales);
      vlast = vcur;
      if constexpr (kPair == 2) {
        x = tree_scores(w, k + kKeyBytes, ql, h);
        finish(x, j + 1, scales + 2 * kTile);
        vlast = vcur + kValueBytes;
      }
      char* const was = vcur;
      vcur = vnext;
      vnext = vfree;
      vfree = was;
      lds_barrier();
    }
    tree_values(w, vlast, ql, h);
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
        load_pages(j + 2 * kGroups);
      }
      if constexpr (kRows == 1)
        wave_lds_fence();
      else
        lds_barrier();
      if (j < t1) {
        uint32_t bits;
        const bool masked = see(j, bits);
        f32x16_t x = tree_scores(w, k, ql, h);
        float top;
        if (tree_relative(w, x, sc, view, h, masked, bits, top)) tree_raise(w, x, top);
        tree_weights(w, x, sc + kTile, h);
        tree_values(w, v, ql, h);
      }
      if constexpr (kRows == 1) wave_lds_fence();   // the next tile behind this one's reads
    }
  }

  // ---- the groups' results joined, by row -------------------------------------
  lds_barrier();   // every wave is done with the tiles
  const f32x2_t ls = half_pair(w.l);
  if (h == 0) {
    // (a node that sees nothing: no result, whatever the unmasked tiles gave)
    const bool blind = view->lo == kBlind;
    wave_lds_fence();   // every lane has read its row's
    sm.rows[wave].ml[ql][0] = blind ? -INFINITY : w.m;
    sm.rows[wave].ml[ql][1] = blind ? 0.f : ls[0] + ls[1];
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
  for (int r = tid >> 5; r < kRows * kTile; r += kTreeThreads / 32) {
    if (row0 + r >= a.n_rows) break;
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
    const int64_t at = part + row0 + r;
    if (blk == 0) *reinterpret_cast<f32x2_t*>(&a.part_ml[2 * at]) = f32x2_t{M, L};
    *reinterpret_cast<f32x4_t*>(&a.part_o[kDim * at + 4 * blk]) = O;
  }
}

// ---- merge of the parts, inverse rotation -------------------------------------
// A row's 128 dims are 32 threads' (4 each); kShare groups of them share its
// parts.  Grid (batch, n_kv_heads, blocks of 8 / kShare rows).
template <int kShare>
__global__ __launch_bounds__(kPrepThreads) void tree_merge_kernel(TreeArgs a) {
  constexpr int kUnroll = 8;
  __shared__ __attribute__((aligned(16))) f32x4_t red_o[kPrepRows][32];
  __shared__ float red_m[kPrepRows], red_l[kPrepRows];
  const int blk = threadIdx.x & 31, slot = static_cast<int>(threadIdx.x) >> 5;
  const int64_t b = blockIdx.x;
  const int g = blockIdx.y;
  const int row = static_cast<int>(blockIdx.z) * (kPrepRows / kShare) + slot / kShare;
  const int r = row < a.n_rows ? row : a.n_rows - 1;   // every lane takes part
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t qleft = par[0], qright = par[1];
  float M = -INFINITY, L = 0.f;
  f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int p0 = a.first[b], p1 = a.first[b + 1];
  for (int s0 = p0 + slot % kShare; s0 < p1; s0 += kShare * kUnroll) {
    f32x2_t ml[kUnroll];
    f32x4_t o[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int s = s0 + kShare * u < p1 ? s0 + kShare * u : s0;
      const int64_t at = (static_cast<int64_t>(s) * a.n_kv_heads + g) * a.n_rows + r;
      ml[u] = *reinterpret_cast<const f32x2_t*>(&a.part_ml[2 * at]);
      o[u] = *reinterpret_cast<const f32x4_t*>(&a.part_o[kDim * at + 4 * blk]);
      if (s0 + kShare * u >= p1) ml[u] = f32x2_t{-INFINITY, 0.f};
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
      // (a group without a maximum: nothing seen, or only NaN scores, whose sum is NaN)
      const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      L += c * red_l[slot + u];
      O += c * red_o[slot + u][blk];
    }
  }
  // (a row that sees nothing is zero; a sum that is NaN stays visible)
  const f32x4_t x = rotate_inverse(O * (L == 0.f ? 0.f : 1.0f / L), qleft, qright, blk);
  if (row >= a.n_rows) return;
  const int t = row_node(r, __builtin_amdgcn_rcpf(static_cast<float>(a.group)));
  const int h = r - t * a.group;
  *reinterpret_cast<f32x4_t*>(
      a.out + (((b * a.n_tok + t) * a.n_kv_heads + g) * a.group + h) * kDim + 4 * blk) = x;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Waves of rows for n_rows rows per KV head: the fewest that hold them, four above
// 64.  Eight decode a tile for 256 rows where four do for 128 (256 rows of 4
// sequences of 8192: 69.9 us, by fours 72.6; 512 rows over 32K: attention 159 us,
// by fours 179, both in a profile of single calls), but their last 128 rows are half idle where blocks of 128 do not
// pair up (640 rows of 2 sequences of 8192: 48.0 us, by fours 45.3).
int tree_row_waves(int64_t n_rows) {
  if (n_rows <= 64) return n_rows <= 32 ? 1 : 2;
  return (n_rows + 127) / 128 % 2 ? 4 : 8;
}

}  // namespace

// Pieces and workspace.  The chip holds 512 workgroups of four waves, 256 of
// eight: pieces enough for one round of them (a round and a little more would
// take the time of two), or for at least two per sequence on average (long
// sequences beside short ones) where the sequences alone fill half of it.  (Even
// sequences get two by that as well, which they would not need: 64 of 24 nodes, 4
// heads per KV head and 8 KV heads over 1024 positions 111 us, over 4096 289, for
// products of 45 and 180.)
void tree_plan(int64_t batch, int64_t n_tok, int64_t n_kv_heads, int64_t group,
               int64_t max_seq_len, int64_t window, int64_t n_sinks, TreePlan* plan) {
  const int64_t n_rows = n_tok * group;
  const int rows = tree_row_waves(n_rows);
  const int64_t kWorkgroups = rows == 8 ? 256 : 512;
  const int64_t blocks = (n_rows + 32 * rows - 1) / (32 * rows);
  int64_t seen = max_seq_len;
  if (window > 0 && n_sinks < seen && window < seen) {
    const int64_t w = (n_sinks + kTile - 1) / kTile * kTile + window + 2 * kTile;
    seen = w < seen ? w : seen;
  }
  const int64_t tiles = (seen + kTile - 1) / kTile + (n_tok + kTile - 1) / kTile;
  const int64_t groups = rows < 4 ? 4 / rows : 1;
  int64_t shares = kWorkgroups / (n_kv_heads * blocks) - batch;
  shares = shares > batch ? shares : batch;
  // (no more than there can be pieces of a tile per group of waves)
  const int64_t most = batch * ((tiles + groups - 1) / groups);
  shares = shares < most ? shares : most;
  shares = shares > 1 ? shares : 1;
  plan->row_waves = rows;
  plan->row_blocks = blocks;
  plan->shares = shares;
  plan->min_tiles = groups;
  plan->max_pieces = shares + batch < most ? shares + batch : (most > 1 ? most : 1);
  const size_t all = static_cast<size_t>(batch) * n_kv_heads * n_rows;
  const size_t parts = static_cast<size_t>(plan->max_pieces) * n_kv_heads * n_rows;
  plan->q_op = 0;
  plan->q_down = align256(plan->q_op + all * 512);
  plan->nodes = align256(plan->q_down + all * 4);
  plan->seqs = align256(plan->nodes + static_cast<size_t>(batch) * n_tok * sizeof(TreeNode));
  plan->first = align256(plan->seqs + static_cast<size_t>(batch) * sizeof(TreeSequence));
  plan->pieces = align256(plan->first + static_cast<size_t>(batch + 1) * 4);
  plan->part_ml =
      align256(plan->pieces + static_cast<size_t>(plan->max_pieces) * sizeof(TreePiece));
  plan->part_o = align256(plan->part_ml + parts * 8);
  plan->total_bytes = align256(plan->part_o + parts * 4 * kDim);
  // What no smaller batch, tree, length or window needs more of: the pieces that one
  // block of rows would have, and for the rows of all pieces those that the chip's
  // workgroups hold (512 of up to 128 rows, 256 of up to 256) or two pieces of every
  // row.
  const int64_t one_block = 512 / n_kv_heads > 2 * batch ? 512 / n_kv_heads : 2 * batch;
  const int64_t most_pieces = one_block < most ? one_block : (most > 1 ? most : 1);
  const int64_t all_rows = batch * n_kv_heads * n_rows, held = 512 * (n_rows < 128 ? n_rows : 128);
  int64_t most_parts = held > 2 * all_rows ? held : 2 * all_rows;
  const int64_t by_tiles = (most > 1 ? most : 1) * n_kv_heads * n_rows;
  most_parts = most_parts < by_tiles ? most_parts : by_tiles;
  const size_t ml =
      align256(plan->pieces + static_cast<size_t>(most_pieces) * sizeof(TreePiece));
  plan->bound_bytes = align256(align256(ml + static_cast<size_t>(most_parts) * 8) +
                               static_cast<size_t>(most_parts) * 4 * kDim);
}

hipError_t launch_decode_tree(const TreePlan& plan, const TreeCall& c, const PageTable* pages,
                              int bits, void* workspace, hipStream_t stream) {
  TreeArgs a;
  a.q = c.q;
  a.k_codes = c.k_codes;
  a.k_norms = c.k_norms;
  a.v_codes = c.v_codes;
  a.v_norms = c.v_norms;
  a.dk_codes = c.dk_codes;
  a.dk_norms = c.dk_norms;
  a.dv_codes = c.dv_codes;
  a.dv_norms = c.dv_norms;
  a.seq_lens = c.seq_lens;
  a.tree_mask = c.tree_mask;
  a.quats = c.quats;
  a.out = c.out;
  a.capacity = c.capacity;
  a.draft_capacity = c.draft_capacity;
  a.max_seq_len = static_cast<int32_t>(c.max_seq_len);
  a.batch = static_cast<int32_t>(c.batch);
  a.n_tok = static_cast<int32_t>(c.n_tok);
  a.n_kv_heads = static_cast<int32_t>(c.n_kv_heads);
  a.group = static_cast<int32_t>(c.group);
  a.n_rows = static_cast<int32_t>(c.n_tok * c.group);
  // a window that no position of a row lies before sees everything
  a.window = c.window > c.max_seq_len + c.n_tok ? 0 : static_cast<int32_t>(c.window);
  a.n_sinks = static_cast<int32_t>(c.n_sinks < c.max_seq_len + c.n_tok ? c.n_sinks
                                                                       : c.max_seq_len + c.n_tok);
  a.row_blocks = static_cast<int32_t>(plan.row_blocks);
  a.shares = static_cast<int32_t>(plan.shares);
  a.min_tiles = static_cast<int32_t>(plan.min_tiles);
  a.max_pieces = static_cast<int32_t>(plan.max_pieces);
  a.qscale = c.scale * kLog2e;
  a.pages = pages ? *pages : PageTable{nullptr, 0, 4, 1};
  char* ws = static_cast<char*>(workspace);
  a.q_op = ws + plan.q_op;
  a.q_down = reinterpret_cast<float*>(ws + plan.q_down);
  a.nodes = reinterpret_cast<TreeNode*>(ws + plan.nodes);
  a.seqs = reinterpret_cast<TreeSequence*>(ws + plan.seqs);
  a.first = reinterpret_cast<int32_t*>(ws + plan.first);
  a.pieces = reinterpret_cast<TreePiece*>(ws + plan.pieces);
  a.part_ml = reinterpret_cast<float*>(ws + plan.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
  const unsigned batch = static_cast<unsigned>(c.batch), heads = static_cast<unsigned>(c.n_kv_heads);
  const unsigned q_blocks = static_cast<unsigned>((a.n_rows + kTile - 1) / kTile);
  hipLaunchKernelGGL(tree_prep_kernel, dim3(1 + batch, heads, 1 + q_blocks), dim3(kPrepThreads), 0,
                     stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(static_cast<unsigned>(plan.max_pieces), heads,
                  static_cast<unsigned>(plan.row_blocks));
#define IQ_LAUNCH_TREE(ROWS_, PAGED_, BITS_)                                                 \
  hipLaunchKernelGGL((tree_kernel<ROWS_, PAGED_, BITS_>), grid, dim3(64 * tree_waves<ROWS_>()), 0, stream, \
                     a, codebook_for<BITS_>(nullptr))
#define IQ_LAUNCH_TREE_R(ROWS_)        \
  if (pages) {                         \
    IQ_LAUNCH_TREE(ROWS_, true, 3);    \
  } else if (bits == 2) {              \
    IQ_LAUNCH_TREE(ROWS_, false, 2);   \
  } else if (bits == 4) {              \
    IQ_LAUNCH_TREE(ROWS_, false, 4);   \
  } else {                             \
    IQ_LAUNCH_TREE(ROWS_, false, 3);   \
  }
  switch (plan.row_waves) {
    case 1: IQ_LAUNCH_TREE_R(1); break;
    case 2: IQ_LAUNCH_TREE_R(2); break;
    case 4: IQ_LAUNCH_TREE_R(4); break;
    default: IQ_LAUNCH_TREE_R(8); break;
  }
#undef IQ_LAUNCH_TREE_R
#undef IQ_LAUNCH_TREE
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (rows of many parts on average are read by 8 groups of threads)
#define IQ_LAUNCH_TREE_MERGE(SHARE_)                                                            \
  hipLaunchKernelGGL(tree_merge_kernel<SHARE_>,                                                 \
                     dim3(batch, heads,                                                         \
                          static_cast<unsigned>((a.n_rows * SHARE_ + kPrepRows - 1) / kPrepRows)), \
                     dim3(kPrepThreads), 0, stream, a)
  if (plan.max_pieces > 16 * c.batch) {
    IQ_LAUNCH_TREE_MERGE(8);
  } else {
    IQ_LAUNCH_TREE_MERGE(1);
  }
#undef IQ_LAUNCH_TREE_MERGE
  return hipGetLastError();
}

}  // namespace iq

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
// Work decomposition: the waves of a workgroup (8) are kRows waves of 32 rows
// times 8 / kRows groups of keys, each group with tiles of its own; workgroups
// split the tiles of a sequence and KV head evenly.  The rotated queries are
// prepared by a kernel of their own (a workgroup of 256 rows would spend more
// on them than on a short stretch of tiles), the parts are merged and rotated
// back by a third.
#include <hip/hip_runtime.h>
#include <math.h>

#include "iq_span_device.h"

namespace iq {
namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
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

struct TileBuf {
  char k[kTile * kKeyStride];
  char v[kDim * kValStride];
  float ks[kTile];   // key scales
  float vs[kTile];   // value scales times 2^kUnitBits / unit, 0 past the end
  uint32_t unit[4];  // [0]: the unit
};

// What a node sees, by the prep kernel: the nodes (bits), cached positions from
// lo on, and those before sinks (-1: it sees nothing).
struct TreeNode {
  uint64_t nodes;
  int32_t lo, sinks;
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
  int32_t n_splits, row_blocks;
  float qscale;
  PageTable pages;
  // workspace
  char* q_op;          // [batch][n_kv_heads][n_rows][2][128] fp16: hi and lo parts
  float* q_down;       // [batch][n_kv_heads][n_rows]: 2^-(exponent of the parts)
  TreeNode* nodes;     // [batch][n_tok]
  int32_t* lo_max;     // [batch]: largest lo of a node that sees anything
  float* part_ml;      // [batch][n_kv_heads][n_splits][n_rows][2]
  float* part_o;       // [batch][n_kv_heads][n_splits][n_rows][128]
};

__device__ __forceinline__ int tree_length(const TreeArgs& a, int b) {
  return span_length(a.seq_lens[b], a.max_seq_len);
}

// ---- the rotated queries and the nodes' views --------------------------------
constexpr int kPrepThreads = 256;
constexpr int kPrepRows = kPrepThreads / 32;
__global__ __launch_bounds__(kPrepThreads) void tree_prep_kernel(TreeArgs a, int q_blocks) {
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) >= q_blocks) {
    // one wave per sequence, lane u its node u
    const int b = (static_cast<int>(blockIdx.x) - q_blocks) * (kPrepThreads / 64) + (tid >> 6);
    const int u = tid & 63;
    if (b >= a.batch) return;
    const int len = tree_length(a, b);
    const uint64_t all = a.n_tok == 64 ? ~uint64_t{0} : (uint64_t{1} << a.n_tok) - 1;
    const uint64_t word =
        u < a.n_tok ? static_cast<uint64_t>(a.tree_mask[static_cast<int64_t>(b) * a.n_tok + u]) & all
                    : 0;
    const int pos = len + __builtin_popcountll(word & ~(uint64_t{1} << u));
    // (window 0: everything; positions are below 2^31, windows clamped to it)
    const int lo = a.window > 0 ? pos - a.window + 1 : 0;
    uint64_t mine = 0;
    for (int t = 0; t < a.n_tok; ++t) {
      const uint64_t wt =
          static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(
              static_cast<int>(word), t))) |
          (static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(
               static_cast<int>(word >> 32), t)))
           << 32);
      const int lt = __builtin_amdgcn_readlane(lo, t);
      const bool in = (wt >> u & 1) && (a.window == 0 || pos >= lt || pos < a.n_sinks);
      const uint64_t view = __ballot(in);
      mine = u == t ? view : mine;
    }
    if (u < a.n_tok)
      a.nodes[static_cast<int64_t>(b) * a.n_tok + u] =
          TreeNode{mine, word ? lo : 0x7fffffff, word ? a.n_sinks : -1};
    int top = word ? lo : INT32_MIN;
    for (int m = 1; m < 64; m <<= 1) {
      const int o = __shfl_xor(top, m);
      top = o > top ? o : top;
    }
    if (u == 0) a.lo_max[b] = top;
    return;
  }
  // one query row per 32 lanes, lane blk its dims 4 blk .. 4 blk + 3
  const int blk = tid & 31;
  const int64_t n = static_cast<int64_t>(a.batch) * a.n_kv_heads * a.n_rows;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kPrepRows + (tid >> 5);
  const int64_t rc = row < n ? row : n - 1;   // every lane takes part in the rotation
  const int r = static_cast<int>(rc % a.n_rows);
  const int64_t bg = rc / a.n_rows;
  const int g = static_cast<int>(bg % a.n_kv_heads);
  const int64_t b = bg / a.n_kv_heads;
  const int t = r / a.group, h = r - t * a.group;
  const f32x4_t x = *reinterpret_cast<const f32x4_t*>(
      a.q + (((b * a.n_tok + t) * a.n_kv_heads + g) * a.group + h) * kDim + 4 * blk);
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  const f32x4_t y = rotate_forward(x, par[0], par[1], blk, kInvSqrtDim * a.qscale);
  // an exact power of two brings the largest entry below 2^14 (see attend_split)
  const float am = group32_max(fmaxf(fmaxf(fabsf(y[0]), fabsf(y[1])),
                                     fmaxf(fabsf(y[2]), fabsf(y[3]))));
  int e = 0;
  if (am > 0.f) {
    frexpf(am, &e);
    e = 14 - e;
    e = e > 100 ? 100 : (e < -100 ? -100 : e);
  }
  const float up = ldexpf(1.0f, e);
  uint32_t hi[2], lo[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float x0 = y[2 * j] * up, x1 = y[2 * j + 1] * up;
    const _Float16 h0 = static_cast<_Float16>(x0), h1 = static_cast<_Float16>(x1);
    hi[j] = __builtin_bit_cast(uint32_t, half2_t{h0, h1});
    lo[j] = __builtin_bit_cast(uint32_t,
                               half2_t{static_cast<_Float16>(x0 - static_cast<float>(h0)),
                                       static_cast<_Float16>(x1 - static_cast<float>(h1))});
  }
  if (row >= n) return;
  uint2* dst = reinterpret_cast<uint2*>(a.q_op + row * 512 + 8 * blk);
  dst[0] = uint2{hi[0], hi[1]};
  dst[32] = uint2{lo[0], lo[1]};
  if (blk == 0) a.q_down[row] = ldexpf(1.0f, -e);
}

// ---- the attention -----------------------------------------------------------
// One wave's rows: what it carries from tile to tile.
struct TreeRows {
  u32x4_t qh[8], ql[8];   // query operands: dims 16 s + 8 h .. of row lane % 32
  f32x16_t o[4];          // outputs, in units of unit / 2^kUnitBits
  float m, l;             // reference (scaled domain), this lane's share of the sum
  float down;             // scaled domain to log2 units
  uint32_t unit;
  uint64_t nodes;
  int lo, sinks;
};

// The lowest n (clamped to 0 .. 32) of 32 bits.
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n >= 32 ? ~0u : (n > 0 ? (1u << n) - 1 : 0u);
}

// One tile in `t`.  masked: the row sees only the tile's keys whose bits of `see`
// (of keys 4 h ..) are set.  (One body for both: two move the outputs between
// registers, and spill.)
__device__ __forceinline__ void tree_tile(TreeRows& w, const TileBuf& t, int ql, int h,
                                          bool masked, uint32_t see) {
  f32x16_t x;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
  const char* kp = t.k + ql * kKeyStride + 16 * h;
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const u32x4_t k = *reinterpret_cast<const u32x4_t*>(kp + 32 * s);
    x = mfma32(k, w.qh[s], x);
    x = mfma32(k, w.ql[s], x);
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&t.ks[8 * c + 4 * h]);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 * c + j] *= ks[j];
  }
  if (masked) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      x[i] = see >> (8 * (i / 4) + i % 4) & 1 ? x[i] : -INFINITY;
  }
  float top = x[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
  const f32x2_t tops = half_pair(top);
  top = fmaxf(tops[0], tops[1]);
  const uint32_t unit = __builtin_amdgcn_readfirstlane(t.unit[0]);
  if (unit != w.unit || __any((top - w.m) * w.down > kSlack)) {
    const float m = fmaxf(w.m, top);
    const float f = w.m == m ? 1.0f
                             : (w.m == -INFINITY ? 0.f
                                                 : __builtin_amdgcn_exp2f((w.m - m) * w.down));
    // the old unit over the new, exactly (0 if beyond the exponent range)
    const int de = static_cast<int>(w.unit >> 23) - static_cast<int>(unit >> 23) + 127;
    const float fu =
        f * (de > 0 ? __builtin_bit_cast(float, static_cast<uint32_t>(de) << 23) : 0.f);
    w.l *= f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[d][i] *= fu;
    w.m = m;
    w.unit = unit;
  }
  const float mq = w.m == -INFINITY ? 0.f : -w.m * w.down;
  u32x4_t ph[2], pl[2];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&t.vs[8 * c + 4 * h]);
    float p[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * c + j], w.down, mq));
      w.l += e;
      p[j] = e * vs[j];
    }
    if (masked) {   // (a scale that is not finite counts where its key is seen)
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = x[4 * c + j] == -INFINITY ? 0.f : p[j];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const _Float16 h0 = static_cast<_Float16>(p[2 * j]), h1 = static_cast<_Float16>(p[2 * j + 1]);
      ph[c >> 1][2 * (c & 1) + j] = __builtin_bit_cast(uint32_t, half2_t{h0, h1});
      pl[c >> 1][2 * (c & 1) + j] = __builtin_bit_cast(
          uint32_t, half2_t{static_cast<_Float16>(p[2 * j] - static_cast<float>(h0)),
                            static_cast<_Float16>(p[2 * j + 1] - static_cast<float>(h1))});
    }
  }
  // (the values' reads stay behind the weights: earlier they spill)
  __builtin_amdgcn_sched_barrier(0);
  const char* vp = t.v + ql * kValStride + 16 * h;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(vp + 32 * d * kValStride + 32 * s);
      w.o[d] = mfma32(v, ph[s], w.o[d]);
      w.o[d] = mfma32(v, pl[s], w.o[d]);
    }
}

// kRows: waves of rows.  Decoding a tile is 128 tasks of keys (a record's
// quarter) and 128 of values (8 dims of 4 records): a lane of a group's only
// wave has two of each, of two waves one has the keys and one the values, of
// four or eight the first two the keys and the next two the values.
template <int kRows, bool kPaged, int kBits>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void tree_kernel(TreeArgs a, CodebookB<kBits> cb) {
  constexpr int kGroups = kWaves / kRows;
  constexpr int kBufs = kRows == 1 ? 1 : 2;
  constexpr int kTasks = kRows <= 2 ? 2 : 1;
  constexpr int kRB = record_bytes<kBits>();
  constexpr int kScaleWave = kRows == 8 ? 4 : 0;
  struct Smem {
    uint32_t lut[1 << (2 * kBits)];
    float ml[kWaves][kTile][2];
    union {
      TileBuf tile[kGroups][kBufs];
      float o[kWaves][kTile][kORow];
    };
  };
  __shared__ __attribute__((aligned(16))) Smem sm;
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63, ql = lane & 31, h = lane >> 5;
  const int kg = wave / kRows, rw = wave % kRows;
  int id = blockIdx.x;
  const int rb = id % a.row_blocks;
  id /= a.row_blocks;
  const int split = id % a.n_splits, bg = id / a.n_splits;
  const int g = bg % a.n_kv_heads, b = bg / a.n_kv_heads;
  const int row0 = rb * (kRows * kTile);
  const int64_t part = static_cast<int64_t>(id) * a.n_rows;   // rows of this part

  // ---- the tiles: those of the sinks, of the window, of the drafts ----------
  const int len = tree_length(a, b);
  const int lo0 = a.window > 0 && len >= a.window ? len - a.window + 1 : 0;   // the root's
  const int seen = a.n_sinks < len ? a.n_sinks : len;
  const int n_sink = (seen + kTile - 1) / kTile;
  const int skip = lo0 / kTile > n_sink ? lo0 / kTile - n_sink : 0;
  const int n_cache = (len + kTile - 1) / kTile - skip;
  const int n_tiles = n_cache + (a.n_tok + kTile - 1) / kTile;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * split / a.n_splits);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (split + 1) / a.n_splits);
  if (t1 <= t0) {
    for (int r = row0 + tid; r < a.n_rows && r < row0 + kRows * kTile; r += kThreads)
      *reinterpret_cast<f32x2_t*>(&a.part_ml[2 * (part + r)]) = f32x2_t{-INFINITY, 0.f};
    return;
  }
  // positions of tile j start at first(j); before limit(j) they are there
  auto first = [&](int j) {
    return j >= n_cache ? (j - n_cache) * kTile : (j < n_sink ? j : j + skip) * kTile;
  };

  // ---- loads of a tile: the tasks' record slices, and the scales ------------
  // task i of this lane: keys of record lane / 4 + 16 slot(i), quarter lane % 4;
  // values of records 4 (lane / 16 + 4 slot(i)) .. + 3, dims 8 (lane % 16) ..
  uint32_t raw_k[kTasks][kBits], raw_v[kTasks][4];
  float raw_scale = 0.f;
  const bool keys = kRows == 1 || (kRows == 2 ? rw == 0 : rw < 2);
  const bool values = kRows == 1 || (kRows == 2 ? rw == 1 : (rw & 6) == 2);
  auto slot = [&](int i) { return kRows >= 4 ? rw & 1 : i; };
  // (a value's dword, or the record's last one where that one reaches past it)
  const int vu = lane & 15;
  const int voff = kBits * vu < kRB - 4 ? kBits * vu : kRB - 4;
  const uint32_t vshift = static_cast<uint32_t>(8 * (kBits * vu - voff));
  auto load = [&](int j) {
    const int p0 = first(j);
    const bool draft = j >= n_cache;
    const int last = (draft ? a.n_tok : len) - 1;
    const uint8_t* kc = draft ? a.dk_codes : a.k_codes;
    const uint8_t* vc = draft ? a.dv_codes : a.v_codes;
    // record of position p: base0 + p in the tile's lower half, base1 + p in its
    // upper one (pages hold at least 16)
    int64_t base0 = static_cast<int64_t>(bg) * (draft ? a.draft_capacity : a.capacity);
    int64_t base1 = base0;
    if (kPaged && !draft) {
      auto page_base = [&](int at) {
        const int p = at < last ? at : last;
        const int32_t pg =
            a.pages.tables[static_cast<int64_t>(b) * a.pages.max_pages + (p >> a.pages.page_shift)];
        const int64_t page =
            static_cast<uint32_t>(pg) < static_cast<uint32_t>(a.pages.n_pages) ? pg : 0;
        return ((page * a.n_kv_heads + g) << a.pages.page_shift) -
               (static_cast<int64_t>(p >> a.pages.page_shift) << a.pages.page_shift);
      };
      base0 = page_base(p0);
      base1 = page_base(p0 + 16);
    }
    auto record = [&](int key) {
      const int p = p0 + key < last ? p0 + key : last;
      return (p - p0 < 16 ? base0 : base1) + p;
    };
    if (rw == kScaleWave) {
      const float* s = h ? (draft ? a.dv_norms : a.v_norms) : (draft ? a.dk_norms : a.k_norms);
      raw_scale = s[record(ql)];
    }
    if (keys) {
#pragma unroll
      for (int i = 0; i < kTasks; ++i) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(
            kc + record((lane >> 2) + 16 * slot(i)) * kRB + 4 * kBits * (lane & 3));
#pragma unroll
        for (int e = 0; e < kBits; ++e) raw_k[i][e] = src[e];
      }
    }
    if (values) {
#pragma unroll
      for (int i = 0; i < kTasks; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          raw_v[i][e] = *reinterpret_cast<const u32_a1_t*>(
              vc + record(4 * ((lane >> 4) + 4 * slot(i)) + e) * kRB + voff);
    }
  };
  uint32_t unit = kMinScaleBits;   // the scale wave's
  auto store = [&](TileBuf& t, int j) {
    if (rw == kScaleWave) {
      const int there = (j >= n_cache ? a.n_tok : len) - first(j);
      const float s = ql < there ? raw_scale : 0.f;
      // (of finite scales only: one that is not is no unit for the others)
      const uint32_t e =
          __builtin_bit_cast(uint32_t, wave64_max(h && fabsf(s) < INFINITY ? s : 0.f)) & 0x7F800000u;
      unit = e > unit ? e : unit;
      const float up = __builtin_bit_cast(float, ((127u + 127u + kUnitBits) << 23) - unit);
      if (h)
        t.vs[ql] = s * up;
      else
        t.ks[ql] = s;
      if (lane == 0) t.unit[0] = unit;
    }
    if (keys) {
#pragma unroll
      for (int i = 0; i < kTasks; ++i) {
        u32x4_t p[4];
        key_pairs<kBits>(sm.lut, raw_k[i], p);
        char* dst = t.k + ((lane >> 2) + 16 * slot(i)) * kKeyStride + 64 * (lane & 3);
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<u32x4_t*>(dst + 16 * e) = p[e];
      }
    }
    if (values) {
#pragma unroll
      for (int i = 0; i < kTasks; ++i) {
        const int q4 = (lane >> 4) + 4 * slot(i);
        u32x4_t p[4];
        window_pairs<kBits>(sm.lut, raw_v[i], vshift, p);
        // dims 8 u + 2 n, + 1 of the 4 records: 8 bytes each, in the order of
        // the weights (see the top): records 4 q4 .. in half q4 / 2 % 2 of
        // 16-byte slot 2 (q4 / 4) + q4 % 2
        char* dst = t.v + 8 * vu * kValStride + 16 * (2 * (q4 >> 2) + (q4 & 1)) + 8 * (q4 >> 1 & 1);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          *reinterpret_cast<uint2*>(dst + 2 * n * kValStride) =
              uint2{__builtin_amdgcn_perm(p[n][1], p[n][0], 0x05040100u),
                    __builtin_amdgcn_perm(p[n][3], p[n][2], 0x05040100u)};
          *reinterpret_cast<uint2*>(dst + (2 * n + 1) * kValStride) =
              uint2{__builtin_amdgcn_perm(p[n][1], p[n][0], 0x07060302u),
                    __builtin_amdgcn_perm(p[n][3], p[n][2], 0x07060302u)};
        }
      }
    }
  };

  int j = t0 + kg;
  if (j < t1) load(j);
  // ---- the wave's rows --------------------------------------------------------
  TreeRows w;
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
    w.down = a.q_down[qrow];
    const TreeNode node = a.nodes[static_cast<int64_t>(b) * a.n_tok + rc / a.group];
    w.nodes = node.nodes;
    w.lo = node.lo;
    w.sinks = node.sinks;
  }
  const int lo_max = a.lo_max[b];
  w.m = -INFINITY;
  w.l = 0.f;
  w.unit = kMinScaleBits;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] = 0.f;
  build_pair_table(sm, cb, tid);
  lds_barrier();   // the pair table

  const int n_iter = (t1 - t0 + kGroups - 1) / kGroups;
  for (int it = 0; it < n_iter; ++it, j += kGroups) {
    TileBuf& t = sm.tile[kg][it % kBufs];
    if (j < t1) store(t, j);
    if (j + kGroups < t1) load(j + kGroups);
    if constexpr (kRows == 1)
      wave_lds_fence();
    else
      lds_barrier();
    if (j < t1) {
      const int p0 = first(j);
      const bool draft = j >= n_cache;
      const bool masked = draft || p0 + kTile > len || (p0 < lo_max && p0 + kTile > a.n_sinks);
      uint32_t bits = 0;
      if (masked)
        bits = draft ? static_cast<uint32_t>(w.nodes >> p0)
                     : low_bits(len - p0) & (~low_bits(w.lo - p0) | low_bits(w.sinks - p0));
      tree_tile(w, t, ql, h, masked, bits >> (4 * h));
    }
    if constexpr (kRows == 1) wave_lds_fence();   // the next tile behind this one's reads
  }

  // ---- the groups' results joined, by row -------------------------------------
  lds_barrier();   // every wave is done with the tiles
  const f32x2_t ls = half_pair(w.l);
  if (h == 0) {
    // (a node that sees nothing: no result, whatever the unmasked tiles gave)
    sm.ml[wave][ql][0] = w.sinks < 0 ? -INFINITY : w.m * w.down;
    sm.ml[wave][ql][1] = w.sinks < 0 ? 0.f : ls[0] + ls[1];
  }
  const float oscale = __builtin_bit_cast(float, w.unit) * (1.0f / (1 << kUnitBits));
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      *reinterpret_cast<f32x4_t*>(&sm.o[wave][ql][32 * d + 8 * c + 4 * h]) =
          f32x4_t{w.o[d][4 * c], w.o[d][4 * c + 1], w.o[d][4 * c + 2], w.o[d][4 * c + 3]} * oscale;
  lds_barrier();
  const int blk = tid & 31;
  for (int r = tid >> 5; r < kRows * kTile; r += kThreads / 32) {
    if (row0 + r >= a.n_rows) break;
    float M = -INFINITY, L = 0.f;
    f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGroups; ++k) M = fmaxf(M, sm.ml[k * kRows + r / kTile][r % kTile][0]);
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const int wv = k * kRows + r / kTile;
      const float m = sm.ml[wv][r % kTile][0];
      // (without a maximum: nothing seen, a sum of 0, or only NaN scores)
      const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
      L += c * sm.ml[wv][r % kTile][1];
      if (m != -INFINITY)
        O += c * *reinterpret_cast<const f32x4_t*>(&sm.o[wv][r % kTile][4 * blk]);
    }
    const int64_t at = part + row0 + r;
    if (blk == 0) *reinterpret_cast<f32x2_t*>(&a.part_ml[2 * at]) = f32x2_t{M, L};
    *reinterpret_cast<f32x4_t*>(&a.part_o[kDim * at + 4 * blk]) = O;
  }
}

// ---- merge of the parts, inverse rotation -------------------------------------
__global__ __launch_bounds__(kPrepThreads) void tree_merge_kernel(TreeArgs a) {
  const int blk = threadIdx.x & 31;
  const int64_t n = static_cast<int64_t>(a.batch) * a.n_kv_heads * a.n_rows;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kPrepRows + (threadIdx.x >> 5);
  const int64_t rc = row < n ? row : n - 1;
  const int r = static_cast<int>(rc % a.n_rows);
  const int64_t bg = rc / a.n_rows;
  const int g = static_cast<int>(bg % a.n_kv_heads);
  const int64_t b = bg / a.n_kv_heads;
  float M = -INFINITY, L = 0.f;
  f32x4_t O = f32x4_t{0.f, 0.f, 0.f, 0.f};
  constexpr int kUnroll = 8;
  for (int s0 = 0; s0 < a.n_splits; s0 += kUnroll) {
    f32x2_t ml[kUnroll];
    f32x4_t o[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int s = s0 + u < a.n_splits ? s0 + u : s0;
      const int64_t at = (bg * a.n_splits + s) * a.n_rows + r;
      ml[u] = *reinterpret_cast<const f32x2_t*>(&a.part_ml[2 * at]);
      o[u] = *reinterpret_cast<const f32x4_t*>(&a.part_o[kDim * at + 4 * blk]);
      if (s0 + u >= a.n_splits) ml[u][0] = -INFINITY;
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
  const f32x4_t* par =
      reinterpret_cast<const f32x4_t*>(a.quats + static_cast<int64_t>(g) * kQuatFloats + 8 * blk);
  // (a row that sees nothing is zero; a sum that is NaN stays visible)
  const f32x4_t x = rotate_inverse(O * (L == 0.f ? 0.f : 1.0f / L), par[0], par[1], blk);
  if (row >= n) return;
  const int t = r / a.group, h = r - t * a.group;
  *reinterpret_cast<f32x4_t*>(
      a.out + (((b * a.n_tok + t) * a.n_kv_heads + g) * a.group + h) * kDim + 4 * blk) = x;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// waves of rows for n_rows rows per KV head
int tree_row_waves(int64_t n_rows) {
  return n_rows <= 32 ? 1 : (n_rows <= 64 ? 2 : (n_rows <= 128 ? 4 : 8));
}

}  // namespace

// Workgroups per (sequence, KV head) and block of rows, and the workspace.
void tree_plan(int64_t batch, int64_t n_tok, int64_t n_kv_heads, int64_t group,
               int64_t max_seq_len, int64_t window, int64_t n_sinks, TreePlan* plan) {
  constexpr int64_t kWorkgroups = 256;
  const int64_t n_rows = n_tok * group;
  const int rows = tree_row_waves(n_rows);
  const int64_t blocks = (n_rows + 32 * rows - 1) / (32 * rows);
  int64_t seen = max_seq_len;
  if (window > 0 && n_sinks < seen && window < seen) {
    const int64_t w = (n_sinks + kTile - 1) / kTile * kTile + window + 2 * kTile;
    seen = w < seen ? w : seen;
  }
  const int64_t tiles = (seen + kTile - 1) / kTile + (n_tok + kTile - 1) / kTile;
  const int64_t wgs = batch * n_kv_heads * blocks;
  int64_t s = wgs > 0 ? kWorkgroups / wgs : 1;
  const int64_t most = tiles / (kWaves / rows);   // a tile per group of waves
  s = s < most ? s : most;
  s = s > 1 ? s : 1;
  plan->row_waves = rows;
  plan->row_blocks = blocks;
  plan->n_splits = s;
  const size_t all = static_cast<size_t>(batch) * n_kv_heads * n_rows;
  plan->q_op = 0;
  plan->q_down = align256(plan->q_op + all * 512);
  plan->nodes = align256(plan->q_down + all * 4);
  plan->lo_max = align256(plan->nodes + static_cast<size_t>(batch) * n_tok * sizeof(TreeNode));
  plan->part_ml = align256(plan->lo_max + static_cast<size_t>(batch) * 4);
  plan->part_o = align256(plan->part_ml + all * s * 8);
  plan->total_bytes = align256(plan->part_o + all * s * 4 * kDim);
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
  a.n_splits = static_cast<int32_t>(plan.n_splits);
  a.row_blocks = static_cast<int32_t>(plan.row_blocks);
  a.qscale = c.scale * kLog2e;
  a.pages = pages ? *pages : PageTable{nullptr, 0, 4, 1};
  char* ws = static_cast<char*>(workspace);
  a.q_op = ws + plan.q_op;
  a.q_down = reinterpret_cast<float*>(ws + plan.q_down);
  a.nodes = reinterpret_cast<TreeNode*>(ws + plan.nodes);
  a.lo_max = reinterpret_cast<int32_t*>(ws + plan.lo_max);
  a.part_ml = reinterpret_cast<float*>(ws + plan.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + plan.part_o);
  const int64_t rows = c.batch * c.n_kv_heads * a.n_rows;
  const int64_t q_blocks = (rows + kPrepRows - 1) / kPrepRows;
  const int64_t b_blocks = (c.batch + kPrepThreads / 64 - 1) / (kPrepThreads / 64);
  hipLaunchKernelGGL(tree_prep_kernel, dim3(static_cast<unsigned>(q_blocks + b_blocks)),
                     dim3(kPrepThreads), 0, stream, a, static_cast<int>(q_blocks));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(static_cast<unsigned>(c.batch * c.n_kv_heads * plan.n_splits * plan.row_blocks));
#define IQ_LAUNCH_TREE(ROWS_, PAGED_, BITS_)                                                 \
  hipLaunchKernelGGL((tree_kernel<ROWS_, PAGED_, BITS_>), grid, dim3(kThreads), 0, stream, a, \
                     codebook_for<BITS_>(nullptr))
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
  hipLaunchKernelGGL(tree_merge_kernel, dim3(static_cast<unsigned>(q_blocks)), dim3(kPrepThreads),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace iq

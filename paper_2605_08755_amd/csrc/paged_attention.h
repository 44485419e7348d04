// Attention over paged key/value caches: what its kernels share for every type
// of cache.  The work of a batch and its division into items, the kernel for
// prompts' chunks (256 or 128 query rows a block), the joining of split
// sequences, and the sizes that follow.  fp32 sums and softmax statistics, fixed reduction
// orders (deterministic).  Head dimension 128.
//
// A batch of B sequences: sequence b owns rows token_start[b] ..
// token_start[b + 1] - 1, which are the last of its seq_len[b] positions;
// position t lies in page page_table[b][t / page_size].  These arrays live in
// device memory and the host never reads them, so a captured graph serves a
// growing batch.  Nothing read from them is trusted as an address: rows are
// clamped to 0 .. T, positions to the table's width, and a page outside the
// cache is a page that is not there.
#pragma once

#include <float.h>
#include <math.h>

#include <algorithm>

#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kHeadDim = 128;
constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;  // log2(e) / sqrt(128)
constexpr float kNoMax = -1e30f;  // running maximum before the first visible score (finite: no inf - inf)

typedef float float16_t __attribute__((ext_vector_type(16)));
typedef float float2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int readlane(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <int CTRL>
__device__ __forceinline__ int dpp_i(int v, int old) {
  return __builtin_amdgcn_update_dpp(old, v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __builtin_bit_cast(float, dpp_i<CTRL>(__builtin_bit_cast(int, v), 0));
}
// Sum over the eight lanes of a half DPP row / maximum and sum over the 16
// lanes of a row, in every lane.
__device__ __forceinline__ float sum8(float v) {
  v += dpp_f<0xB1>(v);   // quad_perm [1,0,3,2]
  v += dpp_f<0x4E>(v);   // quad_perm [2,3,0,1]
  v += dpp_f<0x141>(v);  // row_half_mirror
  return v;
}
__device__ __forceinline__ float row_sum(float v) {
  v = sum8(v);
  v += dpp_f<0x140>(v);  // row_mirror
  return v;
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}
// The larger, NaN where one is: one instruction for three numbers, while fmaxf
// first quiets each that may be a signalling NaN, as it holds a matrix product to
// be.  (Measured on MI355X, two prompts of 8192 and 4001 rows, 32:8 heads, both
// ways in turn in two runs: fp16 caches 757 -> 751 and 758 -> 750 us, codes 721 ->
// 707 and 721 -> 708.)
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// Inclusive prefix sum over the 64 lanes: shifts by 1, 2, 4, 8 within each
// 16-lane row (lanes shifted in read 0), then the rows' totals.
__device__ __forceinline__ int wave_scan(int v, int lane) {
  v += dpp_i<0x111>(v, 0);
  v += dpp_i<0x112>(v, 0);
  v += dpp_i<0x114>(v, 0);
  v += dpp_i<0x118>(v, 0);
  const int t0 = readlane(v, 15), t1 = readlane(v, 31), t2 = readlane(v, 47);
  return v + (lane >= 16 ? t0 : 0) + (lane >= 32 ? t1 : 0) + (lane >= 48 ? t2 : 0);
}
// Sum over the 64 lanes of whole numbers below 2^53 (exact in any order).
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = (uint32_t)dpp_i<CTRL>((int)(uint32_t)u, 0), hi = (uint32_t)dpp_i<CTRL>((int)(u >> 32), 0);
  return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ double lane_d(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)readlane((int)(u >> 32), l) << 32 |
                                        (uint32_t)readlane((int)(uint32_t)u, l));
}
__device__ __forceinline__ double wave_sum_exact(double v) {
  v += dpp_d<0xB1>(v);
  v += dpp_d<0x4E>(v);
  v += dpp_d<0x141>(v);
  v += dpp_d<0x140>(v);
  return (lane_d(v, 0) + lane_d(v, 16)) + (lane_d(v, 32) + lane_d(v, 48));
}
__device__ __forceinline__ int wave_sum(int v) {
  v += dpp_i<0xB1>(v, 0);
  v += dpp_i<0x4E>(v, 0);
  v += dpp_i<0x141>(v, 0);
  v += dpp_i<0x140>(v, 0);
  return (readlane(v, 0) + readlane(v, 16)) + (readlane(v, 32) + readlane(v, 48));
}

// ---------------------------------------------------------------------------
// attention: the work of a batch
// ---------------------------------------------------------------------------

// The work of one key/value head is cut into items: a tile of BM query rows
// (row r = token r / R, query head r % R of the head's R) of one sequence, and
// a range of its positions.  A sequence's positions are split into ranges of
// `chunk` units of 64 positions; the chunk is chosen on the device from the
// batch's own lengths, so that all items together are about kItems per
// launch: a long sequence among short ones, or a single one, still occupies
// the chip, and a sequence that fits one range is written without a second
// pass.  Every block derives the same numbers from the same arrays; the grid
// and the workspace are sized by bounds that hold for any lengths:
//   items <= kItems / Hkv + tiles,  records (ranges of split tiles) <= 2 kItems / Hkv,
//   split tiles <= kItems / Hkv     per key/value head,
// since a sequence of x units has ceil(x / chunk) < x / chunk + 1 ranges, at
// most 2 x / chunk where it is split, and chunk >= (sum of tiles x units) Hkv / kItems.
constexpr int kUnit = 64;
constexpr int kSmallRows = 16;
template <int WAVES>
constexpr int kChunkRows = 32 * WAVES;  // of a block of the chunks' kernel
// Blocks of 16 rows that run at once, two a compute unit; twice the blocks of
// 256.  (Measured on MI355X with 256 and 1024: 16 decoding sequences 44 us -> 54
// and 44, three long ones 160 -> 149 and 159, a chunk beside 15 decoding rows 70
// -> 84 and 78, without the joining.)
constexpr int kItems = 512;
// Units: a shorter range costs more in records than it gains.  (Measured on
// MI355X: one token at 300 positions 7.4 us with 2, 9.5 with 4; a chunk of 16
// rows at 6000, 16.3 us with 4, 17.4 with 3, 22 with 2.)
template <int BM>
constexpr int kMinChunk = BM == kSmallRows ? 2 : 4;

// One sequence, seen from one lane.
struct Seq {
  int s0, n, pos0, end, lo;  // first row, rows, first row's position, positions there are, first position of the ranges
  int tiles, units;
};

// TILE: each tile's own positions are cut into equal ranges, as many as the
// sequence's other tiles have (a window's tiles, or a fresh prompt's, see unlike
// parts of the sequence); else the sequence's are, and a tile skips what it does
// not see.  The chunk then is an upper bound of a range.
template <int BM, bool TILE>
__device__ __forceinline__ Seq load_seq(const PagedBatch& pb, int b, int R, int window) {
  Seq q{0, 0, 0, 0, 0, 0, 0};
  if (b < pb.B) {
    q.s0 = min(max(pb.token_start[b], 0), pb.T);
    const int s1 = min(max(pb.token_start[b + 1], q.s0), pb.T);
    const int len = max(pb.seq_len[b], 0);
    q.n = s1 - q.s0;
    q.pos0 = len - q.n;
    q.end = min(len, pb.table_pages << pb.page_shift);
    if (window > 0) q.lo = max(q.pos0 - window + 1, 0) & -kUnit;
    if (q.n > 0) {
      q.tiles = (q.n * R + BM - 1) / BM;
      q.units = max((q.end - q.lo + kUnit - 1) / kUnit, 1);  // rows that see nothing are an item too
      if (TILE && window > 0) {  // the window of a tile's first token, up to its last one, from a unit's start
        const int tokens = min(q.n, (BM + R - 2) / R + 1);
        q.units = min(q.units, (int)(((int64_t)window + tokens + 2 * (kUnit - 1) - 1) / kUnit));
      }
    }
  }
  return q;
}

// Results of one item: rows of partial sums (split) or of outputs.  And the plan.
struct Out {
  uint16_t* out;
  float* ws;
  const int* plan;
  int Hq, rec_bound, min_chunk;
};

struct Item {
  bool found;
  int b, s0, n, pos0, end, lo;
  int tile, split, splits, chunk;
  int rec;  // first record of the tile's ranges
};

// The smallest chunk by that bound, of all sequences' tiles x units.
// (min_chunk: that of the call, kMinChunk, or all units where nothing is split.)
__device__ __forceinline__ int least_chunk(double total, int Hkv, int min_chunk) {
  const double share = total * Hkv * (1.0 / kItems);
  return uniform(max((int)fmin(share, 33554432.0) + 1, min_chunk));
}

// Batches of more than 64 sequences have a plan in the workspace, which a kernel
// of one block makes first, so that a block's search does not pass over all of
// them, whose time grew with their square.  Whole numbers: the chunk; then per
// group of 64 sequences the items before it, then likewise the records, then the
// split tiles.  (Measured on MI355X, decoding sequences of 128 and of 1024
// positions, 32:8 heads, each block passing over all -> the plan: 65, 14.4 -> 17.6
// and 81 -> 76 us; 256, 46 -> 40 and 206 -> 182; 4096, 3.6 -> 0.55 and 5.9 -> 2.7 ms.)
constexpr int kGroup = 64;
__host__ __device__ constexpr int64_t plan_groups(int64_t B) { return B > kGroup ? (B + kGroup - 1) / kGroup : 0; }

constexpr int kPlanWaves = 16;
template <int BM, bool TILE>
__global__ __launch_bounds__(64 * kPlanWaves) void paged_attention_plan_kernel(PagedBatch pb, int R, int Hkv,
                                                                               int window, int min_chunk,
                                                                               int* __restrict__ plan) {
  __shared__ double totals[kPlanWaves];
  __shared__ int sums[kPlanWaves][3];
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int groups = (int)plan_groups(pb.B);
  double total = 0.0;
  for (int g = w; g < groups; g += kPlanWaves) {
    const Seq q = load_seq<BM, TILE>(pb, g * kGroup + lane, R, window);
    total += wave_sum_exact((double)q.tiles * q.units);
  }
  if (lane == 0) totals[w] = total;
  __syncthreads();
  total = 0.0;
  for (int i = 0; i < kPlanWaves; ++i) total += totals[i];
  const int chunk = least_chunk(total, Hkv, min_chunk);
  if (threadIdx.x == 0) plan[0] = chunk;
  int* const before = plan + 1;
  int upto[3] = {0, 0, 0};
  for (int g0 = 0; g0 < groups; g0 += kPlanWaves) {
    const int g = g0 + w;
    const Seq q = load_seq<BM, TILE>(pb, min(g, groups) * kGroup + lane, R, window);  // (none past the last group)
    const int splits = (q.units + chunk - 1) / chunk;
    const int items = wave_sum(q.tiles * splits), split = wave_sum(splits > 1 ? q.tiles : 0),
              recs = wave_sum(splits > 1 ? q.tiles * splits : 0);
    if (lane == 0) sums[w][0] = items, sums[w][1] = recs, sums[w][2] = split;
    __syncthreads();
    for (int i = 0; i < 3; ++i) {
      int at = upto[i];
      for (int k = 0; k < w; ++k) at += sums[k][i];
      if (lane == 0 && g < groups) before[i * groups + g] = at;
      for (int k = 0; k < kPlanWaves; ++k) upto[i] += sums[k][i];
    }
    __syncthreads();
  }
}

// Item `idx` of a key/value head (SPLIT: the idx-th split tile).
template <int BM, bool TILE, bool SPLIT>
__device__ __forceinline__ Item find_item(const PagedBatch& pb, const Out& o, int idx, int R, int Hkv, int window,
                                          int lane) {
  const int* const plan = o.plan;
  Item it;
  it.found = false;
  int items = 0, recs = 0, b0 = 0;
  Seq q;
  if (pb.B > kGroup) {
    // the last group with no more items before it than idx, 64 groups a step
    const int groups = (int)plan_groups(pb.B);
    const int* const before = plan + 1;
    const int* const first = before + (SPLIT ? 2 * groups : 0);
    int g = 0;
    for (int left = groups; left > 1;) {
      const int step = (left + 63) >> 6, at = lane * step;
      const int n = max(__popcll(__ballot(at < left && first[g + min(at, left - 1)] <= idx)), 1) - 1;
      g += n * step;
      left = min(step, left - n * step);
    }
    g = uniform(g);
    b0 = g * kGroup;
    it.chunk = uniform(plan[0]);
    items = uniform(first[g]);
    recs = uniform(before[groups + g]);
    q = load_seq<BM, TILE>(pb, b0 + lane, R, window);
  } else {
    q = load_seq<BM, TILE>(pb, lane, R, window);
    // That chunk, then up to 3/8 and one unit larger until the items are no more
    // than the blocks that run at once (a few more would run alone).
    const int least = least_chunk(wave_sum_exact((double)q.tiles * q.units), Hkv, o.min_chunk);
    it.chunk = least;
    for (int i = 0; i < 4; ++i) {
      const int c = least + least * i / 8 + (i > 0);
      if (wave_sum(q.tiles * ((q.units + c - 1) / c)) * Hkv <= kItems) {
        it.chunk = c;
        break;
      }
    }
    it.chunk = uniform(it.chunk);
  }
  const int splits = (q.units + it.chunk - 1) / it.chunk;
  const int rec = splits > 1 ? q.tiles * splits : 0;
  const int own = SPLIT ? (splits > 1 ? q.tiles : 0) : q.tiles * splits;
  const int upto = items + wave_scan(own, lane);
  const int rupto = recs + wave_scan(rec, lane);
  const uint64_t past = __ballot(upto > idx);
  if (!past) return it;
  const int l = __ffsll((unsigned long long)past) - 1;
  const int i = idx - readlane(upto - own, l);
  if (i < 0) return it;  // (token_start out of order, so far that sums of a plan pass 2^31)
  it.found = true;
  it.b = b0 + l;
  it.s0 = readlane(q.s0, l);
  it.n = readlane(q.n, l);
  it.pos0 = readlane(q.pos0, l);
  it.end = readlane(q.end, l);
  it.lo = readlane(q.lo, l);
  it.splits = readlane(splits, l);
  // the last tiles of a prompt see the most positions: they go first
  // (divisions of uniform values are vector instructions: their results are made uniform again)
  const int back = SPLIT ? i : uniform(i / it.splits);
  it.tile = readlane(q.tiles, l) - 1 - back;
  it.split = SPLIT ? 0 : i - back * it.splits;
  it.rec = readlane(rupto - rec, l) + it.tile * it.splits;
  return it;
}

// The positions that an item's rows j0 .. j1 (tokens) can see within its range.
struct Span {
  int lo, hi;          // lo a multiple of kUnit
  int all_lo, all_hi;  // positions that every row sees
};
template <bool TILE>
__device__ __forceinline__ Span span_of(const Item& it, int j0, int j1, int window) {
  Span s;
  const int first = it.pos0 + j0, last = it.pos0 + j1;
  const int lo = window > 0 ? max(first - window + 1, 0) & -kUnit : 0;
  s.hi = min(last + 1, it.end);
  if constexpr (TILE) {
    s.lo = lo;
    if (it.splits > 1) {
      const int units = (max(s.hi - lo, 0) + kUnit - 1) / kUnit;
      const int range = uniform((units + it.splits - 1) / it.splits) * kUnit;
      s.lo = lo + it.split * range;  // (below hi + splits * kUnit)
      s.hi = min(s.hi, s.lo + range);
    }
  } else {
    s.lo = max(lo, it.lo + it.split * it.chunk * kUnit);
    if (it.split + 1 < it.splits) s.hi = min(s.hi, it.lo + (it.split + 1) * it.chunk * kUnit);
  }
  s.all_lo = window > 0 ? max(last - window + 1, 0) : 0;
  s.all_hi = min(first + 1, it.end);
  return s;
}

// Sixteen positions from t on (t a multiple of 16, in one page) of one head of a
// cache whose elements take BYTES, in bytes from the head's first row: rows from
// `end` on, and all rows of a page that is not there, lie past the extent and
// read as zeros.  Scalar arithmetic without branches: it stands before every
// tile's loads (page and slot strides are below 2^32 bytes, so the products are
// 32 x 32 -> 64 bits).
struct Rows16 {
  uint64_t at;
  uint32_t bytes;
};
template <int BYTES>
__device__ __forceinline__ Rows16 rows16(const PagedBatch& pb, int page, int t, int end) {
  const uint32_t there = ((unsigned)page < (unsigned)pb.num_pages) & (t < end);
  const uint32_t slot = (uint32_t)t & ((1u << pb.page_shift) - 1);
  const uint32_t slot_bytes = (uint32_t)pb.slot_stride * BYTES;
  Rows16 r;
  r.at = ((uint64_t)(uint32_t)page * pb.page_bytes + (uint64_t)slot * slot_bytes) & -(uint64_t)there;
  r.bytes = ((uint32_t)(min(end - t, 16) - 1) * slot_bytes + kHeadDim * BYTES) & -there;
  return r;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const char* head, const Rows16& r) {
  return rsrc(head + r.at, r.bytes);
}

// Bits of the halves of x that are infinite or NaN: 0x8000 in each.
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return ((x & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t x) { return x & ~((not_finite(x) >> 15) * 0xFFFFu); }
__device__ __forceinline__ u32x4 finite_or_zero(u32x4 x) {
  return u32x4{finite_or_zero(x.x), finite_or_zero(x.y), finite_or_zero(x.z), finite_or_zero(x.w)};
}
__device__ __forceinline__ uint32_t not_finite(u32x4 x) {
  return not_finite(x.x) | not_finite(x.y) | not_finite(x.z) | not_finite(x.w);
}

// Codes in e4m3, four of a word, whose value is code * scale, scale a power of
// two that the position's block has (an e8m0 byte, 2^(byte - 127), taken into
// 112..134: from 2^-15 to 2^7, within which every value is an fp16 one and the
// conversion exact).
__device__ __forceinline__ float block_scale(int byte) {
  return __builtin_bit_cast(float, min(max(byte, 112), 134) << 23);
}
// (Whole words, not their elements: extracting the upper element of the result
// compiles to a copy of the lower one.)
__device__ __forceinline__ uint32_t values01(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false));
}
__device__ __forceinline__ uint32_t values23(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true));
}
// The bytes of x that are NaN (0x7F or 0xFF): 0x80 in each.
__device__ __forceinline__ uint32_t nan_codes(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t number_codes(uint32_t x) { return x & ~((nan_codes(x) >> 7) * 0xFFu); }

// ---------------------------------------------------------------------------
// attention of prompts' chunks: the matrix cores bound it
// ---------------------------------------------------------------------------

// A block of eight or four waves holds the query rows of one item, 32 a wave, and
// walks the positions in tiles of 64.  Scores are formed transposed, keys (rows) x
// queries (columns), so that a lane holds 32 scores of one query: the running
// maximum and the denominator need one exchange between the two halves of the
// wave, and the probabilities are already the second product's operand
// (columns: queries) in the order in which the transposing LDS reads deliver
// the values (lane half h: positions 16 s + 4 h .. + 3 and 8 further).
//
// Probabilities are rounded to fp16 for the matrix cores (half a step: 2^-11
// of each, their errors independent).  They are 2^8 times exp(score - ref),
// where the reference ref only follows the maximum once that has grown by more
// than 2^7: so they stay below 2^15 and full precision reaches down to 2^-22
// of the largest, and the value sums are rarely rescaled.  The denominator is
// the fp32 sum of the unrounded ones.  (As two fp16 numbers each, with twice the
// value products, outputs are as near to 64-bit ones as those of fp32
// probabilities: two prompts of 8192 and 4001 rows over codes, 0.000135 of their
// norm instead of 0.000151, where the rounding of the output alone makes most of
// either; they then take 877 us instead of 707, over fp16 caches 988 instead of 751.)
// A sequence of up to 16 rows (decoding rows beside a chunk, or of a batch with
// much padding) would fill half a wave's rows: the block takes its items as the
// 16-row kernel does, with its probabilities and all waves along the positions.
// Its records have the place of a block's rows.  (Measured on MI355X: a
// chunk beside 15 decoding rows 77.8 -> 78.2 us; two waves more for the
// probabilities' remainders instead, 84.8.)
//
// What bounds it: the issue of matrix and vector instructions by two waves a
// SIMD that do little of the one while the other does the other.  (Counters of
// two prompts of 8192 and 4001 rows, 32:8 heads, on MI355X, fp16 caches and codes:
// matrix instructions 43 and 41 % of the SIMDs' cycles, vector instructions 43 and
// 51 %; LDS active 27 and 31 % of the compute units' cycles.  Kernel alone, without
// the joining, under a kernel trace: 788 and 728 us, the medians of 24 calls, 761
// and 706 the shortest; a call with the joining, untraced, 751 and 707, 907 and 963
// TFLOP/s; a library's fp16 8192^3 product reaches 1150.  Earlier, fp16, where the
// kernel alone took 874: as two blocks of 128 rows, with
// twice the staging instructions, 945; with 128 rows a tile took a wave
// about 5000 cycles: 1400 to 2100 its scores, 240 the maximum, 700 the
// exponentials, 850 the value sums, 1100 issuing the next tile's loads and
// stores.  Not faster: the two waves of a SIMD kept a phase apart, the operands
// of a tile's scores requested at once.)
//
// Tiles of keys and values go memory -> registers -> LDS, two buffers, so that
// a tile's loads are in flight while the one before is computed and a block
// meets once per tile.  Piece p (16 bytes) of key row r sits at p ^ (r & 15)
// and of value row r at p ^ 4 (r & 3): the operand reads touch each bank once.
constexpr int kTile = 64;
constexpr int kTileBytes = kTile * kHeadDim * 2;
template <class C, int WAVES>
constexpr int kChunkLds = std::max(4 * kTileBytes + 64, C::template kItemLds<WAVES>);
constexpr float kProbLog2 = 8.0f, kLagLog2 = 7.0f;
constexpr float kFarLog2 = 65536.0f;

// C: the type of cache: C::Batch, the bytes of an element C::kBytes (2: fp16, 1:
// e4m3 codes, which become fp16 on their way to LDS), and rows16_item, the way
// of items of up to 16 rows, with the LDS that its waves need.
template <class C, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void paged_attention_chunk_kernel(typename C::Batch pb,
                                                                              const uint16_t* __restrict__ q, int R,
                                                                              int Hkv, int window, Out o_) {
  constexpr int kLargeRows = kChunkRows<WAVES>, kThreads = 64 * WAVES;
  constexpr bool kCodes = C::kBytes == 1;
  extern __shared__ u32x4 large_lds[];
  char* const lds = reinterpret_cast<char*>(large_lds);
  int* const flags = reinterpret_cast<int*>(lds + 4 * kTileBytes);  // [4]: tile (& 3) whose values are not all finite
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = uniform(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<kLargeRows, C::kTileRanges, false>(pb, o_, at_item, R, Hkv, window, lane);
  if (!it.found) return;
  if (it.n * R <= kSmallRows) {
    C::template rows16_item<WAVES, kLargeRows>(pb, q, R, window, o_, it, g, lds);
    return;
  }
  const int r0 = it.tile * kLargeRows;
  const int rows = min(it.n * R - r0, kLargeRows);
  const Span sp = span_of<C::kTileRanges>(it, uniform(r0 / R), uniform((r0 + rows - 1) / R), window);

  // This lane's query row and what it sees; its operand: dimensions 16 s + 8 h .. + 7.
  const int my = 32 * w + n;
  const bool live = my < rows;
  const int token = (r0 + min(my, rows - 1)) / R;
  const int64_t qrow = (int64_t)(it.s0 + token) * o_.Hq + g * R + (r0 + min(my, rows - 1)) % R;
  const int pos = it.pos0 + token;
  const int see_hi = live ? min(pos + 1, it.end) : 0;
  const int see_lo = window > 0 ? pos - window + 1 : 0;
  // Tiles beyond these no row of the wave sees.
  int wave_lo, wave_hi;
  {
    const int j0 = uniform((r0 + min(32 * w, rows - 1)) / R), j1 = uniform((r0 + min(32 * w + 31, rows - 1)) / R);
    wave_lo = window > 0 ? it.pos0 + j0 - window + 1 : 0;
    wave_hi = 32 * w < rows ? it.pos0 + j1 + 1 : 0;
  }
  half8_t qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const half8_t*>(q + qrow * kHeadDim + 16 * s + 8 * h);

  const int* const table = pb.page_table + it.b * pb.table_stride;
  const char* const khead = reinterpret_cast<const char*>(pb.k) + g * pb.head_stride * C::kBytes;
  const char* const vhead = reinterpret_cast<const char*>(pb.v) + g * pb.head_stride * C::kBytes;
  // Where the groups of 16 positions lie, 64 groups (16 tiles) at a time: a
  // lane computes a group's byte offset from the head's first row, and the
  // mask says which pages are there; a tile's loads then cost a few scalar
  // instructions.  Two sets are held: rows are loaded two tiles before they
  // are computed.
  constexpr int kSet = 16;  // tiles
  uint32_t set_lo = 0, set_hi = 0, old_lo = 0, old_hi = 0;
  uint64_t set_there = 0, old_there = 0;
  int set_ks = 0, set_vs = 0, old_ks = 0, old_vs = 0;  // codes: the groups' scales
  int set_first = 0;  // its first tile; the set before covers the kSet tiles before that
  auto next_set = [&](int t) {
    old_lo = set_lo, old_hi = set_hi, old_there = set_there;
    const int at = sp.lo + t * kTile + 16 * lane;
    const int page = at < sp.hi ? table[at >> pb.page_shift] : -1;
    const bool there = (unsigned)page < (unsigned)pb.num_pages;
    const uint64_t off = (uint64_t)(uint32_t)page * pb.page_bytes +
                         (uint64_t)((uint32_t)at & ((1u << pb.page_shift) - 1)) * (uint32_t)(pb.slot_stride * C::kBytes);
    set_lo = there ? (uint32_t)off : 0;
    set_hi = there ? (uint32_t)(off >> 32) : 0;
    set_there = __ballot(there);
    set_first = t;
    if constexpr (kCodes) {
      old_ks = set_ks, old_vs = set_vs;
      if (there) {
        const int64_t i = pb.scale_at(page, g, at);
        set_ks = pb.k_scales[i], set_vs = pb.v_scales[i];
      }
    }
  };

  // Staging: thread (row tid / 16 of each half of the tile, piece tid % 16);
  // a wave's rows of a half lie in one group of 16.
  // (codes: row tid / 8, piece tid % 8, of 16 bytes that become two pieces)
  constexpr int kLoads = kTile * 8 * C::kBytes / kThreads;
  constexpr int kPass = kTile / kLoads;  // rows that a load takes, of all waves
  const int sr = kCodes ? tid >> 3 : tid >> 4, spc = kCodes ? tid & 7 : tid & 15;
  const uint32_t src_at = (uint32_t)(sr & 15) * pb.slot_stride * C::kBytes + 16 * spc;
  u32x4 kreg[kLoads], vreg[kLoads];
  // Groups of tile t whose page is not there, for the tiles of the two sets.
  auto bad_of = [&](int t) {
    const int i = (t - set_first) & (kSet - 1);
    return (int)(~(t >= set_first ? set_there : old_there) >> 4 * i) & 15;
  };
  auto group_of = [&](int i) { return kPass / 16 * i + (kCodes ? w >> 1 : w >> 2); };  // of 16 rows, that load i is in
  auto load_rows = [&](u32x4(&r)[kLoads], const char* head, int t) {
    const int i0 = (t - set_first) & (kSet - 1);
    const bool now = t >= set_first;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int gr = group_of(i), l = 4 * i0 + gr;
      const uint32_t lo = readlane((int)(now ? set_lo : old_lo), l), hi = readlane((int)(now ? set_hi : old_hi), l);
      const uint32_t there = (uint32_t)((now ? set_there : old_there) >> l) & 1;
      const int left = sp.hi - (sp.lo + t * kTile + 16 * gr);  // (a page that is there has a row)
      Rows16 at;
      at.at = (uint64_t)hi << 32 | lo;
      at.bytes = ((uint32_t)(min(left, 16) - 1) * (uint32_t)(pb.slot_stride * C::kBytes) + kHeadDim * C::kBytes) & -there;
      r[i] = __builtin_amdgcn_raw_buffer_load_b128(rows_of(head, at), src_at, 0, 0);
    }
  };
  auto load_keys = [&](int t) {
    if (t - set_first >= kSet) next_set(t);
    load_rows(kreg, khead, t);
  };
  auto load_values = [&](int t) { load_rows(vreg, vhead, t); };
  // Tiles that every row of the block sees whole: first .. last - 1.
  const int whole_first = (max(sp.all_lo - sp.lo, 0) + kTile - 1) / kTile;
  const int whole_last = max(min(sp.all_hi, sp.hi) - sp.lo, 0) / kTile;
  auto is_masked = [&](int t) { return (bad_of(t) != 0) | (t < whole_first) | (t >= whole_last); };
  // Codes of a row to LDS as two pieces of fp16, whose places go by XOR with `swap`.
  // (Two lanes' stores meet in a bank; with half of the lanes beginning at the odd
  // piece none do, but the selects cost as much.)
  auto store_codes = [&](char* d, int row, const u32x4& r, float scale, int swap) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = i ? r.z : r.x, b = i ? r.w : r.y;
      *reinterpret_cast<u32x4*>(d + row * 256 + 16 * ((2 * spc + i) ^ swap)) =
          u32x4{values01(a, scale), values23(a, scale), values01(b, scale), values23(b, scale)};
    }
  };
  auto scale_of = [&](int now, int old, int t, int i) {
    const int l = 4 * ((t - set_first) & (kSet - 1)) + group_of(i);
    return block_scale(readlane(t >= set_first ? now : old, l));
  };
  auto store_keys = [&](int t) {
    char* const d = lds + (t & 1) * 2 * kTileBytes;
    if constexpr (kCodes) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) store_codes(d, kPass * i + sr, kreg[i], scale_of(set_ks, old_ks, t, i), sr & 15);
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      *reinterpret_cast<u32x4*>(d + (kPass * i + sr) * 256 + 16 * (spc ^ (sr & 15))) = kreg[i];
  };
  // Values that are infinite or NaN stay out of masked tiles: 0 times one is NaN.
  auto store_values = [&](int t) {
    char* const d = lds + (t & 1) * 2 * kTileBytes + kTileBytes;
    if constexpr (kCodes) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        u32x4 r = vreg[i];
        if (is_masked(t)) {
          if (nan_codes(r.x) | nan_codes(r.y) | nan_codes(r.z) | nan_codes(r.w)) flags[t & 3] = t;
          r = u32x4{number_codes(r.x), number_codes(r.y), number_codes(r.z), number_codes(r.w)};
        }
        store_codes(d, kPass * i + sr, r, scale_of(set_vs, old_vs, t, i), 4 * (sr & 3));
      }
      return;
    }
    if (is_masked(t)) {
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) bad |= not_finite(vreg[i]);
      if (bad) flags[t & 3] = t;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) vreg[i] = finite_or_zero(vreg[i]);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      *reinterpret_cast<u32x4*>(d + (kPass * i + sr) * 256 + 16 * (spc ^ (4 * (sr & 3)))) = vreg[i];
  };

  float ref = kNoMax, l = 0.0f;
  float16_t o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;

  // Scores of a tile: keys from buffer B.
  auto scores = [&](float16_t(&s)[2], int B) {
    const char* const kd = lds + B * 2 * kTileBytes;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt][r] = 0.0f;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const half8_t a = *reinterpret_cast<const half8_t*>(kd + (32 * kt + n) * 256 + 16 * ((2 * ks + h) ^ (n & 15)));
        s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, qf[ks], s[kt], 0, 0, 0);
      }
  };
  auto mask = [&](float16_t(&s)[2], int t0, int bad_groups) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int at = t0 + 32 * kt + 8 * (r >> 2) + 4 * h + (r & 3);
        const bool there = !(bad_groups >> (2 * kt + (r >> 3)) & 1) & (at < sp.hi);
        s[kt][r] = (there & (at >= see_lo) & (at < see_hi)) ? s[kt][r] : -INFINITY;
      }
  };
  // The reference follows the scores that are used next; sums so far are
  // rescaled.  A probability's exponent is then scale x s + bias, fused.  Past
  // |ref| = kFarLog2 a score's scaled value is rounded before ref is subtracted
  // from it: fused, the difference keeps the rounding of ref alone, up to half a
  // step of it (2^12 at the largest scores of fp16 inputs, where ref is 2^36:
  // probabilities would be infinite).  Rounded alike, the largest score is ref.
  uint64_t far_rows = 0;  // lanes of which that is so
  float bias, scale;
  auto follow = [&](float16_t(&s)[2]) {
#pragma clang fp contract(off)
    float m4[4];  // four chains
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m4[i] = maximum(s[0][i], s[1][i]);
#pragma unroll
      for (int r = 4; r < 16; r += 4) m4[i] = maximum(maximum(m4[i], s[0][r + i]), s[1][r + i]);
    }
    float mx = maximum(maximum(m4[0], m4[1]), maximum(m4[2], m4[3]));  // (of a row with a NaN score all is NaN)
    auto x = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, mx), __builtin_bit_cast(uint32_t, mx), false,
                                              false);
    mx = maximum(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1])) * kScaleLog2;
    // (the difference, which is exact where they are near: ref + 7 may be rounded to ref + 8)
    const bool ahead = mx - ref > kLagLog2;
    scale = kScaleLog2;
    if (__ballot(ahead) | far_rows) {
      const float mn = ahead ? mx : ref;  // each query by itself: no row depends on its neighbours
      const float alpha = __builtin_amdgcn_exp2f(ref - mn);
      ref = mn;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      const bool far = fabsf(ref) > kFarLog2 && ref != kNoMax;
      far_rows = __ballot(far);
      if (far_rows) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float scaled = s[kt][r] * kScaleLog2;
            s[kt][r] = far ? scaled - ref : s[kt][r];
          }
        scale = far ? 1.0f : kScaleLog2;
      }
    }
    bias = kProbLog2 - (scale == 1.0f ? 0.0f : ref);
  };
  auto probabilities = [&](half8_t(&pf)[4], const float16_t(&s)[2]) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fmaf(s[kt][r + i], scale, bias);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(p[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += p[i];
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const half2_t pk = __builtin_convertvector((float2_t{p[i], p[i + 1]}), half2_t);
          pf[2 * kt + (r >> 3)][(r & 7) + i] = pk[0];
          pf[2 * kt + (r >> 3)][(r & 7) + i + 1] = pk[1];
        }
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  // Value sums: 16 lanes read 4 positions x 16 dimensions and receive a column each.
  const int vrow = 4 * h + (lane & 15) / 4;
  const int vcol = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);  // dimension within 32
  auto value_sums = [&](const half8_t(&pf)[4], int B) {
    typedef short short4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4_t lds_short4;
    const char* const vd = lds + B * 2 * kTileBytes + kTileBytes;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const int piece = (32 * d + vcol) >> 3;
        const char* const a = vd + (16 * ks + vrow) * 256 + 16 * (piece ^ (4 * (vrow & 3))) + 2 * (vcol & 7);
        const short4_t x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(a));
        const short4_t x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(a + 8 * 256));
        const half8_t v = __builtin_bit_cast(half8_t, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pf[ks], o[d], 0, 0, 0);
      }
  };
  // The rows that see a value that was left out receive it here, from memory,
  // whatever its weight (the result is infinite or NaN).
  auto add_not_finite = [&](int t) {
    typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
#pragma unroll 1
    for (int i = 0; i < kTile; ++i) {
      const int at = sp.lo + t * kTile + i;
      if (at >= sp.hi) break;
      const int page = table[at >> pb.page_shift];
      if ((unsigned)page >= (unsigned)pb.num_pages) continue;
      const char* const row = vhead + (int64_t)page * pb.page_bytes +
                              (int64_t)(at & ((1 << pb.page_shift) - 1)) * pb.slot_stride * C::kBytes;
      const bool sees = (at >= see_lo) & (at < see_hi);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          if constexpr (kCodes) {
            const uint32_t x = nan_codes(*reinterpret_cast<const uint32_t*>(row + 32 * d + 2 * r + 4 * h));
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][r + e] += sees && (x >> (8 * e + 7) & 1) ? __builtin_nanf("") : 0.0f;
            continue;
          }
          const half4_t x = *reinterpret_cast<const half4_t*>(row + (32 * d + 2 * r + 4 * h) * 2);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float add = fabsf((float)x[e]) < INFINITY ? 0.0f : (float)x[e];
            o[d][r + e] += sees ? add : 0.0f;
          }
        }
    }
  };

  const int tiles = sp.hi > sp.lo ? (sp.hi - sp.lo + kTile - 1) / kTile : 0;
  // Tiles of which some row of the wave sees something.
  const int want_first = max(wave_lo - sp.lo, 0) / kTile;
  const int want_last = min(tiles, (max(wave_hi - sp.lo, 0) + kTile - 1) / kTile);
  auto wanted = [&](int t) { return (t >= want_first) & (t < want_last); };
  float16_t s[2];
  half8_t pf[4];
  if (tid < 4) flags[tid] = -1;
  if (tiles > 0) {
    next_set(0);
    load_keys(0);
    load_values(0);
    __syncthreads();
    store_keys(0);
    store_values(0);
    if (tiles > 1) load_keys(1), load_values(1);
    __syncthreads();
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
      if (t + 1 < tiles) store_keys(t + 1), store_values(t + 1);
      if (t + 2 < tiles) load_keys(t + 2), load_values(t + 2);
      if (wanted(t)) {
        scores(s, t & 1);
        if (is_masked(t)) mask(s, sp.lo + t * kTile, bad_of(t));
        follow(s);
        probabilities(pf, s);
        value_sums(pf, t & 1);
        if (uniform(flags[t & 3]) == t) add_not_finite(t);
      }
      __syncthreads();
    }
  }
  // the two halves of the wave hold different positions' parts of the denominator
  {
    auto x = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, l), __builtin_bit_cast(uint32_t, l), false,
                                              false);
    l = __builtin_bit_cast(float, (uint32_t)x[0]) + __builtin_bit_cast(float, (uint32_t)x[1]);
  }
  if (!live) return;
  if (it.splits > 1) {
    const int rec = it.rec + it.split;
    if (rec >= o_.rec_bound) return;  // token_start out of order
    float* const wp = o_.ws + ((int64_t)g * o_.rec_bound + rec) * (kLargeRows * (kHeadDim + 2));
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4_t*>(wp + my * kHeadDim + 32 * d + 2 * r + 4 * h) =
            float4_t{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
    if (h == 0) {
      wp[kLargeRows * kHeadDim + 2 * my] = ref;
      wp[kLargeRows * kHeadDim + 2 * my + 1] = l;
    }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* const dst = o_.out + qrow * kHeadDim;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
      *reinterpret_cast<half4_t*>(dst + 32 * d + 2 * r + 4 * h) =
          half4_t{(_Float16)(o[d][r] * inv), (_Float16)(o[d][r + 1] * inv), (_Float16)(o[d][r + 2] * inv),
                  (_Float16)(o[d][r + 3] * inv)};
    }
}

// Joins the ranges of the split tiles in position order.  Records are weighted
// by 2^(their maximum - the largest of all); a lane holds two dimensions.
// WAVES == 4: a block takes a row (ONE) or every gridDim.y-th of its tile, its
// waves every fourth record, and they meet in LDS (decoding: few rows, many
// ranges).  WAVES == 1: a wave per kJoinRows rows, four times that a block at a
// time (a chunk's rows have few ranges each).  Most blocks
// of the grid can find nothing to do and cost their search, so there are about
// kJoinBlocks of them, which go on to further rows.  (Measured on MI355X: two
// prompts whose tiles are not split, 16.4 -> 4.9 us.)  A wave of two rows and two
// records at a time takes few registers, so that all blocks run at once.  (Calls
// over codes, 4 rows and 4 records a wave -> 4 and 2 -> 2 and 2 -> 1 and 4: a chunk
// of 500 rows beside 15 decoding ones, 40:8 heads, 68.5 -> 65.2 -> 63.6, 66.0 ->
// 61.2 -> 62.7; 1024 rows at 0, 32:8, 41 -> 36 -> 34 -> 38; 512 at 2000, 64:8, 72 ->
// 68 -> 65 -> 68.  Twice the blocks: 63.0, 34.7 and 64.9.)
constexpr int kJoinRows = 2;
template <int BM, bool TILE, int WAVES, bool ONE>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(PagedBatch pb, int R, int Hkv, int window, Out o_) {
  __shared__ float2_t part[4][64];
  constexpr int kRec = BM * (kHeadDim + 2);
  constexpr int kRows = WAVES == 4 ? 1 : kJoinRows;  // rows of a wave
  constexpr int kB = WAVES == 4 ? 8 : 2;             // records loaded at a time
  const int lane = threadIdx.x & 63;
  const int w = uniform(threadIdx.x >> 6);
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<BM, TILE, true>(pb, o_, at_item, R, Hkv, window, lane);
  if (!it.found || it.rec + it.splits > o_.rec_bound) return;
  const int r0 = it.tile * BM;
  const int rows = min(it.n * R - r0, BM);
  const int first = WAVES == 4 ? w : 0;
  const float* const base = o_.ws + ((int64_t)g * o_.rec_bound + it.rec) * kRec;
  // WAVES == 4: every gridDim.y-th row, the same for the whole block; else group of 4 kRows
#pragma unroll 1
  for (int row = WAVES == 4 ? blockIdx.y : (blockIdx.y * 4 + w) * kRows; row < rows; row += (WAVES == 4 ? 1 : 4 * kRows) * gridDim.y) {
    const float *stat[kRows], *sums[kRows];
    float2_t x[kRows][kB], st[kRows][kB], num[kRows];
    float M[kRows], den[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int r = min(row + k, rows - 1);
      stat[k] = base + BM * kHeadDim + 2 * r;
      sums[k] = base + r * kHeadDim + 2 * lane;
      num[k] = float2_t{0.0f, 0.0f};
      M[k] = kNoMax, den[k] = 0.0f;
    }
    auto load = [&](int s0) {
#pragma unroll
      for (int k = 0; k < kRows; ++k)
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const int64_t s = min(s0 + WAVES * i, it.splits - 1);
          st[k][i] = *reinterpret_cast<const float2_t*>(stat[k] + s * kRec);
          x[k][i] = *reinterpret_cast<const float2_t*>(sums[k] + s * kRec);
        }
    };
    load(first);  // before the statistics: up to WAVES * kB ranges cost one memory round trip
    auto over_rows = [](float v, auto&& op) {  // of a value per 16-lane row
      const int u = __builtin_bit_cast(int, v);
      auto f = [](int x) { return __builtin_bit_cast(float, x); };
      return op(op(f(readlane(u, 0)), f(readlane(u, 16))), op(f(readlane(u, 32)), f(readlane(u, 48))));
    };
    for (int s0 = 0; s0 < it.splits; s0 += 64) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int s = s0 + lane;
        const float2_t y = *reinterpret_cast<const float2_t*>(stat[k] + (int64_t)min(s, it.splits - 1) * kRec);
        const float top = fmaxf(M[k], over_rows(row_max(y[0]), [](float a, float b) { return fmaxf(a, b); }));
        const float sum = over_rows(row_sum(s < it.splits ? __builtin_amdgcn_exp2f(y[0] - top) * y[1] : 0.0f),
                                    [](float a, float b) { return a + b; });
        den[k] = fmaf(den[k], __builtin_amdgcn_exp2f(M[k] - top), sum);
        M[k] = top;
      }
    }
    for (int s0 = first; s0 < it.splits; s0 += WAVES * kB) {
      if (s0 > first) load(s0);
#pragma unroll
      for (int k = 0; k < kRows; ++k)
#pragma unroll
        for (int i = 0; i < kB; ++i) {
          const bool in = s0 + WAVES * i < it.splits;  // else the last record again: its sums may be infinite
          const float e = in ? __builtin_amdgcn_exp2f(st[k][i][0] - M[k]) : 0.0f;
          num[k][0] = fmaf(e, in ? x[k][i][0] : 0.0f, num[k][0]);
          num[k][1] = fmaf(e, in ? x[k][i][1] : 0.0f, num[k][1]);
        }
    }
    if constexpr (WAVES == 4) {
      part[w][lane] = num[0];
      __syncthreads();
      if (ONE && w > 0) return;
      num[0] = part[0][lane];
#pragma unroll
      for (int i = 1; i < 4; ++i) num[0] += part[i][lane];
      if constexpr (!ONE) {
        __syncthreads();  // the next row's sums take their place
        if (w > 0) continue;
      }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if (row + k >= rows) break;
      const int r = r0 + row + k;
      const float inv = den[k] == 0.0f ? 0.0f : 1.0f / den[k];
      *reinterpret_cast<half2_t*>(o_.out + ((int64_t)(it.s0 + r / R) * o_.Hq + g * R + r % R) * kHeadDim + 2 * lane) =
          half2_t{(_Float16)(num[k][0] * inv), (_Float16)(num[k][1] * inv)};
    }
    if constexpr (ONE) return;  // (known before: a loop's code costs a row 1.6 to 3 us more)
  }
}

// Which kernel takes a batch, and its bounds: a pure function of the sizes.
struct AttentionPlan {
  int rows;  // of a block: 16, or the chunks' kernel
  int64_t items, split_tiles, records;  // per key/value head
  int64_t most_ranges;                  // of a tile, by the capacity
  int64_t floats;                       // workspace: the records, then the plan
  int64_t plan_at;
  int min_chunk;
};

// split_from: units a sequence must be able to have for any to be split.
template <int BM>
AttentionPlan plan_of(int64_t B, int64_t T, int64_t R, int64_t Hkv, int64_t capacity, int split_from) {
  AttentionPlan p;
  p.rows = BM;
  const int64_t tiles = (T * R + std::min(B, T) * (BM - 1)) / BM;
  const int64_t per_head = (kItems + Hkv - 1) / Hkv;
  // (with kItems heads and more a head's share of the items is one: no sequence is split)
  const bool split = capacity > (int64_t)std::max(kMinChunk<BM>, split_from) * kUnit && Hkv < kItems;
  p.min_chunk = split ? kMinChunk<BM> : std::max((int)((capacity + kUnit - 1) / kUnit), kMinChunk<BM>);
  p.items = tiles + (split ? per_head : 0);
  p.split_tiles = split ? std::min(per_head, tiles) : 0;
  const int64_t most = (capacity + kMinChunk<BM> * kUnit - 1) / (kMinChunk<BM> * kUnit);
  p.most_ranges = most;
  p.records = split ? std::min(2 * kItems / Hkv, tiles * most) : 0;
  p.plan_at = p.records * Hkv * BM * (kHeadDim + 2);
  p.floats = p.plan_at + (B > kGroup ? 1 + 3 * plan_groups(B) : 0);
  return p;
}

// Up to 16 rows per sequence on average go to the 16-row kernel.  (Measured on
// MI355X, 16-row -> 256-row kernel at twice and four times that: 32:8 heads, one
// sequence of 6000, 20 -> 14.5 and 25 -> 16 us; eight of 2000, 35 -> 29 and 52 ->
// 34; 64:8, four of 8000, 47 -> 43 and 75 -> 51; but one of 500, 12 -> 15.  Where
// sequences are of unequal size, at the border, 32:8: 63 decoding rows beside a
// chunk of 193 rows, all at 500 or at 2000, 67 -> 82 and 161 -> 189; a chunk of 256
// rows at 6000 beside 63 waiting sequences 180 -> 119, of 16 rows 30 -> 42; 64
// decoding rows and 193 of padding 98 -> 97, 16 and 49 of padding 35 -> 38.)
//
// C::four_waves: chunks whose blocks of 256 rows are few take blocks of 128.
template <class C>
AttentionPlan attention_plan(int64_t B, int64_t T, int64_t R, int64_t Hkv, int64_t capacity) {
  const int split_from = C::split_from(B, Hkv);
  if (T * R <= kSmallRows * B) return plan_of<kSmallRows>(B, T, R, Hkv, capacity, split_from);
  if (C::four_waves(T * R * Hkv)) return plan_of<kChunkRows<4>>(B, T, R, Hkv, capacity, split_from);
  return plan_of<kChunkRows<8>>(B, T, R, Hkv, capacity, split_from);
}

// Up to 16 rows per tile: an item a block.
constexpr int kWaves = 4;
template <class C>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_rows16_kernel(typename C::Batch pb,
                                                                             const uint16_t* __restrict__ q, int R,
                                                                             int Hkv, int window, Out o_) {
  extern __shared__ u32x4 small_lds[];
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<kSmallRows, C::kTileRanges, false>(pb, o_, at_item, R, Hkv, window, threadIdx.x & 63);
  if (!it.found) return;
  C::template rows16_item<kWaves, kSmallRows>(pb, q, R, window, o_, it, g, reinterpret_cast<char*>(small_lds));
}

template <class C, int BM>
void launch_chunks(const typename C::Batch& pb, const uint16_t* q, int64_t R, int64_t Hkv, int64_t window, const Out& o,
                   dim3 grid, dim3 join, bool by_group, hipStream_t stream, const LaunchEvents& e1, const LaunchEvents& e2) {
  const PagedBatch& rows = pb;
  constexpr int kWavesOf = BM / 32;
  launch((paged_attention_chunk_kernel<C, kWavesOf>), grid, dim3(64 * kWavesOf), kChunkLds<C, kWavesOf>, stream, e1, pb, q,
         (int)R, (int)Hkv, (int)window, o);
  if (join.x == 0) return;
  if (by_group)
    launch((paged_attention_join_kernel<BM, C::kTileRanges, 1, false>), join, dim3(256), 0, stream, e2, rows, (int)R, (int)Hkv, (int)window, o);
  else
    launch((paged_attention_join_kernel<BM, C::kTileRanges, 4, true>), join, dim3(256), 0, stream, e2, rows, (int)R, (int)Hkv, (int)window, o);
}

template <class C>
hipError_t launch_attention(const typename C::Batch& pb, const uint16_t* q, int64_t Hq, int64_t Hkv, int64_t window,
                            uint16_t* out, float* ws, hipStream_t stream, const LaunchEvents& ev) {
  const PagedBatch& rows = pb;
  const int64_t R = Hq / Hkv;
  const AttentionPlan p = attention_plan<C>(pb.B, pb.T, R, Hkv, (int64_t)pb.table_pages << pb.page_shift);
  LaunchEvents e0, e1 = ev, e2;
  if (p.split_tiles > 0) {  // the measurement hook spans all kernels
    e1.stop = nullptr;
    e2.stop = ev.stop;
  }
  int* const plan = reinterpret_cast<int*>(ws + p.plan_at);
  if (pb.B > kGroup) {
    e0.start = e1.start;
    e1.start = nullptr;
    auto* const kernel = p.rows == kSmallRows ? paged_attention_plan_kernel<kSmallRows, C::kTileRanges>
                         : p.rows == kChunkRows<4> ? paged_attention_plan_kernel<kChunkRows<4>, C::kTileRanges>
                                              : paged_attention_plan_kernel<kChunkRows<8>, C::kTileRanges>;
    launch(kernel, dim3(1), dim3(64 * kPlanWaves), 0, stream, e0, rows, (int)R, (int)Hkv, (int)window, p.min_chunk, plan);
  }
  const Out o{out, ws, plan, (int)Hq, (int)p.records, p.min_chunk};
  const dim3 grid((unsigned)(p.items * Hkv));
  // A block joins one row; 4 kJoinRows where the tiles (most of them not split)
  // would make many blocks.  (Calls measured on MI355X, 8:1 heads, by row -> by 8.
  // Tiles of 128 rows over codes: 9 of up to 3 ranges 19.1 -> 18.1 us, of up to 9, 20.8
  // -> 21.4, of up to 65, 33.1 -> 44.3; 16 of up to 9, 23.4 -> 22.8, of up to 17, 29.5
  // -> 31.7; 32 of up to 17, 35.9 -> 33.6.  Tiles of 256 over fp16: 8 of up to 9, 26.5
  // -> 25.8, of up to 65, 50.5 -> 59.3; 16 of up to 9, 33.1 -> 29.5; 32 of up to 9, 49.7
  // -> 40.0; 64 of up to 65, 197 -> 174: their border of 32 is above where the two
  // meet, and stays, as they add ranges up in unlike orders.)
  constexpr int64_t kJoinBlocks = 2048;
  const int64_t few_tiles = p.rows != kChunkRows<4> ? 32 : p.most_ranges >= 16 ? 16 : 8;
  const bool many = p.rows != kSmallRows && p.split_tiles * Hkv > few_tiles;
  const int64_t most_rows = std::min<int64_t>(p.rows, pb.T * R);
  const int64_t groups = (most_rows + 4 * kJoinRows - 1) / (4 * kJoinRows);
  const int64_t turns = (groups * (p.split_tiles * Hkv + 1) + kJoinBlocks - 1) / kJoinBlocks;
  const int64_t by_group = (groups + turns - 1) / turns;  // (as many turns for each)
  // 16-row tiles: a block a row, or fewer blocks that go on where there would be more
  // than run at once, unless rows fill at least half of up to twice as many: where a
  // tile has fewer rows than 16, or is not split, each block costs its search.
  // (Calls measured on MI355X, a block a row -> 2048 / tiles blocks a tile, decoding
  // sequences of 2000 positions, fp16 caches: 64 of four rows a head 99 -> 93 us, 24
  // 54.8 -> 52.7, 16 36.0 -> 35.6; of sixteen rows, 64 100.7 -> 94.2, 16 (half of the
  // blocks have a row) 41.0 -> 42.6.)  Chunks' tiles, few where they are joined by
  // rows: a block a row (of the same sizes, 200 rows at 900, 40:8 heads, 38.8 -> 42.0).
  const int64_t slots = most_rows * p.split_tiles * Hkv;
  const bool one = p.rows != kSmallRows || slots <= kJoinBlocks || (slots <= 2 * kJoinBlocks && 2 * pb.T * R * Hkv >= slots);
  const int64_t by_row = one ? most_rows : std::min(most_rows, std::max<int64_t>(1, kJoinBlocks / (p.split_tiles * Hkv + 1)));
  const dim3 join((unsigned)(p.split_tiles * Hkv), (unsigned)(many ? by_group : by_row));
  if (p.rows == kSmallRows) {
    launch((paged_attention_rows16_kernel<C>), grid, dim3(64 * kWaves), C::template kItemLds<kWaves>, stream, e1, pb, q,
           (int)R, (int)Hkv, (int)window, o);
    if (p.split_tiles > 0) {
      auto* const kernel = one ? paged_attention_join_kernel<kSmallRows, C::kTileRanges, 4, true>
                               : paged_attention_join_kernel<kSmallRows, C::kTileRanges, 4, false>;
      launch(kernel, join, dim3(256), 0, stream, e2, rows, (int)R, (int)Hkv, (int)window, o);
    }
  } else if (p.rows == kChunkRows<8>) {
    launch_chunks<C, kChunkRows<8>>(pb, q, R, Hkv, window, o, grid, join, many, stream, e1, e2);
  } else if constexpr (C::kFourWaves) {
    launch_chunks<C, kChunkRows<4>>(pb, q, R, Hkv, window, o, grid, join, many, stream, e1, e2);
  }
  return hipGetLastError();
}

}  // namespace

}  // namespace laq

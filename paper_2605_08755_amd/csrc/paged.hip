// Batched serving over paged key/value caches: per-head q/k RMSNorm with the
// rotary embedding and the append of new rows, and the attention of new rows
// (one per sequence when decoding, many in a prompt's chunk) over each
// sequence's pages.  fp16 in and out, fp32 sums and softmax statistics, fixed
// reduction orders (deterministic).  Head dimension 128.
//
// A batch of B sequences: sequence b owns rows token_start[b] ..
// token_start[b + 1] - 1, which are the last of its seq_len[b] positions;
// position t lies in page page_table[b][t / page_size].  These arrays live in
// device memory and the host never reads them, so a captured graph serves a
// growing batch.  Nothing read from them is trusted as an address: rows are
// clamped to 0 .. T, positions to the table's width, and a page outside the
// cache is a page that is not there.
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
// append
// ---------------------------------------------------------------------------

// A wave takes one row and every waves_per_row-th group of eight heads, eight
// lanes a head: lane i holds dimensions 8i .. 8i + 7 and their rotation partners 64
// further, so a head's two 128-byte halves are loaded and stored whole and the
// norm needs one sum over eight lanes.  What bounds it: the bytes of the rows
// in and out (measured on MI355X, 16384 rows, 32:8 heads: 84 us, 4.9 TB/s,
// a large copy moves 5.0); few rows are a launch and three dependent reads
// (16 rows: 3.7 us).  The row's table line is read once per wave.
// The row's sequence is found while its first loads are in flight: among the
// sequences' ends, which do not decrease, by 64 of them a step (up to 64
// sequences one step, 2^20 four).
__global__ __launch_bounds__(256) void paged_append_kernel(PagedBatch pb, const uint16_t* __restrict__ qkv,
                                                           int64_t qkv_stride, const uint16_t* __restrict__ qw,
                                                           const uint16_t* __restrict__ kw,
                                                           const float* __restrict__ cos_sin, int rope_rows, int Hq,
                                                           int Hkv, float eps, uint16_t* __restrict__ q_out,
                                                           int waves_per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
  const int row = uniform((int)(wave / waves_per_row));
  const int first = uniform((int)(wave - (int64_t)row * waves_per_row));
  if (row >= pb.T) return;
  const int i = lane & 7;
  const int H = Hq + 2 * Hkv;
  const int groups = (H + 7) >> 3;
  const uint16_t* const src = qkv + row * qkv_stride;

  auto load = [&](int grp, u32x4& a, u32x4& b) {
    const int h = min(grp * 8 + (lane >> 3), H - 1);
    const uint16_t* p = src + (int64_t)h * kHeadDim + 8 * i;
    a = *reinterpret_cast<const u32x4*>(p);
    b = *reinterpret_cast<const u32x4*>(p + 64);
  };
  u32x4 a, b;
  load(first, a, b);

  int seq = 0;  // sequences that end at or before the row
  for (int left = pb.B; left > 0;) {
    const int step = (left + 63) >> 6, last = (lane + 1) * step - 1;  // a lane's step sequences end with the last's end
    const bool before = last < left && pb.token_start[seq + last + 1] <= row;
    const int whole = __popcll(__ballot(before)) * step;
    seq += whole;
    left = min(step - 1, left - whole);
  }
  seq = uniform(seq);
  if (seq >= pb.B) return;  // behind the last sequence
  const int s0 = pb.token_start[seq], s1 = min(pb.token_start[seq + 1], pb.T);
  if (row < s0) return;     // before the first
  const int64_t pos = (int64_t)pb.seq_len[seq] - s1 + row;
  const int64_t cap = (int64_t)pb.table_pages << pb.page_shift;
  const bool placed = pos >= 0 && pos < cap && pos < rope_rows;
  int page = -1;
  if (placed) page = pb.page_table[seq * pb.table_stride + (pos >> pb.page_shift)];
  const bool keep = (unsigned)page < (unsigned)pb.num_pages;
  const int64_t slot = keep ? (int64_t)page * (pb.page_bytes / 2) + (pos & ((1LL << pb.page_shift) - 1)) * pb.slot_stride : 0;

  const float* const cs = cos_sin + (placed ? pos : 0) * kHeadDim + 8 * i;
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = cs[e], s[e] = cs[64 + e];

  for (int grp = first; grp < groups;) {
    const int h = grp * 8 + (lane >> 3);
    half8_t x = __builtin_bit_cast(half8_t, a), y = __builtin_bit_cast(half8_t, b);
    const u32x4 va = a, vb = b;
    const int next = grp + waves_per_row;
    if (next < groups) load(next, a, b);
    if (h < Hq + Hkv) {
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = (float)x[e], v[e] = (float)y[e];
      const uint16_t* const w = h < Hq ? qw : kw;
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(u[e], u[e], fmaf(v[e], v[e], ss));
      ss = sum8(ss);
      if (w != nullptr) {
        const float r = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + eps);
        const half8_t wa = *reinterpret_cast<const half8_t*>(w + 8 * i);
        const half8_t wb = *reinterpret_cast<const half8_t*>(w + 64 + 8 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = u[e] * r * (float)wa[e], v[e] = v[e] * r * (float)wb[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = (_Float16)(u[e] * c[e] - v[e] * s[e]);
        y[e] = (_Float16)(v[e] * c[e] + u[e] * s[e]);
      }
      if (h < Hq) {
        if (!placed) x = half8_t{}, y = half8_t{};
        uint16_t* d = q_out + ((int64_t)row * Hq + h) * kHeadDim + 8 * i;
        *reinterpret_cast<half8_t*>(d) = x;
        *reinterpret_cast<half8_t*>(d + 64) = y;
      } else if (keep) {
        uint16_t* d = pb.k + slot + (h - Hq) * pb.head_stride + 8 * i;
        *reinterpret_cast<half8_t*>(d) = x;
        *reinterpret_cast<half8_t*>(d + 64) = y;
      }
    } else if (h < H && keep) {
      uint16_t* d = pb.v + slot + (h - Hq - Hkv) * pb.head_stride + 8 * i;
      *reinterpret_cast<u32x4*>(d) = va;
      *reinterpret_cast<u32x4*>(d + 64) = vb;
    }
    grp = next;
  }
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
constexpr int kSmallRows = 16, kLargeRows = 256;
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

template <int BM>
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
    }
  }
  return q;
}

struct Item {
  bool found;
  int b, s0, n, pos0, end, lo;
  int tile, split, splits, chunk;
  int rec;  // first record of the tile's ranges
};

// The smallest chunk by that bound, of all sequences' tiles x units.
template <int BM>
__device__ __forceinline__ int least_chunk(double total, int Hkv) {
  const double share = total * Hkv * (1.0 / kItems);
  return uniform(max((int)fmin(share, 33554432.0) + 1, kMinChunk<BM>));
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
template <int BM>
__global__ __launch_bounds__(64 * kPlanWaves) void paged_attention_plan_kernel(PagedBatch pb, int R, int Hkv,
                                                                               int window, int* __restrict__ plan) {
  __shared__ double totals[kPlanWaves];
  __shared__ int sums[kPlanWaves][3];
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int groups = (int)plan_groups(pb.B);
  double total = 0.0;
  for (int g = w; g < groups; g += kPlanWaves) {
    const Seq q = load_seq<BM>(pb, g * kGroup + lane, R, window);
    total += wave_sum_exact((double)q.tiles * q.units);
  }
  if (lane == 0) totals[w] = total;
  __syncthreads();
  total = 0.0;
  for (int i = 0; i < kPlanWaves; ++i) total += totals[i];
  const int chunk = least_chunk<BM>(total, Hkv);
  if (threadIdx.x == 0) plan[0] = chunk;
  int* const before = plan + 1;
  int upto[3] = {0, 0, 0};
  for (int g0 = 0; g0 < groups; g0 += kPlanWaves) {
    const int g = g0 + w;
    const Seq q = load_seq<BM>(pb, min(g, groups) * kGroup + lane, R, window);  // (none past the last group)
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
template <int BM, bool SPLIT>
__device__ __forceinline__ Item find_item(const PagedBatch& pb, const int* __restrict__ plan, int idx, int R, int Hkv,
                                          int window, int lane) {
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
    q = load_seq<BM>(pb, b0 + lane, R, window);
  } else {
    q = load_seq<BM>(pb, lane, R, window);
    // That chunk, then up to 3/8 and one unit larger until the items are no more
    // than the blocks that run at once (a few more would run alone).
    const int least = least_chunk<BM>(wave_sum_exact((double)q.tiles * q.units), Hkv);
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
__device__ __forceinline__ Span span_of(const Item& it, int j0, int j1, int window) {
  Span s;
  const int first = it.pos0 + j0, last = it.pos0 + j1;
  const int lo = window > 0 ? max(first - window + 1, 0) & -kUnit : 0;
  s.lo = max(lo, it.lo + it.split * it.chunk * kUnit);
  s.hi = min(last + 1, it.end);
  if (it.split + 1 < it.splits) s.hi = min(s.hi, it.lo + (it.split + 1) * it.chunk * kUnit);
  s.all_lo = window > 0 ? max(last - window + 1, 0) : 0;
  s.all_hi = min(first + 1, it.end);
  return s;
}

// Sixteen positions from t on (t a multiple of 16, in one page) of one head, in
// bytes from the head's first row: rows from `end` on, and all rows of a page
// that is not there, lie past the extent and read as zeros.  Scalar arithmetic
// without branches: it stands before every tile's loads (page and slot strides
// are below 2^32 bytes, so the products are 32 x 32 -> 64 bits).
struct Rows16 {
  uint64_t at;
  uint32_t bytes;
};
__device__ __forceinline__ Rows16 rows16(const PagedBatch& pb, int page, int t, int end) {
  const uint32_t there = ((unsigned)page < (unsigned)pb.num_pages) & (t < end);
  const uint32_t slot = (uint32_t)t & ((1u << pb.page_shift) - 1);
  const uint32_t slot_bytes = (uint32_t)pb.slot_stride * 2;
  Rows16 r;
  r.at = ((uint64_t)(uint32_t)page * pb.page_bytes + (uint64_t)slot * slot_bytes) & -(uint64_t)there;
  r.bytes = ((uint32_t)(min(end - t, 16) - 1) * slot_bytes + kHeadDim * 2) & -there;
  return r;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint16_t* head, const Rows16& r) {
  return rsrc(reinterpret_cast<const char*>(head) + r.at, r.bytes);
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

// Results of one item: rows of partial sums (split) or of outputs.  And the plan.
struct Out {
  uint16_t* out;
  float* ws;
  const int* plan;
  int Hq, rec_bound;
};

// ---------------------------------------------------------------------------
// attention of up to 16 rows per tile: the cache bytes bound it
// ---------------------------------------------------------------------------

// A block of four waves holds the 16 query rows of one item (decoding: the R
// heads of one token) and each wave walks its own steps of 32 positions with a
// running maximum, denominator and value sums, as the single-sequence
// long-context kernel does: keys go memory -> LDS directly (piece p of row r
// at position p ^ (r & 15)), scores on the matrix cores in fp16, values
// straight into registers as the operand of the fp32 16x16x4 instruction, so
// the probabilities stay in 32 bits.  Two blocks per compute unit: one's
// search for its item, first loads and last joining lie under the other's
// stream.  (Measured on MI355X: sequences of 131072, 77777 and 901 positions,
// 64:8 heads, 147 us, 5.8 TB/s (the shortest of 24 calls 140); 16 of up to 8192,
// 32:8 heads, 40 us (37), of which about 8 are the search, the first loads and
// the joining of the waves; one of 300, 7.6 us (7.3).)  The page numbers of 32
// steps sit in one register of a wave (lane l: half l & 1 of step l >> 1) and
// become scalar buffer descriptors.
constexpr int kWaves = 4;
constexpr int kStep = 32;
constexpr int kRowBytes = (kStep + 4) * 4;         // a row of probabilities (4 words of padding)
constexpr int kKeyBytes = kStep * kHeadDim * 2;    // a step's keys
// Keys and values pass once: loads that do not keep their lines (measured on
// MI355X, three sequences of 131072, 77777 and 901 positions, 64:8 heads: 167 ->
// 151 us; 16 sequences of up to 8192, 32:8: 44 -> 39).
constexpr int kStreamed = 2;
template <int WAVES>
constexpr int kSmallLds = WAVES * (2 * kKeyBytes + 16 * kRowBytes);

__device__ __forceinline__ void lds_read4(u32x4 (&f)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
  asm volatile(
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %5\n\t"
      "ds_read_b128 %2, %6\n\t"
      "ds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
      : "v"(a0), "v"(a1), "v"(a2), "v"(a3)
      : "memory");
}
__device__ __forceinline__ void lds_put(uint32_t addr, float v) {
  asm volatile("ds_write_b32 %0, %1" ::"v"(addr), "v"(v) : "memory");
}

// An item of up to 16 rows, by a block of WAVES waves; REC: rows that a record has room for.
template <int WAVES, int REC>
__device__ __forceinline__ void rows16_item(const PagedBatch& pb, const uint16_t* __restrict__ q, int R, int window,
                                            const Out& o_, const Item& it, int g, char* lds) {
  typedef __attribute__((address_space(3))) void lds_void;
  constexpr int kStride = WAVES * kStep;
  const int lane = threadIdx.x & 63;
  const int w = uniform(threadIdx.x >> 6);
  const int n = lane & 15, j = lane >> 4;
  const int rows = min(it.n * R - it.tile * kSmallRows, kSmallRows);
  const int r0 = it.tile * kSmallRows;
  const Span sp = span_of(it, uniform(r0 / R), uniform((r0 + rows - 1) / R), window);

  // q as matrix operand: lane (m, j), window i: dimensions 32 i + 8 j .. + 7 of row m.
  u32x4 qa[4];
  {
    const int r = r0 + min(n, rows - 1);
    const uint16_t* p = q + ((int64_t)(it.s0 + r / R) * o_.Hq + g * R + r % R) * kHeadDim + 8 * j;
#pragma unroll
    for (int i = 0; i < 4; ++i) qa[i] = *reinterpret_cast<const u32x4*>(p + 32 * i);
  }
  // Rows 4j + r of the results: the positions they see.
  int see_lo[4], see_hi[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int m = 4 * j + r;
    const int pos = it.pos0 + (r0 + m) / R;
    see_hi[r] = m < rows ? min(pos + 1, it.end) : 0;
    see_lo[r] = window > 0 ? pos - window + 1 : 0;
  }

  char* const keys = lds + w * 2 * kKeyBytes;
  const uint32_t probs = lds_byte(lds + WAVES * 2 * kKeyBytes + w * 16 * kRowBytes);
  const int p_first = sp.lo + w * kStep;
  const int* const table = pb.page_table + it.b * pb.table_stride;
  const uint16_t* const khead = pb.k + g * pb.head_stride;
  const uint16_t* const vhead = pb.v + g * pb.head_stride;
  // Page numbers of the 32 steps from step s on (a multiple of 32).
  auto pages_from = [&](int s) {
    const int t = p_first + (s + (lane >> 1)) * kStride + 16 * (lane & 1);
    return t < sp.hi ? table[t >> pb.page_shift] : -1;
  };
  int pages = pages_from(0);

  constexpr int kLoads = kStep / 4;  // load instructions per step for the keys, and for the values
  u32x4 vv[2][kLoads];
  int bad[2];  // whether a page of the step's first (1) or second (2) half is not there
  auto request = [&](auto bc, int s, int p) {
    constexpr int B = decltype(bc)::value;
    if (s > 0 && (s & 31) == 0) pages = pages_from(s);
    const int pg[2] = {readlane(pages, 2 * (s & 31)), readlane(pages, 2 * (s & 31) + 1)};
    bad[B] = ((unsigned)pg[0] >= (unsigned)pb.num_pages ? 1 : 0) | ((unsigned)pg[1] >= (unsigned)pb.num_pages ? 2 : 0);
    const Rows16 at[2] = {rows16(pb, pg[0], p, sp.hi), rows16(pb, pg[1], p + 16, sp.hi)};
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = 4 * i + j;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of(khead, at[i >> 2]), (lds_void*)(keys + B * kKeyBytes + i * 1024), 16,
                                               (uint32_t)(r & 15) * pb.slot_stride * 2 + 16 * (n ^ (r & 15)), 0, 0, kStreamed);
    }
    __builtin_amdgcn_sched_barrier(0);  // the keys' wait below counts the values' loads as the later ones
    // values of step k = 4 kk + i: positions 16 kk + 4 j + i
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      vv[B][k] = __builtin_amdgcn_raw_buffer_load_b128(rows_of(vhead, at[k >> 2]), (uint32_t)(4 * j + (k & 3)) * pb.slot_stride * 2 + 16 * n, 0,
                                                kStreamed);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  float m[4], l[4];
  float4_t o[8];
#pragma unroll
  for (int r = 0; r < 4; ++r) m[r] = kNoMax, l[r] = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = float4_t{0.f, 0.f, 0.f, 0.f};

  // One step: B the buffers that hold it, MORE whether the next step's loads
  // are in flight (compile-time, so that the waits for this step's values,
  // which the compiler counts, leave them in flight).
  auto step = [&](auto bc, auto mc, int p) {
#pragma clang fp contract(off)  // a scaled score is rounded before the maximum, rounded alike, is subtracted
    constexpr int B = decltype(bc)::value;
    constexpr bool MORE = decltype(mc)::value;
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<(MORE ? 3 : 1) * kLoads>();  // the keys: this step's values and the next step's loads may be outstanding
    __builtin_amdgcn_sched_barrier(0);
    const bool masked = (bad[B] != 0) | (p < sp.all_lo) | (p + kStep > sp.all_hi) | (p + kStep > sp.hi);
    float sc[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4 f[4];
      const uint32_t a = lds_byte(keys + B * kKeyBytes) + (16 * t + n) * 256;
      lds_read4(f, a + 16 * (j ^ n), a + 16 * ((4 + j) ^ n), a + 16 * ((8 + j) ^ n), a + 16 * ((12 + j) ^ n));
      float4_t c[4];  // a sum per window of 32 dimensions, added pairwise
#pragma unroll
      for (int i = 0; i < 4; ++i)
        c[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, qa[i]),
                                                      __builtin_bit_cast(half8_t, f[i]),
                                                      float4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      const float4_t cc = (c[0] + c[1]) + (c[2] + c[3]);
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[t][r] = cc[r] * kScaleLog2;
      if (masked) {
        const int at = p + 16 * t + n;
        const bool there = (at < sp.hi) & !(bad[B] >> t & 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][r] = (there & (at >= see_lo[r]) & (at < see_hi[r])) ? sc[t][r] : -INFINITY;
      }
    }
    float alpha[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float mn = fmaxf(m[r], row_max(fmaxf(sc[0][r], sc[1][r])));
      alpha[r] = __builtin_amdgcn_exp2f(m[r] - mn);
      m[r] = mn;
      const float p0 = __builtin_amdgcn_exp2f(sc[0][r] - mn), p1 = __builtin_amdgcn_exp2f(sc[1][r] - mn);
      l[r] = fmaf(l[r], alpha[r], p0 + p1);
      const uint32_t row = probs + (4 * j + r) * kRowBytes + 4 * n;
      lds_put(row, p0);
      lds_put(row + 64, p1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[e][r] *= alpha[r];
    u32x4 pa[4];
    const uint32_t a = probs + n * kRowBytes + 16 * j;  // lane (m, j): positions 16 kk + 4 j .. + 3 of row m
    lds_read4(pa, a, a + 64, a, a + 64);
    __builtin_amdgcn_sched_barrier(0);  // no value is waited for before the softmax is done
    if (masked) {
      // A value that only some rows see may be infinite or NaN, and 0 times it
      // is NaN: such values leave the product and are added to the rows that
      // see them (the result is infinite or NaN whatever their weight).
      uint32_t nf = 0;
#pragma unroll
      for (int k = 0; k < kLoads; ++k) nf |= not_finite(vv[B][k]);
      if (__ballot(nf != 0)) {
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
#pragma unroll 1
          for (int jt = 0; jt < 4; ++jt) {
            const int at = p + 16 * (k >> 2) + 4 * jt + (k & 3);
            const bool there = (at < sp.hi) & !(bad[B] >> (k >> 2) & 1);
            bool sees[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) sees[r] = there & (at >= see_lo[r]) & (at < see_hi[r]);
            u32x4 x;
#pragma unroll
            for (int d = 0; d < 4; ++d) x[d] = __shfl(vv[B][k][d], 16 * jt + n);
            const half8_t v = __builtin_bit_cast(half8_t, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float f = (float)v[e];
              const float add = fabsf(f) < INFINITY ? 0.0f : f;
#pragma unroll
              for (int r = 0; r < 4; ++r) o[e][r] += sees[r] ? add : 0.0f;
            }
          }
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) vv[B][k] = finite_or_zero(vv[B][k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      const u32x4 pk = pa[k >> 2];
      const uint32_t pbits = (k & 3) == 0 ? pk.x : (k & 3) == 1 ? pk.y : (k & 3) == 2 ? pk.z : pk.w;
      const float pf = __builtin_bit_cast(float, pbits);
      const half8_t v = __builtin_bit_cast(half8_t, vv[B][k]);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(pf, (float)v[e], o[e], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr std::integral_constant<int, 0> b0;
  constexpr std::integral_constant<int, 1> b1;
  if (p_first < sp.hi) {
    int p = p_first, s = 0;
    request(b0, 0, p);
    for (; p + 2 * kStride < sp.hi; p += 2 * kStride, s += 2) {
      request(b1, s + 1, p + kStride);
      step(b0, std::true_type{}, p);
      request(b0, s + 2, p + 2 * kStride);
      step(b1, std::true_type{}, p + kStride);
    }
    if (p + kStride < sp.hi) {
      request(b1, s + 1, p + kStride);
      step(b0, std::true_type{}, p);
      step(b1, std::false_type{}, p + kStride);
    } else {
      step(b0, std::false_type{}, p);
    }
  }

  // The waves' results, in wave order: 128 value sums per (wave, row) over the
  // keys' place, maxima and denominators over the probabilities'.
  __syncthreads();
  float* const osum = reinterpret_cast<float*>(lds);                              // [WAVES][16][128]
  float* const stat = reinterpret_cast<float*>(lds + WAVES * 2 * kKeyBytes);     // [WAVES][16][2]
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int h = 4 * j + r;
    const float lt = row_sum(l[r]);
    float* d = osum + (w * 16 + h) * kHeadDim + 8 * n;
    *reinterpret_cast<float4_t*>(d) = float4_t{o[0][r], o[1][r], o[2][r], o[3][r]};
    *reinterpret_cast<float4_t*>(d + 4) = float4_t{o[4][r], o[5][r], o[6][r], o[7][r]};
    if (n == 0) {
      stat[(w * 16 + h) * 2] = m[r];
      stat[(w * 16 + h) * 2 + 1] = lt;
    }
  }
  __syncthreads();
  const int rec = it.rec + it.split;
  if (it.splits > 1 && rec >= o_.rec_bound) return;  // token_start out of order
  float* const wp = o_.ws + ((int64_t)g * o_.rec_bound + rec) * (REC * (kHeadDim + 2));
  for (int idx = threadIdx.x; idx < rows * kHeadDim; idx += 64 * WAVES) {
    const int h = idx / kHeadDim, d = idx % kHeadDim;
    float M = kNoMax;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) M = fmaxf(M, stat[(i * 16 + h) * 2]);
    float den = 0.0f, num = 0.0f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float e = __builtin_amdgcn_exp2f(stat[(i * 16 + h) * 2] - M);
      den = fmaf(e, stat[(i * 16 + h) * 2 + 1], den);
      num = fmaf(e, osum[(i * 16 + h) * kHeadDim + d], num);
    }
    if (it.splits > 1) {
      wp[idx] = num;
      if (d == 0) {
        wp[REC * kHeadDim + 2 * h] = M;
        wp[REC * kHeadDim + 2 * h + 1] = den;
      }
    } else {
      const int r = r0 + h;
      const _Float16 y = (_Float16)(den == 0.0f ? 0.0f : num / den);
      o_.out[((int64_t)(it.s0 + r / R) * o_.Hq + g * R + r % R) * kHeadDim + d] = __builtin_bit_cast(uint16_t, y);
    }
  }
}

__global__ __launch_bounds__(64 * kWaves, 2) void paged_attention_rows16_kernel(PagedBatch pb,
                                                                             const uint16_t* __restrict__ q, int R,
                                                                             int Hkv, int window, Out o_) {
  extern __shared__ u32x4 small_lds[];
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<kSmallRows, false>(pb, o_.plan, at_item, R, Hkv, window, threadIdx.x & 63);
  if (!it.found) return;
  rows16_item<kWaves, kSmallRows>(pb, q, R, window, o_, it, g, reinterpret_cast<char*>(small_lds));
}

// ---------------------------------------------------------------------------
// attention of prompts' chunks: the matrix cores bound it
// ---------------------------------------------------------------------------

// A block of eight waves holds 256 query rows of one item, 32 a wave, and walks
// the positions in tiles of 64.  Scores are formed transposed, keys (rows) x
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
// the fp32 sum of the unrounded ones.
// A sequence of up to 16 rows (decoding rows beside a chunk, or of a batch with
// much padding) would fill half a wave's rows: the block takes its items as the
// 16-row kernel does, with probabilities in 32 bits and eight waves along the
// positions.  Its records have the place of 256 rows.  (Measured on MI355X: a
// chunk beside 15 decoding rows 77.8 -> 78.2 us; two waves more for the
// probabilities' remainders instead, 84.8.)
//
// What bounds it: the issue of matrix and vector instructions by two waves a
// SIMD that do little of the one while the other does the other.  (Counters of
// two prompts of 8192 and 4001 rows, 32:8 heads, on MI355X: matrix instructions
// 42 % of the SIMDs' cycles, vector instructions 48 %; LDS active 27 % of the
// compute units' cycles, no bank conflicts.  Kernel alone, without the joining:
// 874 us, 780 TFLOP/s, the median of 24 calls under a kernel trace, 823 the
// shortest; a call with the joining 768 to 804, 847 to 887 TFLOP/s, untraced; a
// library's fp16 8192^3 product reaches 1150.  As two blocks of 128 rows, with
// twice the staging instructions, 945.  With 128 rows a tile took a wave
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
constexpr int kLargeThreads = 512;
constexpr int kLargeLds = std::max(4 * kTileBytes + 64, kSmallLds<kLargeThreads / 64>);
constexpr float kProbLog2 = 8.0f, kLagLog2 = 7.0f;
constexpr float kFarLog2 = 65536.0f;

__global__ __launch_bounds__(kLargeThreads, 2) void paged_attention_rows256_kernel(PagedBatch pb,
                                                                                   const uint16_t* __restrict__ q,
                                                                                   int R, int Hkv, int window,
                                                                                   Out o_) {
  extern __shared__ u32x4 large_lds[];
  char* const lds = reinterpret_cast<char*>(large_lds);
  int* const flags = reinterpret_cast<int*>(lds + 4 * kTileBytes);  // [4]: tile (& 3) whose values are not all finite
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = uniform(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<kLargeRows, false>(pb, o_.plan, at_item, R, Hkv, window, lane);
  if (!it.found) return;
  if (it.n * R <= kSmallRows) {
    rows16_item<kLargeThreads / 64, kLargeRows>(pb, q, R, window, o_, it, g, lds);
    return;
  }
  const int r0 = it.tile * kLargeRows;
  const int rows = min(it.n * R - r0, kLargeRows);
  const Span sp = span_of(it, uniform(r0 / R), uniform((r0 + rows - 1) / R), window);

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
  const uint16_t* const khead = pb.k + g * pb.head_stride;
  const uint16_t* const vhead = pb.v + g * pb.head_stride;
  // Where the groups of 16 positions lie, 64 groups (16 tiles) at a time: a
  // lane computes a group's byte offset from the head's first row, and the
  // mask says which pages are there; a tile's loads then cost a few scalar
  // instructions.  Two sets are held: rows are loaded two tiles before they
  // are computed.
  constexpr int kSet = 16;  // tiles
  uint32_t set_lo = 0, set_hi = 0, old_lo = 0, old_hi = 0;
  uint64_t set_there = 0, old_there = 0;
  int set_first = 0;  // its first tile; the set before covers the kSet tiles before that
  auto next_set = [&](int t) {
    old_lo = set_lo, old_hi = set_hi, old_there = set_there;
    const int at = sp.lo + t * kTile + 16 * lane;
    const int page = at < sp.hi ? table[at >> pb.page_shift] : -1;
    const bool there = (unsigned)page < (unsigned)pb.num_pages;
    const uint64_t off = (uint64_t)(uint32_t)page * pb.page_bytes +
                         (uint64_t)((uint32_t)at & ((1u << pb.page_shift) - 1)) * (uint32_t)(pb.slot_stride * 2);
    set_lo = there ? (uint32_t)off : 0;
    set_hi = there ? (uint32_t)(off >> 32) : 0;
    set_there = __ballot(there);
    set_first = t;
  };

  // Staging: thread (row tid / 16 of each half of the tile, piece tid % 16);
  // a wave's rows of a half lie in one group of 16.
  const int sr = tid >> 4, spc = tid & 15;
  const uint32_t src_at = (uint32_t)(sr & 15) * pb.slot_stride * 2 + 16 * spc;
  u32x4 kreg[2], vreg[2];
  // Groups of tile t whose page is not there, for the tiles of the two sets.
  auto bad_of = [&](int t) {
    const int i = (t - set_first) & (kSet - 1);
    return (int)(~(t >= set_first ? set_there : old_there) >> 4 * i) & 15;
  };
  auto load_rows = [&](u32x4(&r)[2], const uint16_t* head, int t) {
    const int i0 = (t - set_first) & (kSet - 1);
    const bool now = t >= set_first;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int gr = 2 * i + (w >> 2), l = 4 * i0 + gr;
      const uint32_t lo = readlane((int)(now ? set_lo : old_lo), l), hi = readlane((int)(now ? set_hi : old_hi), l);
      const uint32_t there = (uint32_t)((now ? set_there : old_there) >> l) & 1;
      const int left = sp.hi - (sp.lo + t * kTile + 16 * gr);  // (a page that is there has a row)
      Rows16 at;
      at.at = (uint64_t)hi << 32 | lo;
      at.bytes = ((uint32_t)(min(left, 16) - 1) * (uint32_t)(pb.slot_stride * 2) + kHeadDim * 2) & -there;
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
  auto store_keys = [&](int t) {
    char* const d = lds + (t & 1) * 2 * kTileBytes;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<u32x4*>(d + (32 * i + sr) * 256 + 16 * (spc ^ (sr & 15))) = kreg[i];
  };
  // Values that are infinite or NaN stay out of masked tiles: 0 times one is NaN.
  auto store_values = [&](int t) {
    if (is_masked(t)) {
      if (not_finite(vreg[0]) | not_finite(vreg[1])) flags[t & 3] = t;
#pragma unroll
      for (int i = 0; i < 2; ++i) vreg[i] = finite_or_zero(vreg[i]);
    }
    char* const d = lds + (t & 1) * 2 * kTileBytes + kTileBytes;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<u32x4*>(d + (32 * i + sr) * 256 + 16 * (spc ^ (4 * (sr & 3)))) = vreg[i];
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
      m4[i] = fmaxf(s[0][i], s[1][i]);
#pragma unroll
      for (int r = 4; r < 16; r += 4) m4[i] = fmaxf(m4[i], fmaxf(s[0][r + i], s[1][r + i]));
    }
    float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
    auto x = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, mx), __builtin_bit_cast(uint32_t, mx), false,
                                              false);
    mx = fmaxf(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1])) * kScaleLog2;
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
      const uint16_t* const row = vhead + (int64_t)page * (pb.page_bytes / 2) +
                                  (int64_t)(at & ((1 << pb.page_shift) - 1)) * pb.slot_stride;
      const bool sees = (at >= see_lo) & (at < see_hi);
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const half4_t x = *reinterpret_cast<const half4_t*>(row + 32 * d + 2 * r + 4 * h);
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
// WAVES == 4: a block per row, its waves take every fourth record and meet in
// LDS (decoding: few rows, many ranges).  WAVES == 1: a wave per four rows,
// 16 rows a block at a time (a chunk's rows have few ranges each).  Most blocks
// of the grid can find nothing to do and cost their search, so there are about
// kJoinBlocks of them, which go on to further rows.  (Measured on MI355X: two
// prompts whose tiles are not split, 16.4 -> 4.9 us; a chunk beside 15 decoding
// rows, 14.5 -> 15.5, of the bytes of its records; twice the blocks, 8.7 and 17.)
template <int BM, int WAVES>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(PagedBatch pb, int R, int Hkv, int window, Out o_) {
  __shared__ float2_t part[4][64];
  constexpr int kRec = BM * (kHeadDim + 2);
  constexpr int kRows = WAVES == 4 ? 1 : 4;  // rows of a wave
  constexpr int kB = WAVES == 4 ? 8 : 4;     // records loaded at a time
  const int lane = threadIdx.x & 63;
  const int w = uniform(threadIdx.x >> 6);
  const int at_item = uniform(blockIdx.x / Hkv), g = (int)blockIdx.x - at_item * Hkv;
  const Item it = find_item<BM, true>(pb, o_.plan, at_item, R, Hkv, window, lane);
  if (!it.found || it.rec + it.splits > o_.rec_bound) return;
  const int r0 = it.tile * BM;
  const int rows = min(it.n * R - r0, BM);
  const int first = WAVES == 4 ? w : 0;
  const float* const base = o_.ws + ((int64_t)g * o_.rec_bound + it.rec) * kRec;
  // WAVES == 4: a row, the same for the whole block; else every gridDim.y-th group of 16
#pragma unroll 1
  for (int row = WAVES == 4 ? blockIdx.y : blockIdx.y * 16 + w * 4; row < rows; row += 16 * gridDim.y) {
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
      if (w > 0) return;
      num[0] = part[0][lane];
#pragma unroll
      for (int i = 1; i < 4; ++i) num[0] += part[i][lane];
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if (row + k >= rows) break;
      const int r = r0 + row + k;
      const float inv = den[k] == 0.0f ? 0.0f : 1.0f / den[k];
      *reinterpret_cast<half2_t*>(o_.out + ((int64_t)(it.s0 + r / R) * o_.Hq + g * R + r % R) * kHeadDim + 2 * lane) =
          half2_t{(_Float16)(num[k][0] * inv), (_Float16)(num[k][1] * inv)};
    }
    if constexpr (WAVES == 4) return;
  }
}

// Which kernel takes a batch, and its bounds: a pure function of the sizes.
struct AttentionPlan {
  bool large;
  int64_t items, split_tiles, records;  // per key/value head
  int64_t floats;                       // workspace: the records, then the plan
  int64_t plan_at;
};

template <int BM>
AttentionPlan plan_of(int64_t B, int64_t T, int64_t R, int64_t Hkv, int64_t capacity) {
  AttentionPlan p;
  p.large = BM == kLargeRows;
  const int64_t tiles = (T * R + std::min(B, T) * (BM - 1)) / BM;
  const int64_t per_head = (kItems + Hkv - 1) / Hkv;
  // (with kItems heads and more a head's share of the items is one: no sequence is split)
  const bool split = capacity > (int64_t)kMinChunk<BM> * kUnit && Hkv < kItems;
  p.items = tiles + (split ? per_head : 0);
  p.split_tiles = split ? std::min(per_head, tiles) : 0;
  const int64_t most = (capacity + kMinChunk<BM> * kUnit - 1) / (kMinChunk<BM> * kUnit);
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
AttentionPlan attention_plan(int64_t B, int64_t T, int64_t R, int64_t Hkv, int64_t capacity) {
  if (T * R <= kSmallRows * B) return plan_of<kSmallRows>(B, T, R, Hkv, capacity);
  return plan_of<kLargeRows>(B, T, R, Hkv, capacity);
}

}  // namespace

namespace {
// Waves of a row of the append: one where rows alone fill the chip, else one per group of eight heads.
int64_t append_waves(int64_t T, int64_t Hq, int64_t Hkv) {
  return std::max<int64_t>(1, std::min<int64_t>((Hq + 2 * Hkv + 7) / 8, kResidentWaves / T));
}
}  // namespace

int64_t paged_append_threads(int64_t T, int64_t Hq, int64_t Hkv) {
  return (T * append_waves(T, Hq, Hkv) + 3) / 4 * 256;
}

hipError_t launch_paged_append(const PagedBatch& pb, const uint16_t* qkv, int64_t qkv_stride, const uint16_t* qw,
                               const uint16_t* kw, const float* cos_sin, int64_t rope_rows, int64_t Hq, int64_t Hkv,
                               float eps, uint16_t* q_out, hipStream_t stream, const LaunchEvents& ev) {
  launch(paged_append_kernel, dim3((unsigned)(paged_append_threads(pb.T, Hq, Hkv) / 256)), dim3(256), 0, stream, ev, pb,
         qkv, qkv_stride, qw, kw, cos_sin, (int)std::min<int64_t>(rope_rows, 0x7FFFFFFF), (int)Hq, (int)Hkv, eps, q_out,
         (int)append_waves(pb.T, Hq, Hkv));
  return hipGetLastError();
}

int64_t paged_attention_workspace(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  return attention_plan(B, T, Hq / Hkv, Hkv, capacity).floats * (int64_t)sizeof(float);
}

int64_t paged_attention_threads(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  const AttentionPlan p = attention_plan(B, T, Hq / Hkv, Hkv, capacity);
  return p.items * Hkv * (p.large ? kLargeThreads : 64 * kWaves);
}

hipError_t launch_paged_attention(const PagedBatch& pb, const uint16_t* q, int64_t Hq, int64_t Hkv, int64_t window,
                                  uint16_t* out, float* ws, hipStream_t stream, const LaunchEvents& ev) {
  const int64_t R = Hq / Hkv;
  const AttentionPlan p = attention_plan(pb.B, pb.T, R, Hkv, (int64_t)pb.table_pages << pb.page_shift);
  LaunchEvents e0, e1 = ev, e2;
  if (p.split_tiles > 0) {  // the measurement hook spans all kernels
    e1.stop = nullptr;
    e2.stop = ev.stop;
  }
  int* const plan = reinterpret_cast<int*>(ws + p.plan_at);
  if (pb.B > kGroup) {
    e0.start = e1.start;
    e1.start = nullptr;
    auto* const kernel = p.large ? paged_attention_plan_kernel<kLargeRows> : paged_attention_plan_kernel<kSmallRows>;
    launch(kernel, dim3(1), dim3(64 * kPlanWaves), 0, stream, e0, pb, (int)R, (int)Hkv, (int)window, plan);
  }
  const Out o{out, ws, plan, (int)Hq, (int)p.records};
  const dim3 grid((unsigned)(p.items * Hkv));
  // A block joins one row; 16 rows where the tiles (most of them not split) would make many blocks.
  constexpr int64_t kFewTiles = 32, kJoinBlocks = 2048;
  const bool many = p.large && p.split_tiles * Hkv > kFewTiles;
  const int64_t most_rows = std::min<int64_t>(p.large ? kLargeRows : kSmallRows, pb.T * R);
  const int64_t by_16 = std::min((most_rows + 15) / 16, std::max<int64_t>(1, kJoinBlocks / (p.split_tiles * Hkv + 1)));
  const dim3 join((unsigned)(p.split_tiles * Hkv), (unsigned)(many ? by_16 : most_rows));
  if (p.large) {
    launch(paged_attention_rows256_kernel, grid, dim3(kLargeThreads), kLargeLds, stream, e1, pb, q, (int)R, (int)Hkv,
           (int)window, o);
    if (p.split_tiles > 0 && p.split_tiles * Hkv <= kFewTiles)
      launch((paged_attention_join_kernel<kLargeRows, 4>), join, dim3(256), 0, stream, e2, pb, (int)R, (int)Hkv,
             (int)window, o);
    else if (p.split_tiles > 0)
      launch((paged_attention_join_kernel<kLargeRows, 1>), join, dim3(256), 0, stream, e2, pb, (int)R, (int)Hkv,
             (int)window, o);
  } else {
    launch(paged_attention_rows16_kernel, grid, dim3(64 * kWaves), kSmallLds<kWaves>, stream, e1, pb, q, (int)R, (int)Hkv,
           (int)window, o);
    if (p.split_tiles > 0)
      launch((paged_attention_join_kernel<kSmallRows, 4>), join, dim3(256), 0, stream, e2, pb, (int)R, (int)Hkv, (int)window,
             o);
  }
  return hipGetLastError();
}

}  // namespace laq

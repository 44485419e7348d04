// Batched serving over paged key/value caches of 8 bits: e4m3 codes with an e8m0
// scale (a power of two) for each 16 positions of a head, one of keys and one of
// values.  The append of new rows (per-head q/k RMSNorm, rotary embedding) that
// chooses the scales, and the attention of new rows over such caches.  fp32 sums
// and softmax statistics, fixed reduction orders (deterministic).  Head
// dimension 128.  The work of a batch, the kernel of prompts' chunks and the
// joining of split sequences are paged_attention.h's.
//
// A power of two as scale: where a block's scale grows, its codes are halved
// some times, which rounds only those that become subnormal; and from 2^-15 to
// 2^7 every value that a code stands for is an fp16 number, so that the matrix
// cores work on the values themselves and nothing is rounded on the way to them.
#include "paged_attention.h"

namespace laq {

namespace {

constexpr int kBlock = 16;  // positions that share a scale

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------

// The sequence that row `row` belongs to, by its place among the sequences' ends
// from sequence `seq` on, which do not decrease, 64 of them a step: B, or one
// that begins after the row, where there is none.
__device__ __forceinline__ int sequence_of(const PagedBatch& pb, int seq, int row, int lane) {
  for (int left = pb.B - seq; left > 0;) {
    const int step = (left + 63) >> 6, last = (lane + 1) * step - 1;  // a lane's step sequences end with the last's end
    const bool before = last < left && pb.token_start[seq + last + 1] <= row;
    const int whole = __popcll(__ballot(before)) * step;
    seq += whole;
    left = min(step - 1, left - whole);
  }
  return uniform(seq);
}

// Sixteen dimensions of a head, 8i .. 8i + 7 and their rotation partners 64 further.
struct Part {
  float u[8], v[8];
};

// Their rotation: a row of cosines and sines.
struct Turn {
  float c[8], s[8];
};
__device__ __forceinline__ Turn turn_of(const float* __restrict__ cs, int i) {
  Turn t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t.c[e] = cs[8 * i + e], t.s[e] = cs[64 + 8 * i + e];
  return t;
}

// Normalized (w: not null) and rotated.
__device__ __forceinline__ void norm_rope(Part& p, const uint16_t* __restrict__ w, const Turn& t, int i, float eps) {
  float ss = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss = fmaf(p.u[e], p.u[e], fmaf(p.v[e], p.v[e], ss));
  ss = sum8(ss);
  if (w != nullptr) {
    const float r = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + eps);
    const half8_t wa = *reinterpret_cast<const half8_t*>(w + 8 * i);
    const half8_t wb = *reinterpret_cast<const half8_t*>(w + 64 + 8 * i);
#pragma unroll
    for (int e = 0; e < 8; ++e) p.u[e] = p.u[e] * r * (float)wa[e], p.v[e] = p.v[e] * r * (float)wb[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float u = p.u[e] * t.c[e] - p.v[e] * t.s[e], v = p.v[e] * t.c[e] + p.u[e] * t.s[e];
    p.u[e] = u, p.v[e] = v;
  }
}

struct Raw {
  u32x4 a, b;
};
__device__ __forceinline__ Raw raw_of(const uint16_t* head, int i) {
  return Raw{*reinterpret_cast<const u32x4*>(head + 8 * i), *reinterpret_cast<const u32x4*>(head + 64 + 8 * i)};
}
__device__ __forceinline__ Part part_of(const Raw& r) {
  const half8_t a = __builtin_bit_cast(half8_t, r.a), b = __builtin_bit_cast(half8_t, r.b);
  Part p;
#pragma unroll
  for (int e = 0; e < 8; ++e) p.u[e] = (float)a[e], p.v[e] = (float)b[e];
  return p;
}

// The least exponent (as an e8m0 byte) in 112..134 whose power of two times 448
// (1.75 x 2^8) is a or more: a's own exponent less 8, one more where its
// significand is above 1.75.
__device__ __forceinline__ int least_scale(float a) {
  return min(max((int)((__builtin_bit_cast(uint32_t, a) + 0x1FFFFFu) >> 23) - 8, 112), 134);
}
__device__ __forceinline__ float inverse_scale(int byte) { return __builtin_bit_cast(float, (254 - byte) << 23); }

// e4m3 codes, rounded to nearest even: past 448 saturated, NaN where not finite.
__device__ __forceinline__ float fit(float x, float inv) {
  const float y = x * inv;
  return fabsf(y) < INFINITY ? __builtin_amdgcn_fmed3f(y, -448.0f, 448.0f) : y;
}
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 codes_of(const float (&x)[8], float inv) {
  return u32x2{codes_of(fit(x[0], inv), fit(x[1], inv), fit(x[2], inv), fit(x[3], inv)),
               codes_of(fit(x[4], inv), fit(x[5], inv), fit(x[6], inv), fit(x[7], inv))};
}
__device__ __forceinline__ uint32_t again(uint32_t c, float by) {
  return codes_of(__builtin_amdgcn_cvt_f32_fp8(c, 0) * by, __builtin_amdgcn_cvt_f32_fp8(c, 1) * by,
                  __builtin_amdgcn_cvt_f32_fp8(c, 2) * by, __builtin_amdgcn_cvt_f32_fp8(c, 3) * by);
}

// Largest over the 64 lanes.
__device__ __forceinline__ float wave_max(float v) {
  const int u = __builtin_bit_cast(int, row_max(v));
  auto f = [](int x) { return __builtin_bit_cast(float, x); };
  return fmaxf(fmaxf(f(readlane(u, 0)), f(readlane(u, 16))), fmaxf(f(readlane(u, 32)), f(readlane(u, 48))));
}

// A wave takes either the keys or the values of one key/value head in a window
// of `window` rows: the blocks of 16 positions whose first new row lies in the
// window (all of a block's new rows are one sequence's, so one wave sees the
// whole block and the scale needs no exchange between waves); or one row and
// every q_waves-th group of eight query heads.  Eight lanes a row or head: lane i
// holds dimensions 8i .. 8i + 7 and their partners.  What bounds it: the bytes of
// the rows in and out where there are many (16384 rows, 32:8 heads: 78 us, 4.8
// TB/s on MI355X, a large copy moves 5.2); few rows are a launch and the chain of
// dependent reads: sequence, page, the block's old scale (16 rows: 4.4 us).
__global__ __launch_bounds__(256) void paged_append_codes_kernel(PagedCodes pb, const uint16_t* __restrict__ qkv,
                                                                 int64_t qkv_stride, const uint16_t* __restrict__ qw,
                                                                 const uint16_t* __restrict__ kw,
                                                                 const float* __restrict__ cos_sin, int rope_rows,
                                                                 int Hq, int Hkv, float eps,
                                                                 uint16_t* __restrict__ q_out, int window, int q_waves,
                                                                 uint32_t kv_waves) {
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * 4 + (uint32_t)uniform(threadIdx.x >> 6);
  const int i = lane & 7;
  const int64_t cap = (int64_t)pb.table_pages << pb.page_shift;
  const int most = (int)min(cap, (int64_t)rope_rows);  // positions from here on have no place or no rotation

  if (wave >= kv_waves) {
    const int row = uniform((int)((wave - kv_waves) / (uint32_t)q_waves));
    const int at = uniform((int)(wave - kv_waves - (uint32_t)row * (uint32_t)q_waves));
    if (row >= pb.T) return;
    const int groups = (Hq + 7) >> 3;
    const uint16_t* const src = qkv + row * qkv_stride;
    auto load = [&](int grp) { return raw_of(src + (int64_t)min(grp * 8 + (lane >> 3), Hq - 1) * kHeadDim, i); };
    Raw raw = load(at);
    const int seq = sequence_of(pb, 0, row, lane);
    if (seq >= pb.B) return;  // behind the last sequence
    const int s0 = pb.token_start[seq], s1 = min(pb.token_start[seq + 1], pb.T);
    if (row < s0) return;  // before the first
    const int64_t pos = (int64_t)pb.seq_len[seq] - s1 + row;
    const bool placed = pos >= 0 && pos < most;
    const Turn turn = turn_of(cos_sin + (placed ? pos : 0) * kHeadDim, i);
    for (int grp = at; grp < groups;) {
      const int h = grp * 8 + (lane >> 3);
      Part p = part_of(raw);
      const int next = grp + q_waves;
      if (next < groups) raw = load(next);
      norm_rope(p, qw, turn, i, eps);
      half8_t x, y;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (_Float16)p.u[e], y[e] = (_Float16)p.v[e];
      if (!placed) x = half8_t{}, y = half8_t{};
      if (h < Hq) {
        uint16_t* d = q_out + ((int64_t)row * Hq + h) * kHeadDim + 8 * i;
        *reinterpret_cast<half8_t*>(d) = x;
        *reinterpret_cast<half8_t*>(d + 64) = y;
      }
      grp = next;
    }
    return;
  }

  const int at_window = uniform((int)(wave / (uint32_t)(2 * Hkv)));
  const int unit = uniform((int)(wave - (uint32_t)at_window * (uint32_t)(2 * Hkv)));
  const int first = at_window * window;
  const int end = min(first + window, pb.T);
  int seq = sequence_of(pb, 0, first, lane);
  const int g = unit >> 1;
  const bool values = unit & 1;
  const uint16_t* const src = qkv + (int64_t)(Hq + (values ? Hkv : 0) + g) * kHeadDim;
  char* const cache = reinterpret_cast<char*>(values ? pb.v : pb.k) + g * pb.head_stride;
  uint8_t* const scales = values ? pb.v_scales : pb.k_scales;
  int s1 = -1, s0 = 0, len = 0, lead = 0;
  for (int row = first; row < end;) {
    if (row >= s1) {
      if (s1 >= 0) seq = sequence_of(pb, seq, row, lane);
      if (seq >= pb.B) return;
      s0 = pb.token_start[seq], s1 = min(pb.token_start[seq + 1], pb.T), len = pb.seq_len[seq];
      if (s1 <= row) return;  // token_start out of order: every turn of the loop takes a row
      lead = max(max(s0, 0), (int)min((int64_t)s1 - len, (int64_t)s1));  // the first row whose position is not negative
    }
    if (row < lead) {
      row = lead;
      continue;
    }
    const int64_t p64 = (int64_t)len - s1 + row;
    if (p64 >= most) {
      row = s1;
      continue;
    }
    const int pos = uniform((int)p64), before = pos & (kBlock - 1);
    if (before != 0 && row != lead) {  // the block's first new row lies in the window before
      row = min(row + kBlock - before, s1);
      continue;
    }
    const int n = uniform(min(min(kBlock - before, s1 - row), most - pos));
    const int page = pb.page_table[seq * pb.table_stride + (pos >> pb.page_shift)];
    const bool there = (unsigned)page < (unsigned)pb.num_pages;
    const int64_t scale_at = there ? pb.scale_at(page, g, pos) : 0;
    int was = 112;
    if (there && before != 0) was = min(max((int)scales[scale_at], 112), 134);
    // two passes of eight rows
    Part p[2] = {};
    float a = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (8 * k >= n) break;
      const int r = min(8 * k + (lane >> 3), n - 1);
      p[k] = part_of(raw_of(src + (int64_t)(row + r) * qkv_stride, i));
      if (!values) norm_rope(p[k], kw, turn_of(cos_sin + (int64_t)(pos + r) * kHeadDim, i), i, eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = fabsf(p[k].u[e]), y = fabsf(p[k].v[e]);
        a = fmaxf(a, fmaxf(x < INFINITY ? x : 0.0f, y < INFINITY ? y : 0.0f));
      }
    }
    a = wave_max(a);
    row += n;
    if (!there) continue;
    const int scale = uniform(max(least_scale(a), was));
    const float inv = inverse_scale(scale);
    char* const at = cache + (int64_t)page * pb.page_bytes + (int64_t)((pos & ((1 << pb.page_shift) - 1)) - before) * pb.slot_stride + 8 * i;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = 8 * k + (lane >> 3);
      if (r < n) {
        char* const d = at + (int64_t)(before + r) * pb.slot_stride;
        *reinterpret_cast<u32x2*>(d) = codes_of(p[k].u, inv);
        *reinterpret_cast<u32x2*>(d + 64) = codes_of(p[k].v, inv);
      }
    }
    if (before == 0 || scale != was) {
      if (lane == 0) scales[scale_at] = (uint8_t)scale;
    }
    if (scale > was && before != 0) {  // the earlier positions' codes by the new scale
      const float by = __builtin_bit_cast(float, (127 + was - scale) << 23);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int r = 8 * k + (lane >> 3);
        if (r < before) {
          u32x2* const d = reinterpret_cast<u32x2*>(at + (int64_t)r * pb.slot_stride);
          const u32x2 x = d[0], y = d[8];
          d[0] = u32x2{again(x.x, by), again(x.y, by)};
          d[8] = u32x2{again(y.x, by), again(y.y, by)};
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// attention of up to 16 rows per tile: the cache bytes bound it
// ---------------------------------------------------------------------------

// A block of four waves holds the 16 query rows of one item and each wave walks
// its own steps of 32 positions with a running reference, denominator and value
// sums.  Codes of keys and values go memory -> LDS directly, two steps a wave,
// and become fp16 (exactly) as they leave it.  Scores are formed transposed, keys
// (rows) x queries (columns): a lane holds eight scores of one query, of
// positions 16 t + 4 j + r (t: half of the step, j: quarter of the wave), which
// is the order in which the second product takes the probabilities as its
// columns, if the values' operand has the same positions.  That comes from the
// transposing LDS reads: 16 lanes read eight positions x 16 dimensions and
// receive a dimension's eight codes each.  The probabilities keep up to 22 bits: each
// is the sum of two fp16 numbers, and each value product two instructions.
// Piece p (16 bytes) of key row r sits at p ^ (r / 2 & 7) and of value row r at
// p ^ (r / 2 & 3 | r / 16 << 2): the operand reads touch each bank once.
// Two blocks per compute unit.  (Measured on MI355X, kernel alone: sequences of
// 131072, 120002, 77777 and 901 positions, 64:8 heads, 107 us, 6.3 TB/s, a plain
// read reaches 7.0; 16 of up to 8192, 32:8, 21 us, 4.1 TB/s; one of 300, 64:8, not
// split, 8 to 9 us.)
constexpr int kStep = 32;
constexpr int kStepBytes = kStep * kHeadDim;  // of keys; and of values
constexpr int kStreamed = 2;                  // keys and values pass once: loads that do not keep their lines

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
__device__ __forceinline__ void lds_read_columns8(u32x2 (&f)[8], const uint32_t (&a)[8]) {
  asm volatile(
      "ds_read_b64_tr_b8 %0, %8\n\t"
      "ds_read_b64_tr_b8 %1, %9\n\t"
      "ds_read_b64_tr_b8 %2, %10\n\t"
      "ds_read_b64_tr_b8 %3, %11\n\t"
      "ds_read_b64_tr_b8 %4, %12\n\t"
      "ds_read_b64_tr_b8 %5, %13\n\t"
      "ds_read_b64_tr_b8 %6, %14\n\t"
      "ds_read_b64_tr_b8 %7, %15\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7])
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7])
      : "memory");
}
__device__ __forceinline__ uint32_t lds_read1(uint32_t a) {
  uint32_t x;
  asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x) : "v"(a) : "memory");
  return x;
}

// Of the four quarters of a wave, in every lane.
template <typename F>
__device__ __forceinline__ float over_quarters(float v, F&& op) {
  auto f = [](uint32_t x) { return __builtin_bit_cast(float, x); };
  uint32_t u = __builtin_bit_cast(uint32_t, v);
  auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  v = op(f(x[0]), f(x[1]));
  u = __builtin_bit_cast(uint32_t, v);
  auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return op(f(y[0]), f(y[1]));
}

struct CacheE4M3 {
  typedef PagedCodes Batch;
  static constexpr int kBytes = 1;
  // The second kernel costs what eight units do in a block, and the more blocks
  // there are without it, the less it brings.  (Measured on MI355X, 64:8 heads,
  // split -> not: one sequence of 300 positions, 10.8 -> 9.1 us, of 600, 10.7 ->
  // 11.0, of 1000, 10.6 -> 13.6; eight of 600, 12.7 -> 11.2, of 1000, 14.0 -> 13.7;
  // 16 of 1000, 18.7 -> 14.1; 64 of 1000, 30.5 -> 27.3.  Up to 16 units: where one
  // sequence is long among short ones, a block walks it alone.)
  static int split_from(int64_t B, int64_t Hkv) { return (int)std::min<int64_t>(8 + B * Hkv / 16, 16); }
  static constexpr bool kTileRanges = true;
  static constexpr bool kFourWaves = true;
  // Blocks of 128 query rows (two a compute unit) below 512 blocks of 256, whose
  // every compute unit then has two turns: less is left over in the last one, and
  // fewer rows are split over positions and joined.  (Measured on MI355X, blocks of
  // 256 -> 128, 32:8 heads: chunks of 64 rows at 500 positions 25.2 -> 21.3 us, of
  // 512 at 0, 25.8 -> 20.9, at 2000, 58 -> 46, of 2048 at 0, 85 -> 69, of 4096 at 0
  // (512 blocks) 161 -> 182; 64:8, 2048 at 0 (512) 96 -> 103; 8:1, 4096 at 0 (128),
  // 76 -> 83.)
  static bool four_waves(int64_t rows) { return rows < 512 * kChunkRows<8>; }
  template <int WAVES>
  static constexpr int kItemLds = WAVES * (4 * kStepBytes + 16 * 8);
  template <int WAVES, int REC>
  static __device__ __forceinline__ void rows16_item(const PagedCodes& pb, const uint16_t* __restrict__ q, int R,
                                                     int window, const Out& o_, const Item& it, int g, char* lds);
};

// An item of up to 16 rows, by a block of WAVES waves; REC: rows that a record has room for.
template <int WAVES, int REC>
__device__ __forceinline__ void CacheE4M3::rows16_item(const PagedCodes& pb, const uint16_t* __restrict__ q, int R,
                                                       int window, const Out& o_, const Item& it, int g, char* lds) {
  typedef __attribute__((address_space(3))) void lds_void;
  constexpr int kStride = WAVES * kStep;
  const int lane = threadIdx.x & 63;
  const int w = uniform(threadIdx.x >> 6);
  const int n = lane & 15, j = lane >> 4;
  const int rows = min(it.n * R - it.tile * kSmallRows, kSmallRows);
  const int r0 = it.tile * kSmallRows;
  const Span sp = span_of<kTileRanges>(it, uniform(r0 / R), uniform((r0 + rows - 1) / R), window);

  // q as matrix operand: lane (n, j), window 2a + b: dimensions 64 a + 16 j + 8 b .. + 7 of row n.
  const int mine = min(n, rows - 1);
  half8_t qb[4];
  {
    const int r = r0 + mine;
    const uint16_t* p = q + ((int64_t)(it.s0 + r / R) * o_.Hq + g * R + r % R) * kHeadDim + 16 * j;
#pragma unroll
    for (int i = 0; i < 4; ++i) qb[i] = *reinterpret_cast<const half8_t*>(p + 64 * (i >> 1) + 8 * (i & 1));
  }
  // The positions that row n sees.
  const int pos = it.pos0 + (r0 + mine) / R;
  const int see_hi = n < rows ? min(pos + 1, it.end) : 0;
  const int see_lo = window > 0 ? pos - window + 1 : 0;

  char* const ring = lds + w * 4 * kStepBytes;  // [2 steps][keys, values]
  const uint32_t kbase = lds_byte(ring) + n * kHeadDim + 16 * (j ^ (n >> 1 & 7));
  uint32_t vbase;
  {
    const int r = n >> 1, at = 16 * (r >> 2) + 4 * j + (r & 3);  // this lane's position in the transposing reads
    vbase = lds_byte(ring) + kStepBytes + at * kHeadDim + 16 * ((at >> 1 & 3) | (at >> 4) << 2) + 8 * (n & 1);
  }
  const int p_first = sp.lo + w * kStep;
  const int* const table = pb.page_table + it.b * pb.table_stride;
  const char* const khead = reinterpret_cast<const char*>(pb.k) + g * pb.head_stride;
  const char* const vhead = reinterpret_cast<const char*>(pb.v) + g * pb.head_stride;
  // Page numbers of the 32 steps from step s on (a multiple of 32): lane l has half l & 1 of step l >> 1.
  auto pages_from = [&](int s) {
    const int t = p_first + (s + (lane >> 1)) * kStride + 16 * (lane & 1);
    return t < sp.hi ? table[t >> pb.page_shift] : -1;
  };
  int pages = pages_from(0), pages_next = -1;
  // Their scales: those of the steps requested, and of the steps computed (32 steps change at different times).
  int ks_next = 0, vs_next = 0, ks = 0, vs = 0;
  auto scales_from = [&](int s) {
    const int t = p_first + (s + (lane >> 1)) * kStride + 16 * (lane & 1);
    if ((unsigned)pages < (unsigned)pb.num_pages) {
      const int64_t i = pb.scale_at(pages, g, t);
      ks_next = pb.k_scales[i], vs_next = pb.v_scales[i];
    }
  };

  constexpr int kLoads = kStep / 8;  // load instructions per step for the keys, and for the values
  int bad[2];  // whether a page of the step's first (1) or second (2) half is not there
  auto request = [&](auto bc, int s, int p) {
    constexpr int B = decltype(bc)::value;
    if ((s & 31) == 0) {
      if (s > 0) pages = pages_next;
      scales_from(s);
    }
    if ((s & 31) == 16) pages_next = pages_from(s + 16);
    const int pg[2] = {readlane(pages, 2 * (s & 31)), readlane(pages, 2 * (s & 31) + 1)};
    bad[B] = ((unsigned)pg[0] >= (unsigned)pb.num_pages ? 1 : 0) | ((unsigned)pg[1] >= (unsigned)pb.num_pages ? 2 : 0);
    const Rows16 at[2] = {rows16<1>(pb, pg[0], p, sp.hi), rows16<1>(pb, pg[1], p + 16, sp.hi)};
    const int r = lane >> 3;  // row within eight
    char* const d = ring + B * 2 * kStepBytes;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of(khead, at[i >> 1]), (lds_void*)(d + i * 1024), 16,
                                               (uint32_t)(8 * (i & 1) + r) * pb.slot_stride + 16 * ((lane & 7) ^ (4 * (i & 1) + (r >> 1))), 0, 0, kStreamed);
    __builtin_amdgcn_sched_barrier(0);  // the keys' wait below counts the values' loads as the later ones
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rows_of(vhead, at[i >> 1]), (lds_void*)(d + kStepBytes + i * 1024), 16,
                                               (uint32_t)(8 * (i & 1) + r) * pb.slot_stride + 16 * ((lane & 7) ^ ((r >> 1) | (i >> 1) << 2)), 0, 0, kStreamed);
    __builtin_amdgcn_sched_barrier(0);
  };

  // A probability is 2^(score - ref); ref lies 8 below the maximum when it is
  // set and follows once that has grown by 7 more, so that it is below 2^15 and the
  // largest so far 2^8 or more.  Its second part, cut off like the first, has steps
  // of 2^-21 of the probability, but none below 2^-24 (fp16's least): 22 bits down
  // to 2^-3, 2^-11 of the largest, and an error below 2^-32 of the largest from
  // there on.
  constexpr float kBelow = 8.0f, kLag = 15.0f;
  float ref = kNoMax, l = 0.0f;
  float4_t o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = float4_t{0.f, 0.f, 0.f, 0.f};

  // One step: B the buffer that holds it, MORE whether the next step's loads are in flight.
  auto step = [&](auto bc, auto mc, int s, int p) {
#pragma clang fp contract(off)  // a scaled score is rounded before the reference, rounded alike, is subtracted
    constexpr int B = decltype(bc)::value;
    constexpr bool MORE = decltype(mc)::value;
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<(MORE ? 3 : 1) * kLoads>();  // the keys: this step's values and the next step's loads may be outstanding
    __builtin_amdgcn_sched_barrier(0);
    if ((s & 31) == 0) ks = ks_next, vs = vs_next;
    const bool masked = (bad[B] != 0) | (p < sp.all_lo) | (p + kStep > sp.all_hi) | (p + kStep > sp.hi);
    const float ksc[2] = {block_scale(readlane(ks, 2 * (s & 31))), block_scale(readlane(ks, 2 * (s & 31) + 1))};
    const float vsc[2] = {block_scale(readlane(vs, 2 * (s & 31))), block_scale(readlane(vs, 2 * (s & 31) + 1))};
    u32x4 f[4];
    {
      const uint32_t a = kbase + B * 2 * kStepBytes;
      lds_read4(f, a, a ^ 64, a + 16 * kHeadDim, (a ^ 64) + 16 * kHeadDim);
    }
    float sc[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float4_t c[2];  // a sum per half of the dimensions
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const u32x4 x = f[2 * t + a];
        c[a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            frag(values01(x.x, ksc[t]), values23(x.x, ksc[t]), values01(x.y, ksc[t]), values23(x.y, ksc[t])), qb[2 * a],
            float4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        c[a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
            frag(values01(x.z, ksc[t]), values23(x.z, ksc[t]), values01(x.w, ksc[t]), values23(x.w, ksc[t])),
            qb[2 * a + 1], c[a], 0, 0, 0);
      }
      const float4_t cc = c[0] + c[1];
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[t][r] = cc[r] * kScaleLog2;
      if (masked) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = p + 16 * t + 4 * j + r;
          const bool sees = (at < sp.hi) & !(bad[B] >> t & 1) & (at >= see_lo) & (at < see_hi);
          sc[t][r] = sees ? sc[t][r] : -INFINITY;
        }
      }
    }
    float mx = maximum(maximum(sc[0][0], sc[0][1]), sc[0][2]);
    mx = maximum(maximum(mx, sc[0][3]), sc[1][0]);
    mx = maximum(maximum(mx, sc[1][1]), maximum(sc[1][2], sc[1][3]));  // (of a row with a NaN score all is NaN)
    mx = over_quarters(mx, [](float a, float b) { return maximum(a, b); });
    const bool ahead = mx - ref > kLag;
    if (__ballot(ahead)) {
      const float to = ahead ? mx - kBelow : ref;  // each query by itself
      const float alpha = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[e][r] *= alpha;
    }
    uint32_t hi[4], lo[4];
    float sum[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float pr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[r] = __builtin_amdgcn_exp2f(sc[t][r] - ref);
      sum[t] = (pr[0] + pr[1]) + (pr[2] + pr[3]);
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const half2_t h = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(pr[r], pr[r + 1]));
        hi[2 * t + (r >> 1)] = __builtin_bit_cast(uint32_t, h);
        lo[2 * t + (r >> 1)] = __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_pkrtz(pr[r] - (float)h[0], pr[r + 1] - (float)h[1]));
      }
    }
    l += sum[0] + sum[1];
    const half8_t ph = frag(hi[0], hi[1], hi[2], hi[3]), pl = frag(lo[0], lo[1], lo[2], lo[3]);
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<(MORE ? 2 : 0) * kLoads>();  // the values
    __builtin_amdgcn_sched_barrier(0);
    u32x2 v[8];
    {
      uint32_t a[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = (vbase ^ 16 * e) + B * 2 * kStepBytes;
      lds_read_columns8(v, a);
    }
    if (masked) {
      // A value that only some rows see may be NaN, and 0 times it is NaN: such
      // values leave the product and make the rows that see them NaN.
      uint32_t nan = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) nan |= nan_codes(v[e].x) | nan_codes(v[e].y);
      if (__ballot(nan != 0)) {
#pragma unroll 1
        for (int i = 0; i < kStep; ++i) {
          const bool sees = (p + i < sp.hi) & !(bad[B] >> (i >> 4) & 1) & (p + i >= see_lo) & (p + i < see_hi);
          const uint32_t row = lds_byte(ring) + (2 * B + 1) * kStepBytes + i * kHeadDim + 4 * j;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t x = nan_codes(lds_read1(row + 16 * (e ^ ((i >> 1 & 3) | (i >> 4) << 2))));
#pragma unroll
            for (int r = 0; r < 4; ++r) o[e][r] += sees && (x >> (8 * r + 7) & 1) ? __builtin_nanf("") : 0.0f;
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u32x2{number_codes(v[e].x), number_codes(v[e].y)};
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const half8_t x = frag(values01(v[e].x, vsc[0]), values23(v[e].x, vsc[0]), values01(v[e].y, vsc[1]),
                             values23(v[e].y, vsc[1]));
      o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, ph, o[e], 0, 0, 0);
      o[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, pl, o[e], 0, 0, 0);
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
      step(b0, std::true_type{}, s, p);
      request(b0, s + 2, p + 2 * kStride);
      step(b1, std::true_type{}, s + 1, p + kStride);
    }
    if (p + kStride < sp.hi) {
      request(b1, s + 1, p + kStride);
      step(b0, std::true_type{}, s, p);
      step(b1, std::false_type{}, s + 1, p + kStride);
    } else {
      step(b0, std::false_type{}, s, p);
    }
  }

  // The waves' results, in wave order: 128 value sums per (wave, row) over the
  // ring's place, references and denominators behind it.
  l = over_quarters(l, [](float a, float b) { return a + b; });
  __syncthreads();
  float* const osum = reinterpret_cast<float*>(lds);                            // [WAVES][16][128]
  float* const stat = reinterpret_cast<float*>(lds + WAVES * 4 * kStepBytes);   // [WAVES][16][2]
#pragma unroll
  for (int e = 0; e < 8; ++e) *reinterpret_cast<float4_t*>(osum + (w * 16 + n) * kHeadDim + 16 * e + 4 * j) = o[e];
  if (j == 0) {
    stat[(w * 16 + n) * 2] = ref;
    stat[(w * 16 + n) * 2 + 1] = l;
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

// Rows of a window of the append: the least power of two up to a block's 16 with
// which the windows' waves run at once (a wave whose rows continue a block costs
// its search; one whose rows begin many blocks takes them one after another).
// Waves of a row's query heads: one where rows alone fill the chip, else one per
// group of eight.  (Measured on MI355X, kernel alone, windows of 1 / 2 / 4 / 8 /
// 16 rows: 16 decoding rows, 32:8 heads, 4.4 / 6.3 / 9.9 / 17.2 / 32 us; 1659
// rows of nine sequences and 21 of none, 28:4, 13.6 / 10.4 / 10.8 / 14.6 / 13.9;
// 16384 of four, 32:8, 224 / 221 / 132 / 97 / 78, of which 72 are the bytes as a
// large copy moves them.)
struct AppendShape {
  int64_t window, q_waves, kv_waves, waves;
};
AppendShape append_shape(int64_t T, int64_t Hq, int64_t Hkv) {
  AppendShape s;
  s.window = 1;
  while (s.window < kBlock && (T + s.window - 1) / s.window * 2 * Hkv > kResidentWaves) s.window *= 2;
  s.q_waves = std::max<int64_t>(1, std::min<int64_t>((Hq + 7) / 8, kResidentWaves / T));
  s.kv_waves = (T + s.window - 1) / s.window * 2 * Hkv;
  s.waves = s.kv_waves + T * s.q_waves;
  return s;
}

}  // namespace

int64_t paged_append_codes_threads(int64_t T, int64_t Hq, int64_t Hkv) {
  return (append_shape(T, Hq, Hkv).waves + 3) / 4 * 256;
}

hipError_t launch_paged_append_codes(const PagedCodes& pb, const uint16_t* qkv, int64_t qkv_stride, const uint16_t* qw,
                                     const uint16_t* kw, const float* cos_sin, int64_t rope_rows, int64_t Hq,
                                     int64_t Hkv, float eps, uint16_t* q_out, hipStream_t stream,
                                     const LaunchEvents& ev) {
  const AppendShape s = append_shape(pb.T, Hq, Hkv);
  launch(paged_append_codes_kernel, dim3((unsigned)((s.waves + 3) / 4)), dim3(256), 0, stream, ev, pb, qkv, qkv_stride, qw,
         kw, cos_sin, (int)std::min<int64_t>(rope_rows, 0x7FFFFFFF), (int)Hq, (int)Hkv, eps, q_out, (int)s.window,
         (int)s.q_waves, (uint32_t)s.kv_waves);
  return hipGetLastError();
}

hipError_t launch_paged_attention_codes(const PagedCodes& pb, const uint16_t* q, int64_t Hq, int64_t Hkv,
                                        int64_t window, uint16_t* out, float* ws, hipStream_t stream,
                                        const LaunchEvents& ev) {
  return launch_attention<CacheE4M3>(pb, q, Hq, Hkv, window, out, ws, stream, ev);
}

int64_t paged_attention_codes_workspace(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  return attention_plan<CacheE4M3>(B, T, Hq / Hkv, Hkv, capacity).floats * (int64_t)sizeof(float);
}

int64_t paged_attention_codes_threads(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  const AttentionPlan p = attention_plan<CacheE4M3>(B, T, Hq / Hkv, Hkv, capacity);
  return p.items * Hkv * (p.rows == kSmallRows ? 64 * kWaves : 2 * p.rows);
}

}  // namespace laq

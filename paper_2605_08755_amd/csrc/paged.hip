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
#include "paged_attention.h"

namespace laq {

namespace {

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
constexpr int kStep = 32;
constexpr int kRowBytes = (kStep + 4) * 4;         // a row of probabilities (4 words of padding)
constexpr int kKeyBytes = kStep * kHeadDim * 2;    // a step's keys
// Keys and values pass once: loads that do not keep their lines (measured on
// MI355X, three sequences of 131072, 77777 and 901 positions, 64:8 heads: 167 ->
// 151 us; 16 sequences of up to 8192, 32:8: 44 -> 39).
constexpr int kStreamed = 2;
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

struct CacheF16 {
  typedef PagedBatch Batch;
  static constexpr int kBytes = 2;
  static int split_from(int64_t, int64_t) { return 0; }
  static constexpr bool kTileRanges = false;
  static constexpr bool kFourWaves = false;
  static bool four_waves(int64_t) { return false; }
  template <int WAVES>
  static constexpr int kItemLds = WAVES * (2 * kKeyBytes + 16 * kRowBytes);
  template <int WAVES, int REC>
  static __device__ __forceinline__ void rows16_item(const PagedBatch& pb, const uint16_t* __restrict__ q, int R,
                                                     int window, const Out& o_, const Item& it, int g, char* lds);
};

// An item of up to 16 rows, by a block of WAVES waves; REC: rows that a record has room for.
template <int WAVES, int REC>
__device__ __forceinline__ void CacheF16::rows16_item(const PagedBatch& pb, const uint16_t* __restrict__ q, int R, int window,
                                            const Out& o_, const Item& it, int g, char* lds) {
  typedef __attribute__((address_space(3))) void lds_void;
  constexpr int kStride = WAVES * kStep;
  const int lane = threadIdx.x & 63;
  const int w = uniform(threadIdx.x >> 6);
  const int n = lane & 15, j = lane >> 4;
  const int rows = min(it.n * R - it.tile * kSmallRows, kSmallRows);
  const int r0 = it.tile * kSmallRows;
  const Span sp = span_of<kTileRanges>(it, uniform(r0 / R), uniform((r0 + rows - 1) / R), window);

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
  const char* const khead = reinterpret_cast<const char*>(pb.k + g * pb.head_stride);
  const char* const vhead = reinterpret_cast<const char*>(pb.v + g * pb.head_stride);
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
    const Rows16 at[2] = {rows16<2>(pb, pg[0], p, sp.hi), rows16<2>(pb, pg[1], p + 16, sp.hi)};
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
  return attention_plan<CacheF16>(B, T, Hq / Hkv, Hkv, capacity).floats * (int64_t)sizeof(float);
}

int64_t paged_attention_threads(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  const AttentionPlan p = attention_plan<CacheF16>(B, T, Hq / Hkv, Hkv, capacity);
  return p.items * Hkv * (p.rows == kSmallRows ? 64 * kWaves : 512);
}

hipError_t launch_paged_attention(const PagedBatch& pb, const uint16_t* q, int64_t Hq, int64_t Hkv, int64_t window,
                                  uint16_t* out, float* ws, hipStream_t stream, const LaunchEvents& ev) {
  return launch_attention<CacheF16>(pb, q, Hq, Hkv, window, out, ws, stream, ev);
}

}  // namespace laq

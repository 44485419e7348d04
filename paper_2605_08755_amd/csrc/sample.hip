// Sampling of the next tokens from the LM head's logits: temperature, top-k,
// top-p and min-p, and the draw by a given uniform number, in one kernel.
//
// With tokens ordered by logit (largest first, equal ones by index) and
// weights w = exp((logit - largest) / temperature), what top-k, top-p and
// min-p keep is a prefix of that order, and the draw is the first token at
// which the running weight passes u times the prefix's weight.  fp16 logits
// take at most 65536 values, so a histogram of them is the order: the prefixes
// and the draw are found among counts, with one exponential per value instead
// of one per token, and in 64 bits (a running sum over 150 000 tokens in 32
// bits moves a border by whole tokens).  Counting is in whole numbers, sums
// are added in a fixed order: the same token on every call.
//
// One block of 1024 threads per row, the logits in its registers (read once).
// What bounds a row: the passes over its logits, about a microsecond of one
// compute unit per vector instruction and 150 000 logits; so the logits are
// turned into sortable numbers in place, two per instruction, and the
// histogram holds two 16-bit counts per LDS word (all 65536 values in 128 KiB).
#include <limits.h>
#include <math.h>

#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kThreads = 1024;
constexpr int kWavesS = kThreads / 64;
constexpr int kWords = 32768;           // histogram words: values >= 0 in the upper halves, < 0 in the lower
constexpr int kLines = 1024;            // 64 values each, in falling order
constexpr int kLowest = -31745;         // sortable number of -inf (and of NaN)
constexpr int kHighest = 31744;         // of +inf

typedef short short2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Sortable numbers of two logits: a larger logit has a larger 16-bit integer;
// -0 is -1, +0 is 0, negative NaN lie below -inf and positive ones above +inf.
__device__ __forceinline__ uint32_t sortable(uint32_t x) {
  const short2_t s = __builtin_bit_cast(short2_t, x) >> 15;
  return x ^ (__builtin_bit_cast(uint32_t, s) & 0x7FFF7FFFu);
}
__device__ __forceinline__ int half_of(uint32_t x, int e) { return (int)(short)(uint16_t)(e ? x >> 16 : x); }
__device__ __forceinline__ double logit_of(int k) {
  const uint16_t h = (uint16_t)(k < 0 ? k ^ 0x7FFF : k);
  return (double)__builtin_bit_cast(_Float16, h);
}
// Values in falling order: place b = 32767 - k, line b / 64.
__device__ __forceinline__ int place_of(int k) { return 32767 - k; }
__device__ __forceinline__ int value_at(int b) { return 32767 - b; }

// 2^y for y <= 0, to about 2^-50 of it: y = n + f, |f| <= 1/2, and the series
// of exp(f ln 2), of which the term after the last is below 1e-14.
__device__ __forceinline__ double exp2_neg(double y) {
  y = fmax(y, -2000.0);
  const double n = rint(y);
  const double f = (y - n) * 0.69314718055994530942;
  double r = 1.0 / 39916800.0;
  r = fma(r, f, 1.0 / 3628800.0);
  r = fma(r, f, 1.0 / 362880.0);
  r = fma(r, f, 1.0 / 40320.0);
  r = fma(r, f, 1.0 / 5040.0);
  r = fma(r, f, 1.0 / 720.0);
  r = fma(r, f, 1.0 / 120.0);
  r = fma(r, f, 1.0 / 24.0);
  r = fma(r, f, 1.0 / 6.0);
  r = fma(r, f, 0.5);
  r = fma(r, f, 1.0);
  r = fma(r, f, 1.0);
  return ldexp(r, (int)n);
}

template <int CTRL>
__device__ __forceinline__ int dpp_s(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false);
}
__device__ __forceinline__ double lane_double(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(u >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int CTRL>
__device__ __forceinline__ double dpp_double(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = dpp_s<CTRL>((int)(uint32_t)u), hi = dpp_s<CTRL>((int)(u >> 32));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive prefix sums over the 64 lanes (shifts within 16-lane rows, lanes
// shifted in read 0; then the rows' totals).
__device__ __forceinline__ void wave_scan(double& v, int& c, int lane) {
  v += dpp_double<0x111>(v), c += dpp_s<0x111>(c);
  v += dpp_double<0x112>(v), c += dpp_s<0x112>(c);
  v += dpp_double<0x114>(v), c += dpp_s<0x114>(c);
  v += dpp_double<0x118>(v), c += dpp_s<0x118>(c);
  const double t0 = lane_double(v, 15), t1 = t0 + lane_double(v, 31), t2 = t1 + lane_double(v, 47);
  const int c0 = __builtin_amdgcn_readlane(c, 15), c1 = c0 + __builtin_amdgcn_readlane(c, 31),
            c2 = c1 + __builtin_amdgcn_readlane(c, 47);
  v += lane < 16 ? 0.0 : lane < 32 ? t0 : lane < 48 ? t1 : t2;
  c += lane < 16 ? 0 : lane < 32 ? c0 : lane < 48 ? c1 : c2;
}

struct SampleShared {
  double line_w[kLines];
  int line_c[kLines];
  double wsum[kWavesS], weight;
  int csum[kWavesS];
  int place, nth, found;
};
constexpr int kSampleLds = kWords * 4 + (int)sizeof(SampleShared);
static_assert(kSampleLds <= 160 * 1024, "LDS of a compute unit");

template <int NV>
__global__ __launch_bounds__(kThreads) void sample_kernel(const uint16_t* __restrict__ logits, int64_t stride, int V,
                                                          const float* __restrict__ u_, const float* __restrict__ t_,
                                                          const int* __restrict__ k_, const float* __restrict__ p_,
                                                          const float* __restrict__ mp_, int* __restrict__ token,
                                                          float* __restrict__ prob) {
  extern __shared__ u32x4 sample_lds[];
  uint32_t* const bins = reinterpret_cast<uint32_t*>(sample_lds);
  SampleShared& sh = *reinterpret_cast<SampleShared*>(bins + kWords);
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int row = blockIdx.x;
  const uint16_t* const x = logits + row * stride;
  const int nv = (V + 8 * kThreads - 1) / (8 * kThreads);

  // Sortable numbers of the eight logits (v * 1024 + tid) * 8 .. + 7, -inf past the end.
  auto fetch = [&](int v) {
    const int64_t at = ((int64_t)v * kThreads + tid) * 8;
    u32x4 r;
    if (at + 8 <= V) {
      __builtin_memcpy(&r, x + at, 16);  // rows of an odd vocabulary are 2-byte aligned
    } else {
      uint32_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = at + i < V ? x[at + i] : 0xFC00u;
      r = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
    }
    return r;
  };
  auto to_sortable = [](u32x4 r) { return u32x4{sortable(r.x), sortable(r.y), sortable(r.z), sortable(r.w)}; };
  u32x4 keep[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) keep[v] = fetch(v);
    for (int i = tid; i < kWords / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < NV; ++v) keep[v] = to_sortable(keep[v]);
  } else {
    for (int i = tid; i < kWords / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
  }
#define LAQ_EACH_VECTOR(body)                                    \
  if constexpr (NV > 0) {                                        \
    _Pragma("unroll") for (int v = 0; v < NV; ++v) body(keep[v], v); \
  } else {                                                       \
    for (int v = 0; v < nv; ++v) body(to_sortable(fetch(v)), v);  \
  }
  auto block_max = [&](int m) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) m = max(m, __shfl_xor(m, s));
    if (lane == 0) sh.csum[w] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWavesS; ++i) m = max(m, sh.csum[i]);
    __syncthreads();
    return uni(m);
  };

  // The largest; positive NaN, which sort above it, are looked for only where there are some.
  int top;
  {
    short2_t m = {-32768, -32768};
    auto take = [&](const u32x4& r, int) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = r[i];  // (the cast takes element 0 of a vector element named in it)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(short2_t, two));
      }
    };
    LAQ_EACH_VECTOR(take)
    top = block_max(max((int)m[0], (int)m[1]));
  }
  if (top > kHighest) {
    int m = -32768;
    auto take = [&](const u32x4& r, int) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int k = half_of(r[e >> 1], e & 1);
        m = max(m, k > kHighest ? -32768 : k);
      }
    };
    LAQ_EACH_VECTOR(take)
    top = block_max(m);
  }
  if (top <= kLowest) {  // nothing allowed
    if (tid == 0) {
      token[row] = -1;
      if (prob) prob[row] = 0.0f;
    }
    return;
  }
  if (top == -1) top = 0;  // -0 counts as 0

  const float temp = t_ ? t_[row] : 1.0f;
  int pick = place_of(top), nth = 0;  // place of the drawn value, and which of its tokens
  double chance = 1.0;
  if (temp > 0.0f) {
    const double largest = logit_of(top), per = 1.4426950408889634074 / (double)temp;
    const int first_place = place_of(top);
    auto weight = [&](int b) { return b <= first_place ? 1.0 : exp2_neg((logit_of(value_at(b)) - largest) * per); };
    const int kk = k_ ? k_[row] : 0;
    const int top_k = kk > 0 ? kk : INT_MAX;

    // The histogram.  A value that occurs 65536 times carries into its
    // neighbour or out of the word: the counts then do not add up to the
    // tokens, and the values are counted again, 32 bits each, one sign at a
    // time (a row of one repeated value, say).
    int valid = 0;
    {
      auto add = [&](const u32x4& r, int) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int k = half_of(r[e >> 1], e & 1);
          if (k > kLowest && k <= kHighest) {
            ++valid;
            atomicAdd(&bins[k & 0x7FFF], k < 0 ? 1u : 0x10000u);
          }
        }
      };
      LAQ_EACH_VECTOR(add)
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) valid += __shfl_xor(valid, s);
    if (lane == 0) sh.csum[w] = valid;
    __syncthreads();
    valid = 0;
#pragma unroll
    for (int i = 0; i < kWavesS; ++i) valid += sh.csum[i];
    const uint32_t zero = bins[0], minus_zero = bins[kWords - 1] & 0xFFFFu;  // tokens of +0 and -0: one value
    __syncthreads();
    if (tid == 0 && minus_zero) {
      bins[0] = zero + (minus_zero << 16);
      bins[kWords - 1] -= minus_zero;
    }
    bool packed = (zero >> 16) + minus_zero < 65536u;
    int loaded = 2;  // sign whose values are counted (packed: both)
    __syncthreads();

    auto count_sign = [&](int neg) {  // 32-bit counts of the values >= 0 or < 0
      if (packed || loaded == neg) return;
      __syncthreads();
      for (int i = tid; i < kWords / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
#pragma unroll 1
      for (int v = 0; v < nv; ++v) {
        const u32x4 r = to_sortable(fetch(v));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          int k = half_of(r[e >> 1], e & 1);
          if (k == -1) k = 0;
          if (k > kLowest && k <= kHighest && (k < 0) == (neg != 0)) atomicAdd(&bins[k & 0x7FFF], 1u);
        }
      }
      __syncthreads();
      loaded = neg;
    };
    // Tokens of the value at place b; its sign's counts are loaded.
    auto count_at = [&](int b) {
      const int k = value_at(b);
      const uint32_t word = bins[k & 0x7FFF];
      return (int)(!packed ? word : k < 0 ? word & 0xFFFFu : word >> 16);
    };
    // Totals of the lines, a line's 64 values over the lanes of a wave; the
    // waves take every 16th line.
    auto line_totals = [&](int neg) {
      for (int j = w; j < kLines / 2; j += kWavesS) {
        const int line = neg * (kLines / 2) + j;
        const int b = line * 64 + lane;
        int c = count_at(b);
        double ws = 0.0;
        if (__ballot(c != 0)) {
          ws = c ? c * weight(b) : 0.0;
          wave_scan(ws, c, lane);
        }
        if (lane == 63) sh.line_w[line] = ws, sh.line_c[line] = c;
      }
    };
    // Thread t holds line t: counts and weights of the lines before it, and
    // with its own.
    int cbefore, cupto, ctotal;
    double wbefore, wupto, wtotal;
    auto totals = [&]() {
      for (int neg = 1; neg >= 0; --neg) {
        count_sign(neg);
        line_totals(neg);
      }
      __syncthreads();
      wupto = sh.line_w[tid];
      cupto = sh.line_c[tid];
      wave_scan(wupto, cupto, lane);
      if (lane == 63) sh.wsum[w] = wupto, sh.csum[w] = cupto;
      __syncthreads();
      double wb = 0.0;
      int cb = 0;
      ctotal = 0, wtotal = 0.0;
#pragma unroll
      for (int i = 0; i < kWavesS; ++i) {
        if (i == w) wb = wtotal, cb = ctotal;
        wtotal += sh.wsum[i];
        ctotal += sh.csum[i];
      }
      __syncthreads();
      wupto += wb;
      cupto += cb;
      // the thread before's own numbers, so that no place falls between two
      const double x = __shfl_up(wupto, 1);
      const int c = __shfl_up(cupto, 1);
      wbefore = lane ? x : wb;
      cbefore = lane ? c : cb;
    };
#pragma unroll 1
    for (;;) {
      totals();
      if (!packed || ctotal == valid) break;
      packed = false;
    }

    // The values of one line, one a lane, in the wave that holds the line.
    struct Line {
      int place, c, cb;     // the place, its count, the counts before it
      double w, wb, wupto;  // its weight, the weights before it and up to it
    };
    auto line = [&](int l) {  // l: the line's lane in this wave
      Line r;
      r.place = (w * 64 + l) * 64 + lane;
      r.c = count_at(r.place);
      r.w = r.c ? weight(r.place) : 0.0;
      double ws = r.c * r.w;
      int cs = r.c;
      wave_scan(ws, cs, lane);
      const double base = lane_double(wbefore, l);
      r.cb = __builtin_amdgcn_readlane(cbefore, l) + cs - r.c;
      r.wupto = base + ws;
      const double x = __shfl_up(r.wupto, 1);
      r.wb = lane ? x : base;
      return r;
    };
    // The first line that has tokens and for which `reached` holds: its wave
    // calls take(lane).  False where there is none.
    auto at_first = [&](bool reached, auto&& take) {
      const uint64_t m = __ballot(cupto > cbefore && reached);
      if (lane == 0) sh.csum[w] = m ? w * 64 + __ffsll((unsigned long long)m) - 1 : kLines;
      __syncthreads();
      int owner = kLines;
#pragma unroll
      for (int i = 0; i < kWavesS; ++i) owner = min(owner, sh.csum[i]);
      owner = uni(owner);
      if (owner < kLines) {
        count_sign(owner >= kLines / 2);
        if (owner >> 6 == w) take(owner & 63);
      }
      __syncthreads();
      return owner < kLines;
    };
    // The first lane of a line for which `in` holds (its last token's otherwise).
    auto first_lane = [&](const Line& r, bool in) {
      const uint64_t m = __ballot(in), any = __ballot(r.c > 0);
      return m ? __ffsll((unsigned long long)m) - 1 : 63 - __clzll((long long)any);
    };

    // What is kept: all tokens of the values before cut, cut_count of its own.
    int cut = 65536, cut_count = 0;
    double kept = wtotal;
    if (top_k < ctotal) {
      at_first(top_k <= cupto, [&](int l) {
        const Line r = line(l);
        if (lane == first_lane(r, r.c && top_k <= r.cb + r.c)) {
          sh.place = r.place;
          sh.nth = top_k - r.cb;
          sh.weight = r.wb + (top_k - r.cb) * r.w;
        }
      });
      cut = sh.place;
      cut_count = sh.nth;
      kept = sh.weight;
      __syncthreads();
    }
    bool narrowed = false;
    const float pf = p_ ? p_[row] : 1.0f;
    if (pf < 1.0f) {
      const double target = fmax((double)pf, 0.0) * kept;
      const bool found = at_first(wupto >= target, [&](int l) {
        const Line r = line(l);
        if (lane == first_lane(r, r.c && r.wupto >= target)) {
          // the smallest count whose weight reaches the target
          double c = fmin(fmax(ceil((target - r.wb) / r.w), 1.0), (double)r.c);
          if (c > 1.0 && r.wb + (c - 1.0) * r.w >= target) c -= 1.0;
          if (c < r.c && r.wb + c * r.w < target) c += 1.0;
          sh.place = r.place;
          sh.nth = (int)c;
          sh.weight = r.wb + c * r.w;
        }
      });
      const int b = sh.place, c = sh.nth;
      const double wt = sh.weight;
      __syncthreads();
      if (found && (b < cut || (b == cut && c < cut_count))) cut = b, cut_count = c, kept = wt;
    }
    const float mp = mp_ ? mp_[row] : 0.0f;
    if (mp > 0.0f) {
      // The last value with a weight of min-p: near the inverse, then by the weights themselves.
      const double least = fmin((double)mp, 1.0);
      int b = first_place;
      if (largest < INFINITY) {
        const double edge = fmax(largest + (double)temp * log(least), -65504.0);
        const int k = half_of(sortable(__builtin_bit_cast(uint16_t, (_Float16)(float)edge)), 0);
        const int end = place_of(kLowest) - 1;
        b = min(max(place_of(k), first_place), end);
        while (b > first_place && weight(b) < least) --b;
        while (b < end && weight(b + 1) >= least) ++b;
      }
      if (b + 1 <= cut) cut = b + 1, cut_count = 0, narrowed = true;
    }
    if (narrowed) {  // the weight of all values before cut
      const int b = cut - 1, owner = b >> 6;
      count_sign(owner >= kLines / 2);
      if (w == owner >> 6) {
        const Line r = line(owner & 63);
        if (r.place == b) sh.weight = r.wupto;
      }
      __syncthreads();
      kept = sh.weight;
      __syncthreads();
    }
    // The draw.
    const float uf = u_[row];
    const double target = (uf > 0.0f ? fmin((double)uf, 1.0) : 0.0) * kept;
    bool drawn = at_first(wupto > target, [&](int l) {
      const Line r = line(l);
      if (lane == first_lane(r, r.c && r.wupto > target)) {
        double c = fmin(fmax(floor((target - r.wb) / r.w), 0.0), (double)(r.c - 1));
        if (c > 0.0 && r.wb + c * r.w > target) c -= 1.0;
        if (c + 1.0 < r.c && r.wb + (c + 1.0) * r.w <= target) c += 1.0;
        sh.place = r.place;
        sh.nth = (int)c;
        sh.weight = r.w;
      }
    });
    if (drawn) pick = sh.place, nth = sh.nth, chance = sh.weight / kept;
    __syncthreads();
    if (!drawn || pick > cut || (pick == cut && nth >= cut_count)) {
      // u = 1, or a border met by rounding: the last token kept
      if (cut_count > 0) {
        pick = cut, nth = cut_count - 1;
      } else {
        pick = first_place, nth = 0;
        for (int neg = 1; neg >= 0; --neg) {
          count_sign(neg);
          int mine = -1;
          for (int i = 0; i < kWords / kThreads; ++i) {
            const int b = neg * kWords + tid * (kWords / kThreads) + i;
            if (b < cut && count_at(b)) mine = b;
          }
          mine = block_max(mine);
          if (mine >= 0) {
            pick = mine;
            nth = count_at(mine) - 1;
            break;
          }
        }
      }
      chance = weight(pick) / kept;
    }
    __syncthreads();  // the histogram is done with
  }

  // The nth token of the drawn value, in the order of indices.
  const int want = value_at(pick);
  auto is_wanted = [&](int k) { return k == want || (want == 0 && k == -1); };
  if (tid == 0) sh.found = 0;
  __syncthreads();
  // Indices of the value's tokens, in any order, as far as there is room.
  int* const list = reinterpret_cast<int*>(bins);
  constexpr int kRoom = 1024;
  {
    const uint32_t both = (uint32_t)(want & 0xFFFF) | (uint32_t)want << 16;
    ushort2_t least = {0xFFFF, 0xFFFF};
    auto differ = [&](const u32x4& r, int) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        least = __builtin_elementwise_min(least, __builtin_bit_cast(ushort2_t, r[i] ^ both));
    };
    bool any = want == 0;
    if (!any) {
      LAQ_EACH_VECTOR(differ)
      any = least[0] == 0 || least[1] == 0;
    }
    if (any) {
      auto note = [&](const u32x4& r, int v) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (is_wanted(half_of(r[e >> 1], e & 1))) {
            const int at = atomicAdd(&sh.found, 1);
            if (at < kRoom) list[at] = (v * kThreads + tid) * 8 + e;
          }
      };
      LAQ_EACH_VECTOR(note)
    }
  }
  __syncthreads();
  const int found = sh.found;
  if (found <= kRoom) {
    // a thread per token: its rank among them
    if (tid < found) {
      const int mine = list[tid];
      int rank = 0;
      for (int i = 0; i < found; ++i) rank += list[i] < mine ? 1 : 0;
      if (rank == nth) {
        token[row] = mine;
        if (prob) prob[row] = (float)chance;
      }
    }
    return;
  }
  // Many: counts per vector and wave, then that wave's 512 logits.
  __syncthreads();
  int* const per_wave = reinterpret_cast<int*>(bins);
#pragma unroll 1
  for (int v = 0; v < nv; ++v) {
    const u32x4 r = to_sortable(fetch(v));
    int c = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) c += __popcll(__ballot(is_wanted(half_of(r[e >> 1], e & 1))));
    if (lane == 0) per_wave[v * kWavesS + w] = c;
  }
  __syncthreads();
  if (w > 0) return;
  int before = 0;
  for (int i0 = 0; i0 < nv * kWavesS; i0 += 64) {
    const int c = i0 + lane < nv * kWavesS ? per_wave[i0 + lane] : 0;
    int up = c;
    double unused = 0.0;
    wave_scan(unused, up, lane);
    const uint64_t m = __ballot(before + up > nth);
    if (m) {
      const int l = __ffsll((unsigned long long)m) - 1;
      const int rest = nth - (before + __builtin_amdgcn_readlane(up - c, l));
      const int v = (i0 + l) / kWavesS, ww = (i0 + l) % kWavesS;
      const int64_t at = ((int64_t)v * kThreads + ww * 64 + lane) * 8;
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < V && is_wanted(half_of(sortable(x[at + e]), 0))) mask |= 1u << e;
      const int own = __popc(mask);
      int sum = own;
      wave_scan(unused, sum, lane);
      if (sum - own <= rest && rest < sum) {
        for (int i = rest - (sum - own); i > 0; --i) mask &= mask - 1;
        token[row] = (int)(at + __ffs((int)mask) - 1);
        if (prob) prob[row] = (float)chance;
      }
      return;
    }
    before += __builtin_amdgcn_readlane(up, 63);
  }
#undef LAQ_EACH_VECTOR
}

}  // namespace

hipError_t launch_sample(const uint16_t* logits, int64_t stride, int64_t rows, int64_t V, const float* u,
                         const float* temperature, const int* top_k, const float* top_p, const float* min_p, int* token,
                         float* prob, hipStream_t stream, const LaunchEvents& ev) {
  const dim3 grid((unsigned)rows), block(kThreads);
  const int64_t nv = (V + 8 * kThreads - 1) / (8 * kThreads);
#define LAQ_SAMPLE(NV)                                                                                             \
  launch(sample_kernel<NV>, grid, block, kSampleLds, stream, ev, logits, stride, (int)V, u, temperature, top_k, top_p, \
         min_p, token, prob)
  // Logits stay in registers where the row fits: 19 vectors of eight a thread.
  if (nv <= 1) LAQ_SAMPLE(1);
  else if (nv <= 4) LAQ_SAMPLE(4);
  else if (nv <= 10) LAQ_SAMPLE(10);
  else if (nv <= 19) LAQ_SAMPLE(19);
  else LAQ_SAMPLE(0);
#undef LAQ_SAMPLE
  return hipGetLastError();
}

}  // namespace laq

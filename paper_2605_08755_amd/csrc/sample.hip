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
// One block of 1024 threads per row, two passes over its logits: the histogram
// (two 16-bit counts per LDS word, so that all 65536 values fit one compute
// unit) and, once a value is drawn, the search for its index.  What bounds a
// row: the LDS additions of the first pass (14 of its 31 us at 151936 logits,
// one addition of a wave about every 13 cycles), and the instruction fetch of
// code that runs once, so loops stay rolled.  (Measured on MI355X, one row of
// 151936: the row held in registers and every pass unrolled 48 us, rolled and
// read twice 33, with words and increments of two logits at a time 31.)  A
// row does not split over compute units: up to 256 rows cost little more than
// one (64 rows of 151936: 35 us; 256 of 32003: 26), and a decode step has one
// sampling call per token beside its some hundred other launches.

#include <limits.h>
#include <math.h>

#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kThreads = 1024;
constexpr int kWavesS = kThreads / 64;
constexpr int kWords = 32768;           // histogram words: values >= 0 in the upper halves, < 0 in the lower
constexpr int kBinWords = kWords + kWords / 64;  // a word of padding per 64: a lane per line reads without conflicts
constexpr int kLines = 1024;            // 64 values each, in falling order
constexpr int kLowest = -31745;         // sortable number of -inf (and of NaN)
constexpr int kHighest = 31744;         // of +inf

typedef short short2_t __attribute__((ext_vector_type(2)));
typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) uint32_t lds_word;

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

// 2^y for y <= 0, to 2^-46 of it: y = n + f, |f| <= 1/2, and the series of
// exp(f ln 2), of which what is left out is below 9e-15.
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
  double wsum[kWavesS], weight;
  int csum[kWavesS], valid[kWavesS];
  int place, nth, found;
  uint32_t aside[64];
};
constexpr int kSampleLds = kBinWords * 4 + (int)sizeof(SampleShared);
static_assert(kSampleLds <= 160 * 1024, "LDS of a compute unit");

__device__ __forceinline__ int bin_word(int word) { return word + (word >> 6); }

__global__ __launch_bounds__(kThreads) void sample_kernel(const uint16_t* __restrict__ logits, int64_t stride, int V,
                                                          const float* __restrict__ u_, const float* __restrict__ t_,
                                                          const int* __restrict__ k_, const float* __restrict__ p_,
                                                          const float* __restrict__ mp_, int* __restrict__ token,
                                                          float* __restrict__ prob) {
  extern __shared__ u32x4 sample_lds[];
  uint32_t* const bins = reinterpret_cast<uint32_t*>(sample_lds);
  SampleShared& sh = *reinterpret_cast<SampleShared*>(bins + kBinWords);
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int row = blockIdx.x;
  const uint16_t* const x = logits + row * stride;
  const int whole = V >> 3;                               // vectors of eight logits; the last V % 8 come singly
  const int nv = (whole + kThreads - 1) / kThreads;       // a thread's vectors: v * 1024 + tid
  constexpr uint32_t kNone = 0xFC00FC00u;                 // -inf twice

  auto load = [&](int v) {
    const int at = v * kThreads + tid;
    u32x4 r = {kNone, kNone, kNone, kNone};
    if (at < whole) __builtin_memcpy(&r, x + (int64_t)at * 8, 16);  // rows of an odd vocabulary: 2-byte aligned
    return r;
  };
  // f(eight logits, index of the first) over this thread's logits, AHEAD
  // vectors loaded while as many are computed; -inf past the end.
  auto each_vector = [&](auto ahead, auto&& f) {
    constexpr int AHEAD = decltype(ahead)::value;
    const int last = V & ~7;
    const uint32_t single = tid < V - last ? x[last + tid] : kNone & 0xFFFFu;
    u32x4 r[AHEAD], next[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) r[i] = load(i);
#pragma unroll 1
    for (int v0 = 0; v0 < nv; v0 += AHEAD) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) next[i] = load(v0 + AHEAD + i);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) f(r[i], ((v0 + i) * kThreads + tid) * 8);
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) r[i] = next[i];
    }
    f(u32x4{single | (kNone & 0xFFFF0000u), kNone, kNone, kNone}, last + tid);
  };
  // f(sortable numbers of two logits).
  auto each_pair = [&](auto ahead, auto&& f) {
    each_vector(ahead, [&](const u32x4& r, int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(sortable(r[e]));
    });
  };
  constexpr std::integral_constant<int, 5> counted;
  constexpr std::integral_constant<int, 10> searched;  // (little to compute: more loads on their way)
  constexpr std::integral_constant<int, 1> rare;
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

  // The histogram, the largest value and the number of tokens.  Words and signs
  // are formed for two logits at once; then per logit a 16-bit dot product
  // gives the address, a byte permutation the increment of its half, and one
  // comparison (of the upper logit as the whole pair) sends -inf to a word of
  // its lane's own.  (A separate path for vectors without -inf: 1 us less per
  // row of 151936, 1.4 us more where most logits are -inf; additions left out
  // instead of sent aside: 1 us more.)
  for (int i = tid; i < kBinWords / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
  __syncthreads();
  int valid = 0, top;
  {
    short2_t m = {-32768, -32768};
    const uint32_t base = (uint32_t)(uintptr_t)(lds_word*)bins;
    const uint32_t aside = base + (uint32_t)((sh.aside - bins) + lane) * 4;
    auto bump = [&](uint32_t at, uint32_t what) {
      __hip_atomic_fetch_add((lds_word*)at, what, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    };
    each_pair(counted, [&](uint32_t two) {
      m = __builtin_elementwise_max(m, __builtin_bit_cast(short2_t, two));
      const ushort2_t word = __builtin_bit_cast(ushort2_t, two & 0x7FFF7FFFu);
      const ushort2_t at = word + (word >> 6);  // bin_word()
      const uint32_t neg = __builtin_bit_cast(uint32_t, __builtin_bit_cast(short2_t, two) >> 15);
      // bytes of 0 and 1: (value < 0, value >= 0) of the lower logit, then of the upper
      const uint32_t which = (neg & 0x01010101u) ^ 0x01000100u;
      const uint32_t lo = __builtin_amdgcn_udot2(at, ushort2_t{4, 0}, base, false);
      const uint32_t hi = __builtin_amdgcn_udot2(at, ushort2_t{0, 4}, base, false);
      const bool in_lo = (short)(uint16_t)two > (short)kLowest, in_hi = (int)two >= (kLowest + 1) * 65536;
      valid += __popcll(__ballot(in_lo)) + __popcll(__ballot(in_hi));
      bump(in_lo ? lo : aside, __builtin_amdgcn_perm(0u, which, 0x0C010C00u));
      bump(in_hi ? hi : aside, __builtin_amdgcn_perm(0u, which, 0x0C030C02u));
    });
    if (lane == 0) sh.valid[w] = valid;
    top = block_max(max((int)m[0], (int)m[1]));
  }
  const bool nan = top > kHighest;  // positive NaN, which sort above +inf: their counts are taken out
  if (nan) {
    int m = -32768;
    valid = 0;
    each_pair(rare, [&](uint32_t two) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = half_of(two, e);
        m = max(m, k > kHighest ? -32768 : k);
        valid += __popcll(__ballot(k > kLowest && k <= kHighest));
      }
    });
    if (lane == 0) sh.valid[w] = valid;
    top = block_max(m);
    for (int k = kHighest + 1 + tid; k < kWords; k += kThreads) bins[bin_word(k)] &= 0xFFFFu;
    __syncthreads();
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

    // A value that occurs 65536 times carries into its neighbour or out of the
    // word: the counts then do not add up to the tokens, and the values are
    // counted again, 32 bits each, one sign at a time (a row of one repeated
    // value, say).
    valid = 0;
#pragma unroll
    for (int i = 0; i < kWavesS; ++i) valid += sh.valid[i];
    const uint32_t zero = bins[0], minus_zero = bins[bin_word(kWords - 1)] & 0xFFFFu;  // tokens of +0 and -0: one value
    __syncthreads();
    if (tid == 0 && minus_zero) {
      bins[0] = zero + (minus_zero << 16);
      bins[bin_word(kWords - 1)] -= minus_zero;
    }
    bool packed = (zero >> 16) + minus_zero < 65536u;
    int loaded = 2;  // sign whose values are counted (packed: both)
    __syncthreads();

    auto count_sign = [&](int neg) {  // 32-bit counts of the values >= 0 or < 0
      if (packed || loaded == neg) return;
      __syncthreads();
      for (int i = tid; i < kBinWords / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
      each_pair(rare, [&](uint32_t two) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          int k = half_of(two, e);
          if (k == -1) k = 0;
          if (k > kLowest && k <= kHighest && (k < 0) == (neg != 0)) atomicAdd(&bins[bin_word(k & 0x7FFF)], 1u);
        }
      });
      __syncthreads();
      loaded = neg;
    };
    // Tokens of value k; its sign's counts are loaded.
    auto count_of = [&](int k) {
      const uint32_t word = bins[bin_word(k & 0x7FFF)];
      return (int)(word >> (packed && k >= 0 ? 16 : 0) & (packed ? 0xFFFFu : ~0u));
    };
    auto count_at = [&](int b) { return count_of(value_at(b)); };
    // Thread t holds line t: counts and weights of the lines before it, and
    // with its own.
    int cbefore, cupto = 0, ctotal;
    double wbefore, wupto = 0.0, wtotal;
    // The lines' own, a thread per line.  A line's 64 values share an
    // exponent, so they are evenly spaced and their weights a geometric series:
    // summed from its end, a multiplication and an addition per value and two
    // exponentials per line.  In the line of the largest logit the series
    // starts there (weight 1 to the bit).
    auto line_total = [&]() {
      const int k0 = value_at(tid * 64);
      const int e = (k0 < 0 ? ~k0 : k0) >> 10 & 31;
      const double ratio = exp2_neg(-ldexp(per, max(e, 1) - 25));
      const int stop = tid == first_place >> 6 ? first_place & 63 : -64;
      const double first = tid <= first_place >> 6 ? 1.0 : exp2_neg((logit_of(k0) - largest) * per);
      const uint32_t* const words = bins + bin_word((k0 & 0x7FFF) - 63);  // of the line's last value
      const int shift = packed && k0 >= 0 ? 16 : 0;
      const uint32_t mask = packed ? 0xFFFFu : ~0u;
      double sum = 0.0;
      int c = 0;
#pragma unroll 1
      for (int j = 0; j < 64; j += 16) {  // j: places before the line's last
        int n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = (int)(words[j + i] >> shift & mask);
        if (63 - j - 15 >= stop) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            c += n[i];
            sum = fma(sum, ratio, (double)n[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            c += n[i];
            if (63 - j - i >= stop) sum = fma(sum, ratio, (double)n[i]);
          }
        }
      }
      wupto = sum * first;
      cupto = c;
    };
    auto totals = [&]() {
#pragma unroll 1
      for (int neg = 1; neg >= 0; --neg) {  // packed: both signs at once
        count_sign(neg);
        if (packed ? neg == 1 : (tid >= kLines / 2) == (neg == 1)) line_total();
      }
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

    // What is kept is the first kept_n tokens in order, of weight kept.  Up to
    // five places are looked for, each in the line (found among the threads'
    // sums) and then among the line's values, one a lane of the line's wave:
    //   0  top-k: token number top_k
    //   1  top-p: the first token at which the weight reaches top_p x kept
    //   2  min-p: the last value with that weight
    //   3  the draw: the first token at which the weight passes u x kept
    //   4  where that is past the last kept token (u = 1, or a border met by
    //      rounding): the last kept token
    const float pf = p_ ? p_[row] : 1.0f, mp = mp_ ? mp_[row] : 0.0f, uf = u_[row];
    int kept_n = ctotal;
    double kept = wtotal;
#pragma unroll 1
    for (int step = 0; step < 5; ++step) {
      int number = 0, place = 0;
      double target = 0.0;
      if (step == 0) {
        if (top_k >= ctotal) continue;
        number = top_k;
      } else if (step == 1) {
        if (!(pf < 1.0f)) continue;
        target = fmax((double)pf, 0.0) * kept;
      } else if (step == 2) {
        if (!(mp > 0.0f)) continue;
        // near the inverse, then by the weights themselves
        const double least = fmin((double)mp, 1.0);
        place = first_place;
        if (largest < INFINITY) {
          const double edge = fmax(largest + (double)temp * log(least), -65504.0);
          const int end = place_of(kLowest) - 1;
          const int k = half_of(sortable(__builtin_bit_cast(uint16_t, (_Float16)(float)edge)), 0);
          place = min(max(place_of(k), first_place), end);
          while (place > first_place && weight(place) < least) --place;
          while (place < end && weight(place + 1) >= least) ++place;
        }
        place = uni(place);
      } else if (step == 3) {
        target = (uf > 0.0f ? fmin((double)uf, 1.0) : 0.0) * kept;
      } else {
        number = kept_n;
      }
      const bool by_number = step == 0 || step == 4;
      const bool reached = by_number ? number <= cupto : step == 1 ? wupto >= target : wupto > target;
      const uint64_t m = __ballot(step == 2 ? tid == place >> 6 : cupto > cbefore && reached);
      if (lane == 0) sh.csum[w] = m ? w * 64 + __ffsll((unsigned long long)m) - 1 : kLines;
      __syncthreads();
      int owner = kLines;
#pragma unroll
      for (int i = 0; i < kWavesS; ++i) owner = min(owner, sh.csum[i]);
      owner = uni(owner);
      if (owner == kLines) {  // past every weight
        __syncthreads();
        continue;
      }
      count_sign(owner >= kLines / 2);
      if (owner >> 6 == w) {
        const int b = owner * 64 + lane, l = owner & 63;
        const int c = count_at(b);
        const double wt = c ? weight(b) : 0.0;
        double ws = c * wt;
        int cs = c;
        wave_scan(ws, cs, lane);
        const double base = lane_double(wbefore, l), upto = base + ws;
        const double below = __shfl_up(upto, 1), wb = lane ? below : base;
        const int cu = __builtin_amdgcn_readlane(cbefore, l) + cs, cb = cu - c;
        const bool in = by_number ? number <= cu : step == 1 ? upto >= target : upto > target;
        const uint64_t at = __ballot(c > 0 && in), any = __ballot(c > 0);
        const int mine = step == 2 ? place & 63 : at ? __ffsll((unsigned long long)at) - 1 : 63 - __clzll((long long)any);
        if (lane == mine) {
          int n = c;  // tokens of this value up to the place
          if (by_number) {
            n = number - cb;
          } else if (step == 1) {  // the smallest count whose weight reaches the target
            double t = fmin(fmax(ceil((target - wb) / wt), 1.0), (double)c);
            if (t > 1.0 && wb + (t - 1.0) * wt >= target) t -= 1.0;
            if (t < c && wb + t * wt < target) t += 1.0;
            n = (int)t;
          } else if (step == 3) {  // the smallest whose weight passes it
            double t = fmin(fmax(floor((target - wb) / wt), 0.0), (double)(c - 1));
            if (t > 0.0 && wb + t * wt > target) t -= 1.0;
            if (t + 1.0 < c && wb + (t + 1.0) * wt <= target) t += 1.0;
            n = (int)t + 1;
          }
          sh.place = b;
          sh.nth = n;
          sh.found = cb + n;
          sh.weight = wb + n * wt;
        }
      }
      __syncthreads();
      const int n = sh.found;
      if (step < 3) {
        if (step == 0 || n < kept_n) kept_n = n, kept = sh.weight;
      } else if (n <= kept_n) {
        pick = sh.place;
        nth = sh.nth - 1;
        break;
      }
      __syncthreads();
    }
    chance = weight(pick) / kept;
    __syncthreads();  // the histogram is done with
  }

  // The nth token of the drawn value, in the order of indices.
  const int want = value_at(pick);
  // as the logits' own bits, the sign of zeros apart
  const uint32_t bits = (uint32_t)(want < 0 ? want ^ 0x7FFF : want) & 0xFFFFu;
  const uint32_t both = bits | bits << 16, mask = want == 0 ? 0x7FFF7FFFu : ~0u;
  auto is_wanted = [&](uint32_t logit) { return ((logit ^ bits) & mask & 0xFFFFu) == 0; };
  if (tid == 0) sh.found = 0;
  __syncthreads();
  // Indices of the value's tokens, in any order, as far as there is room.
  int* const list = reinterpret_cast<int*>(bins);
  constexpr int kRoom = 1024;
  each_vector(searched, [&](const u32x4& r, int at) {
    ushort2_t least = {0xFFFF, 0xFFFF};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      least = __builtin_elementwise_min(least, __builtin_bit_cast(ushort2_t, (r[e] & mask) ^ both));
    if (least[0] == 0 || least[1] == 0) {
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const uint32_t two = e < 2 ? r.x : e < 4 ? r.y : e < 6 ? r.z : r.w;
        if (is_wanted(two >> (16 * (e & 1)))) {
          const int i = atomicAdd(&sh.found, 1);
          if (i < kRoom) list[i] = at + e;
        }
      }
    }
  });
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
  // Many: counts per wave of a thousand consecutive logits at a time, then the
  // logit itself.
  int before = 0;
#pragma unroll 1
  for (int64_t i0 = 0; i0 < V; i0 += kThreads) {
    const int64_t i = i0 + tid;
    const bool is = i < V && is_wanted(x[i]);
    const uint64_t m = __ballot(is);
    __syncthreads();
    if (lane == 0) sh.csum[w] = __popcll(m);
    __syncthreads();
    int mine = before, all = before;
#pragma unroll
    for (int k = 0; k < kWavesS; ++k) {
      if (k == w) mine = all;
      all += sh.csum[k];
    }
    if (is && mine + __popcll(m & ((1ULL << lane) - 1)) == nth) {
      token[row] = (int)i;
      if (prob) prob[row] = (float)chance;
    }
    if (nth < all) return;
    before = all;
  }
}

}  // namespace

hipError_t launch_sample(const uint16_t* logits, int64_t stride, int64_t rows, int64_t V, const float* u,
                         const float* temperature, const int* top_k, const float* top_p, const float* min_p, int* token,
                         float* prob, hipStream_t stream, const LaunchEvents& ev) {
  const dim3 grid((unsigned)rows), block(kThreads);
  launch(sample_kernel, grid, block, kSampleLds, stream, ev, logits, stride, (int)V, u, temperature, top_k, top_p, min_p,
         token, prob);
  return hipGetLastError();
}

}  // namespace laq

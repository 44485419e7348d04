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
#include <limits.h>
#include <math.h>

#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kThreads = 1024;
constexpr int kWavesS = kThreads / 64;
constexpr int kBins = 32768;                    // values counted at a time, 128 KiB of the compute unit's LDS
constexpr int kPer = kBins / kThreads;          // consecutive bins of a thread
constexpr uint32_t kLowest = 0x03FF;            // key of -inf
constexpr int kSampleLds = kBins * 4 + 1024;

__device__ __forceinline__ int uni(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Order-preserving 16-bit key of a logit; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(uint32_t h) {
  const uint32_t k = h == 0x8000u ? 0x8000u : (h & 0x8000u) ? (~h & 0xFFFFu) : (h | 0x8000u);
  return k > 0xFC00u || k < kLowest ? kLowest : k;
}
__device__ __forceinline__ double logit_of(uint32_t key) {
  const uint32_t h = (key & 0x8000u) ? (key & 0x7FFFu) : (~key & 0xFFFFu);
  return (double)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// Bin b (b-th value below the largest) sits at word b with its place within
// the line of 32 turned by the line: a thread reads a whole line, and the
// threads of a wave then read different banks.
__device__ __forceinline__ int bin_word(int b) { return b ^ ((b >> 5) & 31); }

struct SampleShared {
  double wsum[kWavesS], weight;
  int csum[kWavesS], low[kWavesS];
  int bin, nth;
};

template <int NV>
__global__ __launch_bounds__(kThreads) void sample_kernel(const uint16_t* __restrict__ logits, int64_t stride, int V,
                                                          const float* __restrict__ u_, const float* __restrict__ t_,
                                                          const int* __restrict__ k_, const float* __restrict__ p_,
                                                          const float* __restrict__ mp_, int* __restrict__ token,
                                                          float* __restrict__ prob) {
  extern __shared__ u32x4 sample_lds[];
  uint32_t* const bins = reinterpret_cast<uint32_t*>(sample_lds);
  SampleShared& sh = *reinterpret_cast<SampleShared*>(bins + kBins);
  static_assert(sizeof(SampleShared) <= 1024, "shared results");
  const int tid = threadIdx.x, lane = tid & 63, w = uni(tid >> 6);
  const int row = blockIdx.x;
  const uint16_t* const x = logits + row * stride;
  const int nv = (V + 8 * kThreads - 1) / (8 * kThreads);

  // Eight logits (v * 1024 + tid) * 8 .. + 7 as keys, -inf past the end.
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
  u32x4 keep[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) keep[v] = fetch(v);
  }
  // f(key, v, e) over this thread's logits.
  auto each_vector = [&](auto&& f) {
    if constexpr (NV > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v) f(keep[v], v);
    } else {
      for (int v = 0; v < nv; ++v) f(fetch(v), v);
    }
  };
  auto key_at = [](const u32x4& r, int e) { return key_of((r[e >> 1] >> (16 * (e & 1))) & 0xFFFFu); };

  // the largest, and the smallest that is not -inf
  uint32_t top = 0, low = 0xFFFF;
  each_vector([&](const u32x4& r, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = key_at(r, e);
      top = max(top, k);
      low = min(low, k == kLowest ? 0xFFFFu : k);
    }
  });
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) {
    top = max(top, (uint32_t)__shfl_xor((int)top, s));
    low = min(low, (uint32_t)__shfl_xor((int)low, s));
  }
  if (lane == 0) sh.csum[w] = (int)top, sh.low[w] = (int)low;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWavesS; ++i) top = max(top, (uint32_t)sh.csum[i]), low = min(low, (uint32_t)sh.low[i]);
  top = (uint32_t)uni((int)top);
  low = (uint32_t)uni((int)low);
  __syncthreads();
  if (top == kLowest) {  // nothing allowed
    if (tid == 0) {
      token[row] = -1;
      if (prob) prob[row] = 0.0f;
    }
    return;
  }
  const float temp = t_ ? t_[row] : 1.0f;
  const double largest = logit_of(top);
  int pick = 0, nth = 0;  // bin of the drawn token, and which of the bin's tokens
  double chance = 1.0;
  if (temp > 0.0f) {
    const double T = (double)temp;
    auto weight = [&](int b) { return b == 0 ? 1.0 : exp((logit_of(top - b) - largest) / T); };
    const int kk = k_ ? k_[row] : 0;
    const int top_k = kk > 0 ? kk : INT_MAX;

    // This thread's bins of each window: the counts and weights up to the
    // thread before it, and up to itself.
    int cbefore[2] = {0, 0}, cupto[2] = {0, 0};
    double wbefore[2] = {0.0, 0.0}, wupto[2] = {0.0, 0.0};
    int ctotal = 0;
    double wtotal = 0.0;
    int loaded = -1;  // window whose counts are in LDS
    auto count = [&](int win) {
      if (loaded == win) return;
      for (int i = tid; i < kBins / 4; i += kThreads) reinterpret_cast<u32x4*>(bins)[i] = u32x4{0, 0, 0, 0};
      __syncthreads();
      each_vector([&](const u32x4& r, int) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t k = key_at(r, e);
          const int b = (int)(top - k) - win * kBins;
          if (k != kLowest && b >= 0 && b < kBins) atomicAdd(&bins[bin_word(b)], 1u);
        }
      });
      __syncthreads();
      loaded = win;
    };
    auto total = [&](int win, int& call, double& wall) {
      double ws = 0.0;
      int cs = 0;
      for (int i = 0; i < kPer; ++i) {
        const int c = (int)bins[bin_word(tid * kPer + i)];
        if (c) {
          cs += c;
          ws += c * weight(win * kBins + tid * kPer + i);
        }
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const double x = __shfl_up(ws, d);
        const int c = __shfl_up(cs, d);
        if (lane >= d) ws += x, cs += c;
      }
      if (lane == 63) sh.wsum[w] = ws, sh.csum[w] = cs;
      __syncthreads();
      double wb = 0.0;
      int cb = 0;
      call = 0, wall = 0.0;
#pragma unroll
      for (int i = 0; i < kWavesS; ++i) {
        if (i == w) wb = wall, cb = call;
        wall += sh.wsum[i];
        call += sh.csum[i];
      }
      __syncthreads();
      wupto[win] = wb + ws;
      cupto[win] = cb + cs;
      // the thread before's own numbers, so that no place falls between two
      const double x = __shfl_up(wupto[win], 1);
      const int c = __shfl_up(cupto[win], 1);
      wbefore[win] = lane ? x : wb;
      cbefore[win] = lane ? c : cb;
    };
    // Values top .. top - 32767, then the rest, which top-k may not reach.
    // The first window is counted last where that is known: it is the one
    // that holds most places looked for below.
    int windows = 1, c0, c1;
    double w0, w1;
    if (top - low >= kBins && top_k == INT_MAX) {
      count(1);
      total(1, c1, w1);
      windows = 2;
    }
    count(0);
    total(0, c0, w0);
    if (top - low >= kBins && top_k != INT_MAX && top_k > c0) {
      count(1);
      total(1, c1, w1);
      windows = 2;
    }
    ctotal = c0, wtotal = w0;
    if (windows == 2) {
      cbefore[1] += c0, cupto[1] += c0;
      wbefore[1] += w0, wupto[1] += w0;
      ctotal += c1;
      wtotal = w0 + w1;
    }

    // The bins of one thread, one a lane (lanes 32 and up: none).
    struct Line {
      int bin, c, cb;      // the bin, its count, the counts before it
      double w, wb, wupto; // its weight, the weights before it and up to it
    };
    auto line = [&](int win, int l) {  // l: the owner's lane in this wave
      Line r;
      const int first = (w * 64 + l) * kPer;
      r.bin = win * kBins + first + (lane & 31);
      r.c = lane < kPer ? (int)bins[bin_word(first + (lane & 31))] : 0;
      r.w = r.c ? weight(r.bin) : 0.0;
      double ws = r.c * r.w;
      int cs = r.c;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const double x = __shfl_up(ws, d);
        const int c = __shfl_up(cs, d);
        if (lane >= d) ws += x, cs += c;
      }
      const double base = __shfl(win ? wbefore[1] : wbefore[0], l);
      r.cb = __shfl(win ? cbefore[1] : cbefore[0], l) + cs - r.c;
      r.wupto = base + ws;
      const double x = __shfl_up(r.wupto, 1);
      r.wb = lane ? x : base;
      return r;
    };
    // The first thread, in the order of values, that has tokens and for which
    // reached(window) holds: its wave calls take(window, lane) with that window's counts in
    // LDS.  False where there is none.
    auto at_first = [&](auto&& reached, auto&& take) {
      for (int win = 0; win < windows; ++win) {
        const uint64_t m = __ballot((win ? cupto[1] > cbefore[1] : cupto[0] > cbefore[0]) && reached(win));
        if (lane == 0) sh.csum[w] = m ? w * 64 + __ffsll((unsigned long long)m) - 1 : kThreads;
        __syncthreads();
        int owner = kThreads;
#pragma unroll
        for (int i = 0; i < kWavesS; ++i) owner = min(owner, sh.csum[i]);
        __syncthreads();
        if (owner == kThreads) continue;
        count(win);
        if (uni(owner >> 6) == w) take(win, owner & 63);
        __syncthreads();
        return true;
      }
      return false;
    };
    // The first lane of a line for which `in` holds (its last token's otherwise).
    auto first_lane = [&](const Line& r, bool in) {
      const uint64_t m = __ballot(in), any = __ballot(r.c > 0);
      return m ? __ffsll((unsigned long long)m) - 1 : 63 - __clzll((long long)any);
    };

    // What is kept: all tokens of the bins before cut_bin, cut_count of its own.
    int cut_bin = 65536, cut_count = 0;
    double kept = wtotal;
    if (top_k < ctotal) {
      at_first([&](int win) { return top_k <= (win ? cupto[1] : cupto[0]); },
               [&](int win, int l) {
                 const Line r = line(win, l);
                 if (lane == first_lane(r, r.c && top_k <= r.cb + r.c)) {
                   sh.bin = r.bin;
                   sh.nth = top_k - r.cb;
                   sh.weight = r.wb + (top_k - r.cb) * r.w;
                 }
               });
      cut_bin = sh.bin;
      cut_count = sh.nth;
      kept = sh.weight;
      __syncthreads();
    }
    bool narrowed = false;
    const float pf = p_ ? p_[row] : 1.0f;
    if (pf < 1.0f) {
      const double target = fmax((double)pf, 0.0) * kept;
      const bool found = at_first([&](int win) { return (win ? wupto[1] : wupto[0]) >= target; },
                                  [&](int win, int l) {
                                    const Line r = line(win, l);
                                    if (lane == first_lane(r, r.c && r.wupto >= target)) {
                                      // the smallest count whose weight reaches the target
                                      double c = fmin(fmax(ceil((target - r.wb) / r.w), 1.0), (double)r.c);
                                      if (c > 1.0 && r.wb + (c - 1.0) * r.w >= target) c -= 1.0;
                                      if (c < r.c && r.wb + c * r.w < target) c += 1.0;
                                      sh.bin = r.bin;
                                      sh.nth = (int)c;
                                    }
                                  });
      const int b = sh.bin, c = sh.nth;
      __syncthreads();
      if (found && (b < cut_bin || (b == cut_bin && c < cut_count))) cut_bin = b, cut_count = c, narrowed = true;
    }
    const float mp = mp_ ? mp_[row] : 0.0f;
    if (mp > 0.0f) {
      // The last value with a weight of min-p: near the inverse, then by the weights themselves.
      const double least = fmin((double)mp, 1.0);
      int b = 0;
      if (largest < INFINITY) {
        const double edge = fmax(largest + T * log(least), -65504.0);
        const int end = (int)(top - kLowest) - 1;
        b = (int)(top - key_of(__builtin_bit_cast(uint16_t, (_Float16)(float)edge)));
        b = min(max(b, 0), end);
        while (b > 0 && weight(b) < least) --b;
        while (b < end && weight(b + 1) >= least) ++b;
      }
      if (b + 1 <= cut_bin) cut_bin = b + 1, cut_count = 0, narrowed = true;
    }
    if (narrowed) {
      const int b = cut_count > 0 ? cut_bin : cut_bin - 1;
      const int most = cut_count > 0 ? cut_count : INT_MAX;
      const int owner = b % kBins / kPer;
      if (b / kBins < windows) {
        count(b / kBins);
        if (w == owner >> 6) {
          const Line r = line(b / kBins, owner & 63);
          if (lane < kPer && r.bin == b) sh.weight = r.wb + min(r.c, most) * r.w;
        }
        __syncthreads();
        kept = sh.weight;
        __syncthreads();
      } else {
        kept = wtotal;  // every value that was counted
      }
    }
    // The draw.
    const float uf = u_[row];
    const double target = (uf > 0.0f ? fmin((double)uf, 1.0) : 0.0) * kept;
    bool drawn = at_first([&](int win) { return (win ? wupto[1] : wupto[0]) > target; },
                          [&](int win, int l) {
                            const Line r = line(win, l);
                            if (lane == first_lane(r, r.c && r.wupto > target)) {
                              double c = fmin(fmax(floor((target - r.wb) / r.w), 0.0), (double)(r.c - 1));
                              if (c > 0.0 && r.wb + c * r.w > target) c -= 1.0;
                              if (c + 1.0 < r.c && r.wb + (c + 1.0) * r.w <= target) c += 1.0;
                              sh.bin = r.bin;
                              sh.nth = (int)c;
                            }
                          });
    if (drawn) pick = sh.bin, nth = sh.nth;
    __syncthreads();
    if (drawn && (pick > cut_bin || (pick == cut_bin && nth >= cut_count))) drawn = false;
    if (!drawn) {  // u = 1, or a border met by rounding: the last token kept
      if (cut_count > 0) {
        pick = cut_bin, nth = cut_count - 1;
      } else {
        pick = 0, nth = 0;
        for (int win = windows - 1; win >= 0; --win) {
          count(win);
          int mine = -1;
          for (int i = 0; i < kPer; ++i)
            if (win * kBins + tid * kPer + i < cut_bin && bins[bin_word(tid * kPer + i)]) mine = tid * kPer + i;
#pragma unroll
          for (int s = 32; s >= 1; s >>= 1) mine = max(mine, __shfl_xor(mine, s));
          if (lane == 0) sh.csum[w] = mine;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < kWavesS; ++i) mine = max(mine, sh.csum[i]);
          __syncthreads();
          if (mine >= 0) {
            pick = win * kBins + mine;
            nth = (int)bins[bin_word(mine)] - 1;
            break;
          }
        }
      }
    }
    chance = weight(pick) / kept;
    __syncthreads();  // the bins are done with
  }

  // The nth token with the drawn value, in the order of indices.
  const uint32_t want = top - pick;
  int* const found = reinterpret_cast<int*>(bins);  // per vector and wave; bins are done with
  each_vector([&](const u32x4& r, int v) {
    int c = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) c += __popcll(__ballot(key_at(r, e) == want));
    if (lane == 0 && v < nv) found[v * kWavesS + w] = c;
  });
  __syncthreads();
  if (w == 0) {
    int before = 0;
    for (int i0 = 0; i0 < nv * kWavesS; i0 += 64) {
      int c = i0 + lane < nv * kWavesS ? found[i0 + lane] : 0;
      int up = c;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int t = __shfl_up(up, d);
        up += lane >= d ? t : 0;
      }
      const uint64_t m = __ballot(before + up > nth);
      if (m) {
        const int l = __ffsll((unsigned long long)m) - 1;
        const int rest = nth - (before + __shfl(up - c, l));
        // that wave's 512 logits of that vector, eight a lane
        const int v = (i0 + l) / kWavesS, ww = (i0 + l) % kWavesS;
        const int64_t at = ((int64_t)v * kThreads + ww * 64 + lane) * 8;
        uint32_t mask = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at + e < V && key_of(x[at + e]) == want) mask |= 1u << e;
        const int own = __popc(mask);
        int sum = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int t = __shfl_up(sum, d);
          sum += lane >= d ? t : 0;
        }
        if (sum - own <= rest && rest < sum) {
          for (int i = rest - (sum - own); i > 0; --i) mask &= mask - 1;
          token[row] = (int)(at + __ffs((int)mask) - 1);
          if (prob) prob[row] = (float)chance;
        }
        break;
      }
      before += __shfl(up, 63);
    }
  }
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

// Logits before sampling: penalties for repeated tokens, biases of listed
// tokens and a mask (of a grammar, say), in one pass.
//
// For a token that the row's history names, with c of the mentions generated
// (the others are the prompt's):
//   x = x > 0 ? x / repetition : x * repetition
//   x = x - frequency * c - presence   (where c > 0)
// then x + bias for a listed token and -inf for one that the mask leaves out, in
// fp32, rounded to fp16 once.  What bounds it: the logits' bytes in and out
// (tokens that nothing names are copied as they are), for few rows a launch and
// the chain from the history to its counts.
//
// A block takes a range of a row's tokens and a word of LDS for each: how often
// the history names it, whether it does at all, and the last bias listed for
// it.  Every block of a row reads the whole history (from the L2 that it shares
// with others) and counts what falls in its range, so counts need no memory, no
// second kernel and no atomics beyond LDS, whose whole numbers come out the
// same in any order.
#include <algorithm>

#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kBiasShift = 20;
constexpr uint32_t kSeen = 0x80000000u;                     // named by the prompt
constexpr uint32_t kCount = (1u << kBiasShift) - 1;         // mentions among the generated tokens
constexpr uint32_t kBias = ~(kSeen | kCount) >> kBiasShift;  // 1 + place of the bias that counts

typedef unsigned short ushort8_t __attribute__((ext_vector_type(8)));

// THREADS threads take VECS vectors of eight tokens each.
template <int THREADS, int VECS>
__global__ __launch_bounds__(THREADS) void adjust_logits_kernel(Adjust a, int ranges) {
#pragma clang fp contract(off)
  extern __shared__ u32x4 adjust_lds[];
  constexpr int kTokens = 8 * THREADS * VECS;
  uint32_t* const words = reinterpret_cast<uint32_t*>(adjust_lds);
  const int tid = threadIdx.x;
  const int row = blockIdx.x / ranges, range = (int)blockIdx.x - row * ranges;
  const uint16_t* const src = a.logits + (int64_t)row * a.stride;
  uint16_t* const dst = a.out + (int64_t)row * a.out_stride;
  // Vectors start where 16 bytes of the row's logits do: tokens 8 v - shift.
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) >> 1) & 7);
  const int first = range * kTokens - shift;
  const bool wide = ((reinterpret_cast<uintptr_t>(dst) >> 1) & 7) == (uintptr_t)shift;
  const int* const mask = a.mask ? a.mask + (int64_t)row * a.mask_stride : nullptr;

  ushort8_t x[VECS];
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int t = first + 8 * (k * THREADS + tid);
    if (t >= 0 && t + 8 <= a.V) x[k] = *reinterpret_cast<const ushort8_t*>(src + t);
    else
#pragma unroll
      for (int e = 0; e < 8; ++e) x[k][e] = t + e >= 0 && t + e < a.V ? src[t + e] : (unsigned short)0;
  }
  uint32_t allowed[VECS];
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int t = first + 8 * (k * THREADS + tid);
    allowed[k] = 0xFFu;
    if (mask && t + 8 > 0 && t < a.V) {
      const int lo = max(t, 0), hi = min(t + 7, a.V - 1);
      const uint64_t m = (uint32_t)mask[lo >> 5] | (uint64_t)(uint32_t)mask[hi >> 5] << 32;
      // (both words are one where the vector lies in it; bits below token 0 fall out of the row)
      const uint32_t bits = (lo >> 5) == (hi >> 5) ? (uint32_t)m >> (lo & 31) : (uint32_t)(m >> (lo & 31));
      allowed[k] = bits << (lo - t) & 0xFFu;
    }
  }

  const bool counts = a.history != nullptr || a.bias_token != nullptr;
  if (counts) {
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      u32x4* const w = reinterpret_cast<u32x4*>(words + 8 * (k * THREADS + tid));
      w[0] = w[1] = u32x4{0, 0, 0, 0};
    }
    __syncthreads();
    if (a.bias_token) {
      const int* const listed = a.bias_token + (int64_t)row * a.bias_stride;
      for (int i = tid; i < a.biases; i += THREADS) {
        const int t = listed[i];
        const uint32_t at = (uint32_t)t - (uint32_t)first;
        if (t >= 0 && at < kTokens) atomicMax(words + at, (uint32_t)(i + 1) << kBiasShift);
      }
      __syncthreads();
    }
    if (a.history) {
      const int* const told = a.history + (int64_t)row * a.history_stride;
      const int len = min(max(a.history_len[row], 0), a.room), prompt = a.prompt_len ? a.prompt_len[row] : 0;
      auto mention = [&](int t, int i) {
        const uint32_t at = (uint32_t)t - (uint32_t)first;
        if (t < 0 || at >= kTokens) return;
        if (i < prompt) atomicOr(words + at, kSeen);
        else atomicAdd(words + at, 1u);
      };
      typedef int int4_t __attribute__((ext_vector_type(4)));
      constexpr int kAhead = 4;  // vectors in flight
      int i = 4 * tid;
      for (; i + 4 * THREADS * (kAhead - 1) + 4 <= len; i += 4 * THREADS * kAhead) {
        int4_t t[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) __builtin_memcpy(&t[k], told + i + 4 * THREADS * k, 16);  // 4-byte aligned
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) mention(t[k][e], i + 4 * THREADS * k + e);
      }
      for (; i < len; i += 4 * THREADS)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i + e < len) mention(told[i + e], i + e);
    }
    __syncthreads();
  }

  const float repetition = a.repetition ? a.repetition[row] : 1.0f;
  const float frequency = a.frequency ? a.frequency[row] : 0.0f, presence = a.presence ? a.presence[row] : 0.0f;
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int v = k * THREADS + tid, t = first + 8 * v;
    if (t + 8 <= 0 || t >= a.V) continue;
    u32x4 w[2] = {};
    if (counts) {
      const u32x4* const p = reinterpret_cast<const u32x4*>(words + 8 * v);
      w[0] = p[0], w[1] = p[1];
    }
    const u32x4 any = w[0] | w[1];
    const bool named = (any.x | any.y | any.z | any.w) != 0;
    if (a.in_place && !named && allowed[k] == 0xFFu) continue;
    if (named) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = w[e >> 2][e & 3];
        if (u == 0) continue;
        float y = (float)__builtin_bit_cast(_Float16, (unsigned short)x[k][e]);
        const uint32_t c = u & kCount, b = u >> kBiasShift & kBias;
        if (u & (kSeen | kCount)) y = y > 0.0f ? y / repetition : y * repetition;
        if (c) y = y - frequency * (float)c - presence;
        if (b) y = y + a.bias_value[(int64_t)row * a.bias_stride + b - 1];
        x[k][e] = __builtin_bit_cast(unsigned short, (_Float16)y);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[k][e] = allowed[k] >> e & 1 ? x[k][e] : (unsigned short)0xFC00;
    if (wide && t >= 0 && t + 8 <= a.V) *reinterpret_cast<ushort8_t*>(dst + t) = x[k];
    else
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (t + e >= 0 && t + e < a.V) dst[t + e] = x[k][e];
  }
}

// Tokens of a block.
int range_tokens(const Adjust& a, int64_t rows) {
  if (a.room > 16384) return 32768;
  return rows * a.V > (1 << 21) || a.room > 4096 ? 8192 : 2048;
}
int64_t ranges_of(const Adjust& a, int64_t rows) { return (a.V + 7 + range_tokens(a, rows) - 1) / range_tokens(a, rows); }

}  // namespace

int64_t adjust_logits_threads(const Adjust& a, int64_t rows) {
  return rows * ranges_of(a, rows) * std::min(range_tokens(a, rows) / 8, 1024);
}

hipError_t launch_adjust_logits(const Adjust& a, int64_t rows, hipStream_t stream, const LaunchEvents& ev) {
  const int tokens = range_tokens(a, rows);
  const int64_t ranges = ranges_of(a, rows);
  const dim3 grid((unsigned)(rows * ranges));
  const uint32_t lds = a.history || a.bias_token ? (uint32_t)tokens * 4 : 0;
  if (tokens == 2048) launch((adjust_logits_kernel<256, 1>), grid, dim3(256), lds, stream, ev, a, (int)ranges);
  else if (tokens == 8192) launch((adjust_logits_kernel<1024, 1>), grid, dim3(1024), lds, stream, ev, a, (int)ranges);
  else launch((adjust_logits_kernel<1024, 4>), grid, dim3(1024), lds, stream, ev, a, (int)ranges);
  return hipGetLastError();
}

}  // namespace laq

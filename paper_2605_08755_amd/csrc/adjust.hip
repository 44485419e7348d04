// Logits before sampling: penalties for repeated tokens, biases of listed
// tokens and a mask (of a grammar, say), in one pass.
//
// For a token that the row's history names, with c of the mentions generated
// (the others are the prompt's):
//   x = x * (x > 0 ? 1 / repetition : repetition)
//   x = x - frequency * c - presence   (where c > 0)
// then x + bias for a listed token and -inf for one that the mask leaves out, in
// fp32, rounded to fp16 once.  What bounds it: the logits' bytes in and out
// (tokens that nothing names are copied as they are), for few rows a launch and
// the chain from the history to its counts.
//
// A block takes a range of a row's tokens.  It copies their logits (masked), and
// beside that counts in LDS, a word a token: how often the history names it,
// whether it does at all, and the last bias listed for it.  Every block of a row
// reads the whole history (from the L2 that it shares with others) and counts
// what falls in its range, so counts need no memory, no second kernel and no
// atomics beyond LDS, whose whole numbers come out the same in any order.  The
// tokens that turn out named, a few in a hundred, are then listed, and their
// logits computed and written over the copies: a thread each, where a pass over
// all tokens would spend on every one what these need.  (Measured on MI355X,
// kernel alone: one row of 151936 tokens and a history of 700, 4.6 us; 64 rows,
// histories of up to 8192, 20 biases each, 13.8 us, of which the copy is 7.6, 5.2
// TB/s; 256 rows of 32003, 300 biases and a mask each, 13.5 us.)
#include "mfma_util.h"

namespace laq {

namespace {

constexpr int kListed = 4;  // tokens for which a list has one place
constexpr int kBiasShift = 20;
constexpr uint32_t kSeen = 0x80000000u;                     // named by the prompt
constexpr uint32_t kCount = (1u << kBiasShift) - 1;         // mentions among the generated tokens
constexpr uint32_t kBias = ~(kSeen | kCount) >> kBiasShift;  // 1 + place of the bias that counts

// THREADS threads take VECS vectors of eight tokens each.  Everything that a
// block reads whatever the counts come out as is requested before it waits for
// any of it: a block is a chain of memory round trips, and few run at once.
template <int THREADS, int VECS>
__global__ __launch_bounds__(THREADS) void adjust_logits_kernel(Adjust a, int rows) {
#pragma clang fp contract(off)
  extern __shared__ u32x4 adjust_lds[];
  constexpr int kTokens = 8 * THREADS * VECS;
  typedef int int4_t __attribute__((ext_vector_type(4)));
  constexpr int kShare = 512 * VECS;  // of a wave, consecutive
  uint32_t* const words = reinterpret_cast<uint32_t*>(adjust_lds);       // [kTokens]
  uint16_t* const lists = reinterpret_cast<uint16_t*>(words + kTokens);  // [kTokens / kListed]: named ones
  const int tid = threadIdx.x;
  // Blocks of a row lie `rows` apart: with a multiple of eight rows they share an
  // XCD, and its L2 the row's history.
  const int range = (int)(blockIdx.x / (unsigned)rows), row = (int)(blockIdx.x - (unsigned)range * (unsigned)rows);
  const uint16_t* const src = a.logits + (int64_t)row * a.stride;
  uint16_t* const dst = a.out + (int64_t)row * a.out_stride;
  // Vectors start where 16 bytes of the row's logits do: tokens 8 v - shift.
  const int shift = (int)((reinterpret_cast<uintptr_t>(src) >> 1) & 7);
  const int first = range * kTokens - shift;

  constexpr int kAhead = 4;  // vectors of the history in flight
  constexpr int kTurn = 4 * THREADS * kAhead;
  const int* const told = a.history ? a.history + (int64_t)row * a.history_stride : nullptr;
  int4_t t[kAhead];
  auto load_told = [&](int i) {  // this thread's vectors of a turn: whole ones inside the room
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + 4 * THREADS * k + 4 <= a.room) __builtin_memcpy(&t[k], told + i + 4 * THREADS * k, 16);  // 4-byte aligned
  };
  if (told) load_told(4 * tid);
  const int len = told ? min(max(a.history_len[row], 0), a.room) : 0;
  const int prompt = a.prompt_len ? a.prompt_len[row] : 0;
  const int* const biased = a.bias_token ? a.bias_token + (int64_t)row * a.bias_stride : nullptr;
  const int bias = biased && tid < a.biases ? biased[tid] : -1;
  const float repetition = a.repetition ? a.repetition[row] : 1.0f, inverse = 1.0f / repetition;
  const float frequency = a.frequency ? a.frequency[row] : 0.0f, presence = a.presence ? a.presence[row] : 0.0f;
  const uint32_t* const mask = a.mask ? a.mask + (int64_t)row * a.mask_stride : nullptr;

  const bool counts = told || biased;
  const int lane = tid & 63, base = __builtin_amdgcn_readfirstlane(tid >> 6) * kShare;
  const int mine = base + 8 * lane;  // this lane's vectors: tokens first + mine + 512 k
  // The copy.  In place only what the mask leaves out is written.
  const bool copies = !a.in_place || mask;
  u32x4 x[VECS];
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int at = first + mine + 512 * k;
    if (copies && at >= 0 && at + 8 <= a.V) x[k] = *reinterpret_cast<const u32x4*>(src + at);
  }
  if (counts) {
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      u32x4* const w = reinterpret_cast<u32x4*>(words + mine + 512 * k);
      w[0] = w[1] = u32x4{0, 0, 0, 0};
    }
  }
  if (copies) {
    const bool wide = ((reinterpret_cast<uintptr_t>(dst) >> 1) & 7) == (uintptr_t)shift;
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      const int at = first + mine + 512 * k;
      if (at >= 0 && at + 8 <= a.V) {
        if (mask) {
          const uint32_t bits = (uint32_t)(((uint64_t)mask[(at + 7) >> 5] << 32 | mask[at >> 5]) >> (at & 31));
          if (a.in_place && (bits & 0xFF) == 0xFF) continue;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t keep = ((uint32_t)((int)(bits << (31 - 2 * e)) >> 31) & 0xFFFFu) |
                                  (uint32_t)((int)(bits << (30 - 2 * e)) >> 31) << 16;
            x[k][e] = (x[k][e] & keep) | (0xFC00FC00u & ~keep);
          }
        }
        if (wide) *reinterpret_cast<u32x4*>(dst + at) = x[k];
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[at + e] = (uint16_t)(x[k][e >> 1] >> 16 * (e & 1));
      } else if (at + 8 > 0 && at < a.V) {  // the row's ends
#pragma unroll 1
        for (int e = max(at, 0); e < min(at + 8, a.V); ++e) {
          const bool keep = !mask || (mask[e >> 5] >> (e & 31) & 1);
          if (!a.in_place || !keep) dst[e] = keep ? src[e] : (uint16_t)0xFC00;
        }
      }
    }
  }
  if (!counts) return;

  __syncthreads();
  // (Tokens below 0 may fall on the words before the row's first, of which
  // nothing is written.)
  if (biased) {
    for (int i = tid; i < a.biases; i += THREADS) {
      const uint32_t at = (uint32_t)(i == tid ? bias : biased[i]) - (uint32_t)first;
      if (at < kTokens) atomicMax(words + at, (uint32_t)(i + 1) << kBiasShift);
    }
    __syncthreads();
  }
  auto prompted = [&](int token) {
    const uint32_t at = (uint32_t)token - (uint32_t)first;
    if (at < kTokens) atomicOr(words + at, kSeen);
  };
  auto generated = [&](int token) {
    const uint32_t at = (uint32_t)token - (uint32_t)first;
    if (at < kTokens) atomicAdd(words + at, 1u);
  };
  for (int i = 4 * tid; i < len;) {
    int4_t now[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) now[k] = t[k];
    if (i + kTurn < len) load_told(i + kTurn);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int at = i + 4 * THREADS * k;
      if (at >= prompt && at + 4 <= len) {
#pragma unroll
        for (int e = 0; e < 4; ++e) generated(now[k][e]);
      } else if (at + 4 <= min(prompt, len)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) prompted(now[k][e]);
      } else if (at < len) {  // across the prompt's end, or the history's
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (at + e >= len) break;
          const int token = at + 4 <= a.room ? now[k][e] : told[at + e];
          if (at + e < prompt) prompted(token);
          else generated(token);
        }
      }
    }
    i += kTurn;
  }
  __syncthreads();  // (and the copies are written: what follows overwrites some of them)

  auto settle = [&](int at, uint32_t u) {
    const int token = first + at;
    if (token < 0 || token >= a.V) return;
    if (mask && !(mask[token >> 5] >> (token & 31) & 1)) return;
    const uint32_t c = u & kCount, b = u >> kBiasShift & kBias;
    float y = (float)__builtin_bit_cast(_Float16, src[token]);
    if (u & (kSeen | kCount)) y = y * (y > 0.0f ? inverse : repetition);
    if (c) y = y - frequency * (float)c - presence;
    if (b) y = y + a.bias_value[(int64_t)row * a.bias_stride + b - 1];
    dst[token] = __builtin_bit_cast(uint16_t, (_Float16)y);
  };
  // Each wave lists the named ones of its share, and its lanes take them from
  // there; where more than a quarter are named, a lane takes its own.
  uint16_t* const list = lists + base / kListed;
  uint32_t some = 0;  // bit 8 k + e: this lane's word e of vector k
#pragma unroll
  for (int k = 0; k < 2 * VECS; ++k) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(words + mine + 512 * (k >> 1) + 4 * (k & 1));
#pragma unroll
    for (int e = 0; e < 4; ++e) some |= min(w[e], 1u) << (4 * k + e);
  }
  const int own = __popc(some);
  int upto = own;  // of the lanes up to this one: shifts by 1, 2, 4, 8 within 16 lanes, then the rows' totals
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xF, 0xF, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xF, 0xF, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xF, 0xF, false);
  upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xF, 0xF, false);
  const int t0 = __builtin_amdgcn_readlane(upto, 15), t1 = __builtin_amdgcn_readlane(upto, 31),
            t2 = __builtin_amdgcn_readlane(upto, 47), n = t0 + t1 + t2 + __builtin_amdgcn_readlane(upto, 63);
  upto += (lane >= 16 ? t0 : 0) + (lane >= 32 ? t1 : 0) + (lane >= 48 ? t2 : 0);
  const bool listed = n <= kShare / kListed;
  for (int place = upto - own; some != 0; ++place) {
    const int bit = __ffs(some) - 1, at = mine + 512 * (bit >> 3) + (bit & 7);
    some &= some - 1;
    if (listed) list[place] = (uint16_t)at;
    else settle(at, words[at]);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the list is the wave's own
  if (listed)
    for (int i = lane; i < n; i += 64) {
      const int at = list[i];
      settle(at, words[at]);
    }
}

// Tokens of a block: 2048 where that makes few blocks (latency counts), 16384
// where every block of a row reads a long history, else 8192.  (Measured on
// MI355X, kernel alone, 2048 / 8192 / 16384: one row of 151936 and a history of
// 700, 4.5 / 5.2 / 5.6 us; 64 rows and up to 8192, 18.7 / 14.3 / 14.2; 256 rows
// of 32003 with 300 biases and masks, 17.0 / 13.4 / 13.6; 16 rows of 151936 and
// up to 131072, 46 / 26.5 / 19.7.)
int range_tokens(const Adjust& a, int64_t rows) {
  if (a.room > 16384) return 16384;
  return rows * a.V > (1 << 21) || a.room > 4096 ? 8192 : 2048;
}
int64_t ranges_of(const Adjust& a, int64_t rows) { return (a.V + 7 + range_tokens(a, rows) - 1) / range_tokens(a, rows); }

}  // namespace

int64_t adjust_logits_threads(const Adjust& a, int64_t rows) {
  return rows * ranges_of(a, rows) * (range_tokens(a, rows) == 2048 ? 256 : range_tokens(a, rows) == 8192 ? 512 : 1024);
}

hipError_t launch_adjust_logits(const Adjust& a, int64_t rows, hipStream_t stream, const LaunchEvents& ev) {
  const int tokens = range_tokens(a, rows);
  const int64_t ranges = ranges_of(a, rows);
  const dim3 grid((unsigned)(rows * ranges));
  const uint32_t lds = a.history || a.bias_token ? (uint32_t)(tokens * 4 + tokens / kListed * 2) : 0;
  if (tokens == 2048) launch((adjust_logits_kernel<256, 1>), grid, dim3(256), lds, stream, ev, a, (int)rows);
  else if (tokens == 8192) launch((adjust_logits_kernel<512, 2>), grid, dim3(512), lds, stream, ev, a, (int)rows);
  else launch((adjust_logits_kernel<1024, 2>), grid, dim3(1024), lds, stream, ev, a, (int)rows);
  return hipGetLastError();
}

}  // namespace laq

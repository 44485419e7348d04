// C ABI of the library (include/laq.h): argument validation on the host,
// then an asynchronous launch on the caller's stream.  Nothing is enqueued
// when validation fails.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>

#include "laq.h"
#include "laq_internal.h"

namespace {

thread_local std::string g_last_error;
thread_local laq::LaunchEvents g_next_events;  // measurement hook, consumed by the next launch

laq::LaunchEvents take_events() {
  laq::LaunchEvents ev = g_next_events;
  g_next_events = laq::LaunchEvents{};
  return ev;
}

laq_status fail(laq_status st, const char* fn, const char* what) {
  char buf[256];
  std::snprintf(buf, sizeof(buf), "%s: %s", fn, what);
  g_last_error = buf;
  return st;
}

laq_status ok() {
  g_last_error.clear();
  return LAQ_OK;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

laq_status check_shape(const char* fn, int64_t N, int64_t K) {
  if (N < 1) return fail(LAQ_ERR_BAD_SHAPE, fn, "N must be >= 1");
  if (K < 128 || K % 128 != 0) return fail(LAQ_ERR_BAD_SHAPE, fn, "K must be a positive multiple of 128");
  if (N > 0x7FFFFFFFLL) return fail(LAQ_ERR_BAD_SHAPE, fn, "N must be < 2^31");
  if (K > (1LL << 24)) return fail(LAQ_ERR_BAD_SHAPE, fn, "K must be <= 2^24");
  if (N * K >= (1LL << 40)) return fail(LAQ_ERR_BAD_SHAPE, fn, "N*K must be < 2^40");
  return LAQ_OK;
}

laq_status hip_status(const char* fn, hipError_t e) {
  if (e != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e));
  return ok();
}

template <int BITS>
laq_status quantize(const char* fn, const void* w, int64_t N, int64_t K, uint32_t* qweight,
                    void* scales, uint8_t* zeros, void* stream) {
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!w || !qweight || !scales || !zeros) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (!aligned(w, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "w and qweight must be 16-byte aligned");
  if (!aligned(scales, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales must be 2-byte aligned");
  return hip_status(fn, laq::launch_quantize<BITS>(static_cast<const uint16_t*>(w), N, K, qweight,
                                                   static_cast<uint16_t*>(scales), zeros,
                                                   static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status pack(const char* fn, const void* w, const void* scales, const uint8_t* zeros, int64_t N,
                int64_t K, uint32_t* qweight, void* stream) {
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!w || !qweight || !scales || !zeros) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (!aligned(w, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "w and qweight must be 16-byte aligned");
  if (!aligned(scales, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales must be 2-byte aligned");
  return hip_status(fn, laq::launch_pack<BITS>(static_cast<const uint16_t*>(w),
                                               static_cast<const uint16_t*>(scales), zeros, N, K, qweight,
                                               static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status linear(const char* fn, const void* x, const uint32_t* qweight, const void* scales,
                  const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K, void* stream) {
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!x || !qweight || !scales || !zeros || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (M < 1 || M > LAQ_MAX_M) return fail(LAQ_ERR_BAD_M, fn, "M must be in 1..16");
  if (!aligned(x, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  return hip_status(fn, laq::launch_linear<BITS>(static_cast<const uint16_t*>(x), qweight,
                                                 static_cast<const uint16_t*>(scales), zeros,
                                                 static_cast<uint16_t*>(y), (int)M, N, K,
                                                 static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status linear_ws(const char* fn, const void* x, const uint32_t* qweight, const void* scales,
                     const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!x || !qweight || !scales || !zeros || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if (workspace_bytes < 0) return fail(LAQ_ERR_BAD_SHAPE, fn, "workspace_bytes must be >= 0");
  if (workspace_bytes > 0 && !workspace) return fail(LAQ_ERR_NULL_POINTER, fn, "null workspace with workspace_bytes > 0");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (M < 1 || M > LAQ_MAX_M) return fail(LAQ_ERR_BAD_M, fn, "M must be in 1..16");
  if (!aligned(x, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  if (workspace && !aligned(workspace, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "workspace must be 16-byte aligned");
  return hip_status(fn, laq::launch_linear<BITS>(static_cast<const uint16_t*>(x), qweight,
                                                 static_cast<const uint16_t*>(scales), zeros,
                                                 static_cast<uint16_t*>(y), (int)M, N, K,
                                                 static_cast<hipStream_t>(stream), ev,
                                                 workspace_bytes > 0 ? static_cast<float*>(workspace) : nullptr,
                                                 (size_t)workspace_bytes));
}

template <int BITS>
laq_status linear_group(const char* fn, const laq_linear_call* calls, int32_t count, int64_t M, void* stream) {
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!calls) return fail(LAQ_ERR_NULL_POINTER, fn, "null calls array");
  if (count < 1 || count > LAQ_MAX_GROUP) return fail(LAQ_ERR_BAD_SHAPE, fn, "count must be in 1..8");
  if (M < 1 || M > LAQ_MAX_M) return fail(LAQ_ERR_BAD_M, fn, "M must be in 1..16");
  laq::LinearCall lc[laq::kMaxGroup];
  int64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    const laq_linear_call& c = calls[i];
    if (!c.x || !c.qweight || !c.scales || !c.zeros || !c.y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer in a call");
    laq_status st = check_shape(fn, c.N, c.K);
    if (st != LAQ_OK) return st;
    if (!aligned(c.x, 16) || !aligned(c.qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
    if (!aligned(c.scales, 2) || !aligned(c.y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
    blocks += c.N;  // an upper bound of the grid: at least one row per block
    lc[i] = laq::LinearCall{static_cast<const uint16_t*>(c.x), c.qweight, static_cast<const uint16_t*>(c.scales),
                            c.zeros, static_cast<uint16_t*>(c.y), (int)c.N, (int)(c.K / 128), 0, 0, 0.0f};
  }
  if (blocks >= (1LL << 31)) return fail(LAQ_ERR_BAD_SHAPE, fn, "the calls' rows must total < 2^31");
  return hip_status(fn, laq::launch_linear_group<BITS>(lc, count, (int)M, static_cast<hipStream_t>(stream), ev));
}

}  // namespace

extern "C" {

int32_t laq_abi_version(void) { return LAQ_ABI_VERSION; }

const char* laq_status_string(laq_status status) {
  switch (status) {
    case LAQ_OK: return "ok";
    case LAQ_ERR_NULL_POINTER: return "null pointer argument";
    case LAQ_ERR_BAD_SHAPE: return "bad shape (need N >= 1, K >= 128, K % 128 == 0)";
    case LAQ_ERR_BAD_M: return "M outside 1..16";
    case LAQ_ERR_MISALIGNED: return "misaligned pointer";
    case LAQ_ERR_HIP: return "HIP runtime error";
    default: return "unknown status";
  }
}

const char* laq_last_error(void) { return g_last_error.c_str(); }

laq_status laq_profile_next_launch(void* start_event, void* stop_event) {
  g_next_events.start = static_cast<hipEvent_t>(start_event);
  g_next_events.stop = static_cast<hipEvent_t>(stop_event);
  return LAQ_OK;
}

laq_status laq_quantize_w3g128(const void* w, int64_t N, int64_t K, uint32_t* qweight, void* scales,
                               uint8_t* zeros, void* stream) {
  return quantize<3>("laq_quantize_w3g128", w, N, K, qweight, scales, zeros, stream);
}

laq_status laq_quantize_w4g128(const void* w, int64_t N, int64_t K, uint32_t* qweight, void* scales,
                               uint8_t* zeros, void* stream) {
  return quantize<4>("laq_quantize_w4g128", w, N, K, qweight, scales, zeros, stream);
}

laq_status laq_pack_w3g128(const void* w, const void* scales, const uint8_t* zeros, int64_t N, int64_t K,
                           uint32_t* qweight, void* stream) {
  return pack<3>("laq_pack_w3g128", w, scales, zeros, N, K, qweight, stream);
}

laq_status laq_pack_w4g128(const void* w, const void* scales, const uint8_t* zeros, int64_t N, int64_t K,
                           uint32_t* qweight, void* stream) {
  return pack<4>("laq_pack_w4g128", w, scales, zeros, N, K, qweight, stream);
}

laq_status laq_linear_w3g128(const void* x, const uint32_t* qweight, const void* scales,
                             const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K,
                             void* stream) {
  return linear<3>("laq_linear_w3g128", x, qweight, scales, zeros, y, M, N, K, stream);
}

int64_t laq_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (M < 1 || M > LAQ_MAX_M || N < 1 || N > 0x7FFFFFFFLL || K < 128 || K % 128 != 0 || K > (1LL << 24) ||
      N * K >= (1LL << 40))
    return 0;
  const laq::SplitPlan p = laq::mfma_split_plan((int)M, N, (int)(K / 128));
  return (int64_t)laq::split_workspace_bytes(p, (int)M, N);
}

laq_status laq_linear_ws_w3g128(const void* x, const uint32_t* qweight, const void* scales,
                                const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  return linear_ws<3>("laq_linear_ws_w3g128", x, qweight, scales, zeros, y, M, N, K, workspace, workspace_bytes,
                      stream);
}

laq_status laq_linear_ws_w4g128(const void* x, const uint32_t* qweight, const void* scales,
                                const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  return linear_ws<4>("laq_linear_ws_w4g128", x, qweight, scales, zeros, y, M, N, K, workspace, workspace_bytes,
                      stream);
}

laq_status laq_linear_group_w3g128(const laq_linear_call* calls, int32_t count, int64_t M, void* stream) {
  return linear_group<3>("laq_linear_group_w3g128", calls, count, M, stream);
}

laq_status laq_linear_group_w4g128(const laq_linear_call* calls, int32_t count, int64_t M, void* stream) {
  return linear_group<4>("laq_linear_group_w4g128", calls, count, M, stream);
}

laq_status laq_linear_w4g128(const void* x, const uint32_t* qweight, const void* scales,
                             const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K,
                             void* stream) {
  return linear<4>("laq_linear_w4g128", x, qweight, scales, zeros, y, M, N, K, stream);
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Decode-step operations
// ---------------------------------------------------------------------------
namespace {
constexpr int64_t kHeadDimAbi = 128;

laq_status check_heads(const char* fn, int64_t Hq, int64_t Hkv, int64_t head_dim) {
  if (head_dim != kHeadDimAbi) return fail(LAQ_ERR_BAD_SHAPE, fn, "head_dim must be 128");
  if (Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return fail(LAQ_ERR_BAD_SHAPE, fn, "Hq must be a positive multiple of Hkv");
  const int64_t r = Hq / Hkv;
  if (r != 1 && r != 2 && r != 4 && r != 8) return fail(LAQ_ERR_BAD_SHAPE, fn, "Hq / Hkv must be 1, 2, 4 or 8");
  if (Hq > 4096) return fail(LAQ_ERR_BAD_SHAPE, fn, "Hq must be <= 4096");
  return LAQ_OK;
}
}  // namespace

extern "C" {

laq_status laq_add_rmsnorm_f16(float* residual, const void* delta, const void* weight, void* y, int64_t M,
                               int64_t D, float eps, void* stream) {
  const char* fn = "laq_add_rmsnorm_f16";
  const laq::LaunchEvents ev = take_events();
  if (!residual || !weight || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if (M < 1 || M > 0x7FFFFFFFLL || D < 1 || D > (1LL << 20)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= M < 2^31 and 1 <= D <= 2^20");
  if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if (!aligned(residual, 4) || !aligned(weight, 2) || !aligned(y, 2) || (delta && !aligned(delta, 2)))
    return fail(LAQ_ERR_MISALIGNED, fn, "residual must be 4-byte, fp16 arrays 2-byte aligned");
  return hip_status(fn, laq::launch_add_rmsnorm(residual, static_cast<const uint16_t*>(delta),
                                                static_cast<const uint16_t*>(weight), static_cast<uint16_t*>(y), M, D,
                                                eps, static_cast<hipStream_t>(stream), ev));
}

laq_status laq_qk_norm_rope_f16(const void* qkv, const void* q_norm_weight, const void* k_norm_weight,
                                const float* cos_sin, int64_t pos, int64_t Hq, int64_t Hkv, int64_t head_dim,
                                float eps, void* q_out, void* k_cache, void* v_cache, int64_t S_max, void* stream) {
  const char* fn = "laq_qk_norm_rope_f16";
  const laq::LaunchEvents ev = take_events();
  if (!qkv || !q_norm_weight || !k_norm_weight || !cos_sin || !q_out || !k_cache || !v_cache)
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_heads(fn, Hq, Hkv, head_dim);
  if (st != LAQ_OK) return st;
  if (S_max < 1 || S_max > (1LL << 21) || pos < 0 || pos >= S_max)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= S_max <= 2^21 and 0 <= pos < S_max");
  if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if (!aligned(qkv, 2) || !aligned(q_norm_weight, 2) || !aligned(k_norm_weight, 2) || !aligned(cos_sin, 4) ||
      !aligned(q_out, 2) || !aligned(k_cache, 16) || !aligned(v_cache, 16))
    return fail(LAQ_ERR_MISALIGNED, fn, "caches must be 16-byte, cos_sin 4-byte, fp16 arrays 2-byte aligned");
  return hip_status(fn, laq::launch_qk_norm_rope(
                            static_cast<const uint16_t*>(qkv), static_cast<const uint16_t*>(q_norm_weight),
                            static_cast<const uint16_t*>(k_norm_weight), cos_sin, pos, Hq, Hkv, eps,
                            static_cast<uint16_t*>(q_out), static_cast<uint16_t*>(k_cache),
                            static_cast<uint16_t*>(v_cache), S_max, static_cast<hipStream_t>(stream), ev));
}

int64_t laq_decode_attention_workspace_bytes(int64_t Hq, int64_t L) {
  if (Hq < 1 || L < 1 || Hq > 4096 || L > (1LL << 21)) return 0;
  return Hq * laq::decode_attention_tiles(L) * (kHeadDimAbi + 2) * (int64_t)sizeof(float);
}

laq_status laq_decode_attention_f16(const void* q, const void* k_cache, const void* v_cache, int64_t Hq,
                                    int64_t Hkv, int64_t head_dim, int64_t L, int64_t S_max, void* out,
                                    void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "laq_decode_attention_f16";
  const laq::LaunchEvents ev = take_events();
  if (!q || !k_cache || !v_cache || !out || !workspace) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_heads(fn, Hq, Hkv, head_dim);
  if (st != LAQ_OK) return st;
  if (S_max < 1 || S_max > (1LL << 21) || L < 1 || L > S_max)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= L <= S_max <= 2^21");
  if (workspace_bytes < laq_decode_attention_workspace_bytes(Hq, L))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "workspace_bytes below laq_decode_attention_workspace_bytes(Hq, L)");
  if (!aligned(q, 2) || !aligned(out, 2) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(workspace, 16))
    return fail(LAQ_ERR_MISALIGNED, fn, "caches and workspace must be 16-byte, q and out 2-byte aligned");
  return hip_status(fn, laq::launch_decode_attention(
                            static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k_cache),
                            static_cast<const uint16_t*>(v_cache), Hq, Hkv, L, S_max, static_cast<uint16_t*>(out),
                            static_cast<float*>(workspace), static_cast<hipStream_t>(stream), ev));
}

int64_t laq_decode_attention_qkv_workspace_bytes(int64_t Hq, int64_t Hkv, int64_t L) {
  if (Hq < 1 || Hkv < 1 || L < 1 || Hq > 4096 || Hkv > Hq || L > (1LL << 21)) return 0;
  // The tile length grows with the context, so the tile count is largest at
  // the end of a tile-length regime: the maximum over every L' <= L.
  int64_t tiles = 0;
  for (int64_t lp : {L, std::min(L, 32767 / Hkv), std::min(L, 4095 / Hkv)})
    if (lp >= 1) tiles = std::max(tiles, laq::decode_attention_qkv_tiles(Hkv, lp));
  return Hq * tiles * (kHeadDimAbi + 2) * (int64_t)sizeof(float);
}

laq_status laq_decode_attention_qkv_f16(const void* qkv, const void* q_norm_weight, const void* k_norm_weight,
                                        const float* cos_sin, int64_t pos, int64_t Hq, int64_t Hkv,
                                        int64_t head_dim, float eps, void* k_cache, void* v_cache, int64_t S_max,
                                        void* out, void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "laq_decode_attention_qkv_f16";
  const laq::LaunchEvents ev = take_events();
  if (!qkv || !q_norm_weight || !k_norm_weight || !cos_sin || !k_cache || !v_cache || !out || !workspace)
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_heads(fn, Hq, Hkv, head_dim);
  if (st != LAQ_OK) return st;
  if (S_max < 1 || S_max > (1LL << 21) || pos < 0 || pos >= S_max)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= S_max <= 2^21 and 0 <= pos < S_max");
  if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if (workspace_bytes < laq_decode_attention_qkv_workspace_bytes(Hq, Hkv, pos + 1))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "workspace_bytes below laq_decode_attention_qkv_workspace_bytes(Hq, Hkv, pos + 1)");
  if (!aligned(qkv, 2) || !aligned(q_norm_weight, 2) || !aligned(k_norm_weight, 2) || !aligned(cos_sin, 4) ||
      !aligned(out, 2) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(workspace, 16))
    return fail(LAQ_ERR_MISALIGNED, fn,
                "caches and workspace must be 16-byte, cos_sin 4-byte, fp16 arrays 2-byte aligned");
  return hip_status(fn, laq::launch_decode_attention_qkv(
                            static_cast<const uint16_t*>(qkv), static_cast<const uint16_t*>(q_norm_weight),
                            static_cast<const uint16_t*>(k_norm_weight), cos_sin, pos, Hq, Hkv, eps,
                            static_cast<uint16_t*>(k_cache), static_cast<uint16_t*>(v_cache), S_max,
                            static_cast<uint16_t*>(out), static_cast<float*>(workspace),
                            static_cast<hipStream_t>(stream), ev));
}

}  // extern "C"

namespace {

template <int BITS>
laq_status linear_swiglu(const char* fn, const void* x, const uint32_t* qweight, const void* scales,
                         const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K, void* stream) {
  const laq::LaunchEvents ev = take_events();
  if (!x || !qweight || !scales || !zeros || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (M < 1 || M > 4) return fail(LAQ_ERR_BAD_M, fn, "M must be in 1..4");
  if (N % 2 != 0) return fail(LAQ_ERR_BAD_SHAPE, fn, "N (gate and up rows interleaved) must be even");
  if (!laq::swiglu_fits((int)M, K))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need K <= 16384 / M' (M' = M rounded up to 1, 2 or 4)");
  if (!aligned(x, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  return hip_status(fn, laq::launch_linear_swiglu<BITS>(static_cast<const uint16_t*>(x), qweight,
                                                        static_cast<const uint16_t*>(scales), zeros,
                                                        static_cast<uint16_t*>(y), (int)M, N, K,
                                                        static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status norm_linear(const char* fn, const float* residual, const void* delta, const void* norm_weight, float eps,
                       float* residual_out, const uint32_t* qweight, const void* scales, const uint8_t* zeros,
                       void* y, int64_t N, int64_t K, bool swiglu, void* stream) {
  const laq::LaunchEvents ev = take_events();
  if (!residual || !norm_weight || !qweight || !scales || !zeros || !y)
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (!laq::norm_linear_fits(K)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need K <= 8192");
  if (swiglu && N % 2 != 0) return fail(LAQ_ERR_BAD_SHAPE, fn, "N (gate and up rows interleaved) must be even");
  if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if (residual_out != nullptr && residual_out < residual + K && residual < residual_out + K)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "residual_out must not overlap residual");
  if (!aligned(residual, 16) || !aligned(delta, 16) || !aligned(norm_weight, 16) || !aligned(residual_out, 16) ||
      !aligned(qweight, 16))
    return fail(LAQ_ERR_MISALIGNED, fn, "residual, residual_out, delta, norm_weight and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  laq::NormPrologue np;
  np.res_in = residual;
  np.delta = static_cast<const uint16_t*>(delta);
  np.weight = static_cast<const uint16_t*>(norm_weight);
  np.res_out = residual_out;
  np.eps = eps;
  return hip_status(fn, laq::launch_linear_norm<BITS>(np, qweight, static_cast<const uint16_t*>(scales), zeros,
                                                      static_cast<uint16_t*>(y), N, K, swiglu,
                                                      static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status linear_residual(const char* fn, const void* x, const uint32_t* qweight, const void* scales,
                           const uint8_t* zeros, void* y, const float* residual_in, float* residual_out, int64_t N,
                           int64_t K, void* stream) {
  const laq::LaunchEvents ev = take_events();
  if (!x || !qweight || !scales || !zeros || !residual_in || !residual_out)  // y may be NULL
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (!laq::residual_linear_fits(N, K))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need K >= 2048 and rows whose activation tile fits in LDS (K <= ~28000)");
  if (residual_out != residual_in && residual_out < residual_in + N && residual_in < residual_out + N)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "residual_out must equal residual_in or not overlap it");
  if (!aligned(x, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  if (!aligned(residual_in, 4) || !aligned(residual_out, 4))
    return fail(LAQ_ERR_MISALIGNED, fn, "residual_in and residual_out must be 4-byte aligned");
  return hip_status(fn, laq::launch_linear_residual<BITS>(
                            static_cast<const uint16_t*>(x), qweight, static_cast<const uint16_t*>(scales), zeros,
                            static_cast<uint16_t*>(y), residual_in, residual_out, N, K,
                            static_cast<hipStream_t>(stream), ev));
}

template <int BITS>
laq_status norm_mlp(const char* fn, const float* residual, const void* delta, const void* norm_weight, float eps,
                    float* residual_out, const uint32_t* gu_qweight, const void* gu_scales, const uint8_t* gu_zeros,
                    const uint32_t* down_qweight, const void* down_scales, const uint8_t* down_zeros, void* y,
                    int64_t D, int64_t I, void* workspace, int64_t workspace_bytes, void* stream) {
  const laq::LaunchEvents ev = take_events();
  if (!residual || !norm_weight || !gu_qweight || !gu_scales || !gu_zeros || !down_qweight || !down_scales ||
      !down_zeros || !y || !workspace)
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  const laq::MlpPlan p = laq::mlp_plan(D, I, BITS);
  if (p.S == 0)
    return fail(LAQ_ERR_BAD_SHAPE, fn,
                "need D and I positive multiples of 128, D <= 2560, I <= 2^20, and the down group's codes in LDS");
  if (!(eps >= 0.0f) || !(eps < INFINITY)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if (residual_out != nullptr && residual_out < residual + D && residual < residual_out + D)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "residual_out must not overlap residual");
  if (workspace_bytes < (int64_t)laq::mlp_workspace_bytes(p, D))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "workspace smaller than laq_mlp_workspace_bytes(D, I)");
  if (!aligned(residual, 16) || !aligned(delta, 16) || !aligned(norm_weight, 16) || !aligned(residual_out, 16) ||
      !aligned(gu_qweight, 16) || !aligned(down_qweight, 16) || !aligned(workspace, 16))
    return fail(LAQ_ERR_MISALIGNED, fn,
                "residual, residual_out, delta, norm_weight, both qweights and workspace must be 16-byte aligned");
  if (!aligned(gu_scales, 2) || !aligned(down_scales, 2) || !aligned(y, 2))
    return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  laq::NormPrologue np;
  np.res_in = residual;
  np.delta = static_cast<const uint16_t*>(delta);
  np.weight = static_cast<const uint16_t*>(norm_weight);
  np.res_out = residual_out;
  np.eps = eps;
  return hip_status(fn, laq::launch_mlp<BITS>(np, gu_qweight, static_cast<const uint16_t*>(gu_scales), gu_zeros,
                                               down_qweight, static_cast<const uint16_t*>(down_scales), down_zeros,
                                               static_cast<uint16_t*>(y), D, I, workspace,
                                               static_cast<hipStream_t>(stream), ev));
}

}  // namespace

extern "C" {

laq_status laq_linear_residual_w3g128(const void* x, const uint32_t* qweight, const void* scales,
                                      const uint8_t* zeros, void* y, const float* residual_in, float* residual_out,
                                      int64_t N, int64_t K, void* stream) {
  return linear_residual<3>("laq_linear_residual_w3g128", x, qweight, scales, zeros, y, residual_in, residual_out, N,
                            K, stream);
}

laq_status laq_linear_residual_w4g128(const void* x, const uint32_t* qweight, const void* scales,
                                      const uint8_t* zeros, void* y, const float* residual_in, float* residual_out,
                                      int64_t N, int64_t K, void* stream) {
  return linear_residual<4>("laq_linear_residual_w4g128", x, qweight, scales, zeros, y, residual_in, residual_out, N,
                            K, stream);
}

int64_t laq_mlp_workspace_bytes(int64_t D, int64_t I) {
  const laq::MlpPlan p = laq::mlp_plan(D, I, 3);
  return (int64_t)laq::mlp_workspace_bytes(p, D);
}

laq_status laq_add_rmsnorm_mlp_w3g128(const float* residual, const void* delta, const void* norm_weight, float eps,
                                      float* residual_out, const uint32_t* gu_qweight, const void* gu_scales,
                                      const uint8_t* gu_zeros, const uint32_t* down_qweight, const void* down_scales,
                                      const uint8_t* down_zeros, void* y, int64_t D, int64_t I, void* workspace,
                                      int64_t workspace_bytes, void* stream) {
  return norm_mlp<3>("laq_add_rmsnorm_mlp_w3g128", residual, delta, norm_weight, eps, residual_out, gu_qweight,
                     gu_scales, gu_zeros, down_qweight, down_scales, down_zeros, y, D, I, workspace, workspace_bytes,
                     stream);
}

laq_status laq_linear_swiglu_w3g128(const void* x, const uint32_t* qweight, const void* scales,
                                    const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K, void* stream) {
  return linear_swiglu<3>("laq_linear_swiglu_w3g128", x, qweight, scales, zeros, y, M, N, K, stream);
}

laq_status laq_linear_swiglu_w4g128(const void* x, const uint32_t* qweight, const void* scales,
                                    const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K, void* stream) {
  return linear_swiglu<4>("laq_linear_swiglu_w4g128", x, qweight, scales, zeros, y, M, N, K, stream);
}

laq_status laq_add_rmsnorm_linear_w3g128(const float* residual, const void* delta, const void* norm_weight, float eps,
                                         float* residual_out, const uint32_t* qweight, const void* scales,
                                         const uint8_t* zeros, void* y, int64_t N, int64_t K, void* stream) {
  return norm_linear<3>("laq_add_rmsnorm_linear_w3g128", residual, delta, norm_weight, eps, residual_out, qweight,
                        scales, zeros, y, N, K, false, stream);
}

laq_status laq_add_rmsnorm_linear_w4g128(const float* residual, const void* delta, const void* norm_weight, float eps,
                                         float* residual_out, const uint32_t* qweight, const void* scales,
                                         const uint8_t* zeros, void* y, int64_t N, int64_t K, void* stream) {
  return norm_linear<4>("laq_add_rmsnorm_linear_w4g128", residual, delta, norm_weight, eps, residual_out, qweight,
                        scales, zeros, y, N, K, false, stream);
}

laq_status laq_add_rmsnorm_linear_swiglu_w3g128(const float* residual, const void* delta, const void* norm_weight,
                                                float eps, float* residual_out, const uint32_t* qweight,
                                                const void* scales, const uint8_t* zeros, void* y, int64_t N,
                                                int64_t K, void* stream) {
  return norm_linear<3>("laq_add_rmsnorm_linear_swiglu_w3g128", residual, delta, norm_weight, eps, residual_out,
                        qweight, scales, zeros, y, N, K, true, stream);
}

laq_status laq_add_rmsnorm_linear_swiglu_w4g128(const float* residual, const void* delta, const void* norm_weight,
                                                float eps, float* residual_out, const uint32_t* qweight,
                                                const void* scales, const uint8_t* zeros, void* y, int64_t N,
                                                int64_t K, void* stream) {
  return norm_linear<4>("laq_add_rmsnorm_linear_swiglu_w4g128", residual, delta, norm_weight, eps, residual_out,
                        qweight, scales, zeros, y, N, K, true, stream);
}

laq_status laq_silu_mul_f16(const void* gate_up, void* y, int64_t M, int64_t I, void* stream) {
  const char* fn = "laq_silu_mul_f16";
  const laq::LaunchEvents ev = take_events();
  if (!gate_up || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if (M < 1 || I < 1 || M > 65535 || I > (1LL << 30))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= M <= 65535 and 1 <= I <= 2^30");
  if (!aligned(gate_up, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "fp16 arrays must be 2-byte aligned");
  return hip_status(fn, laq::launch_silu_mul(static_cast<const uint16_t*>(gate_up), static_cast<uint16_t*>(y), M, I,
                                             static_cast<hipStream_t>(stream), ev));
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Batched serving: paged caches, sampling
// ---------------------------------------------------------------------------
namespace {

bool finite_eps(float eps) { return eps >= 0.0f && eps < INFINITY; }

// Checks a batch's sizes (no pointers: an empty batch may have none).
// bytes: of an element of the caches.
laq_status check_batch(const char* fn, const laq_paged_batch* b, int64_t Hq, int64_t Hkv, int64_t head_dim, int bytes = 2) {
  if (!b) return fail(LAQ_ERR_NULL_POINTER, fn, "null batch");
  if (head_dim != kHeadDimAbi) return fail(LAQ_ERR_BAD_SHAPE, fn, "head_dim must be 128");
  if (Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq > 4096)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "Hq must be a positive multiple of Hkv, at most 4096");
  // (the threads of a launch, 2^32 - 1 at most, are checked by the calls themselves)
  if (b->B < 0 || b->B > (1 << 20) || b->T < 0 || b->T >= (1LL << 26) || b->T * Hq > (1LL << 30))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 0 <= B <= 2^20, 0 <= T < 2^26 and T * Hq <= 2^30");
  if (b->page_size < 16 || b->page_size > (1 << 20) || (b->page_size & (b->page_size - 1)) != 0)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "page_size must be a power of two from 16 to 2^20");
  if (b->num_pages < 1 || b->num_pages > 0x7FFFFFFFLL) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= num_pages < 2^31");
  if (b->table_pages < 1 || b->table_pages > (1LL << 30) / b->page_size)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= table_pages and table_pages * page_size <= 2^30");
  if (b->table_stride < b->table_pages && b->B > 1)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "table_stride must be at least table_pages");
  if (b->table_stride < 0 || b->table_stride > (1LL << 40)) return fail(LAQ_ERR_BAD_SHAPE, fn, "table_stride must be in 0..2^40");
  if (b->slot_stride < kHeadDimAbi || b->slot_stride > (1 << 26) || b->head_stride < kHeadDimAbi ||
      b->head_stride > (1LL << 40) || b->page_stride < kHeadDimAbi || b->page_stride >= (1LL << 31))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "strides must be at least 128 (slots at most 2^26, pages below 2^31, heads at most 2^40)");
  if (b->slot_stride * bytes % 16 != 0 || b->head_stride * bytes % 16 != 0 || b->page_stride * bytes % 16 != 0)
    return fail(LAQ_ERR_MISALIGNED, fn, "strides must be multiples of 16 bytes");
  return LAQ_OK;
}

laq_status check_batch_pointers(const char* fn, const laq_paged_batch* b) {
  if (!b->k_pages || !b->v_pages || !b->page_table || !b->token_start || !b->seq_len)
    return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer in the batch");
  if (!aligned(b->k_pages, 16) || !aligned(b->v_pages, 16) || !aligned(b->page_table, 4) ||
      !aligned(b->token_start, 4) || !aligned(b->seq_len, 4))
    return fail(LAQ_ERR_MISALIGNED, fn, "pages must be 16-byte, page_table, token_start and seq_len 4-byte aligned");
  return LAQ_OK;
}

laq::PagedBatch internal_batch(const laq_paged_batch& b) {
  laq::PagedBatch p;
  p.k = static_cast<uint16_t*>(b.k_pages);
  p.v = static_cast<uint16_t*>(b.v_pages);
  p.page_table = b.page_table;
  p.token_start = b.token_start;
  p.seq_len = b.seq_len;
  p.page_bytes = (uint32_t)(b.page_stride * 2);
  p.head_stride = b.head_stride;
  p.table_stride = b.table_stride;
  p.slot_stride = (int)b.slot_stride;
  p.page_shift = __builtin_ctzll((unsigned long long)b.page_size);
  p.num_pages = (int)b.num_pages;
  p.table_pages = (int)b.table_pages;
  p.B = (int)b.B;
  p.T = (int)b.T;
  return p;
}

laq::PagedCodes internal_codes(const laq_paged_batch& b, uint8_t* k_scales, uint8_t* v_scales, int64_t Hkv) {
  laq::PagedCodes p;
  static_cast<laq::PagedBatch&>(p) = internal_batch(b);
  p.page_bytes = (uint32_t)b.page_stride;
  p.k_scales = k_scales;
  p.v_scales = v_scales;
  p.scale_page = Hkv * (b.page_size / 16);
  return p;
}

// What is checked of an append and of an attention, whatever the type of the
// caches, in this order; a batch without rows is `nothing`.
laq_status check_append(const char* fn, const laq_paged_batch* batch, const void* qkv, int64_t qkv_stride,
                        const void* q_norm_weight, const void* k_norm_weight, const float* cos_sin, int64_t rope_rows,
                        int64_t Hq, int64_t Hkv, int64_t head_dim, float eps, const void* q_out, int bytes,
                        bool* nothing) {
  laq_status st = check_batch(fn, batch, Hq, Hkv, head_dim, bytes);
  if (st != LAQ_OK) return st;
  if (rope_rows < 1 || rope_rows > (1LL << 31)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= rope_rows <= 2^31");
  if (qkv_stride < (Hq + 2 * Hkv) * head_dim || qkv_stride > (1LL << 40))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "qkv_stride must be at least (Hq + 2 Hkv) * 128");
  if (qkv_stride % 8 != 0) return fail(LAQ_ERR_MISALIGNED, fn, "qkv_stride must be a multiple of 8 elements");
  if (!finite_eps(eps)) return fail(LAQ_ERR_BAD_SHAPE, fn, "eps must be finite and >= 0");
  if ((*nothing = batch->B == 0 || batch->T == 0)) return LAQ_OK;
  if (!qkv || !cos_sin || !q_out) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if ((st = check_batch_pointers(fn, batch)) != LAQ_OK) return st;
  const int64_t threads = bytes == 2 ? laq::paged_append_threads(batch->T, Hq, Hkv)
                                     : laq::paged_append_codes_threads(batch->T, Hq, Hkv);
  if (threads > 0xFFFFFFFFLL) return fail(LAQ_ERR_BAD_SHAPE, fn, "the batch has too many rows for one launch");
  if (!aligned(qkv, 16) || !aligned(q_norm_weight, 16) || !aligned(k_norm_weight, 16) || !aligned(cos_sin, 4) ||
      !aligned(q_out, 16))
    return fail(LAQ_ERR_MISALIGNED, fn, "cos_sin must be 4-byte, fp16 arrays 16-byte aligned");
  return LAQ_OK;
}

laq_status check_attention(const char* fn, const laq_paged_batch* batch, const void* q, int64_t Hq, int64_t Hkv,
                           int64_t head_dim, int64_t window, const void* out, const void* workspace,
                           int64_t workspace_bytes, int bytes, bool* nothing) {
  laq_status st = check_batch(fn, batch, Hq, Hkv, head_dim, bytes);
  if (st != LAQ_OK) return st;
  if (window < 0 || window > (1LL << 30)) return fail(LAQ_ERR_BAD_SHAPE, fn, "window must be in 0..2^30");
  if ((*nothing = batch->B == 0 || batch->T == 0)) return LAQ_OK;
  if (!q || !out) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if ((st = check_batch_pointers(fn, batch)) != LAQ_OK) return st;
  const int64_t capacity = batch->table_pages * batch->page_size;
  const int64_t need = (bytes == 2 ? laq::paged_attention_workspace : laq::paged_attention_codes_workspace)(
      batch->B, batch->T, Hq, Hkv, capacity);
  if (need > 0 && !workspace) return fail(LAQ_ERR_NULL_POINTER, fn, "null workspace");
  if (workspace_bytes < need)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "workspace_bytes below the call's workspace_bytes query");
  const int64_t threads = (bytes == 2 ? laq::paged_attention_threads : laq::paged_attention_codes_threads)(
      batch->B, batch->T, Hq, Hkv, capacity);
  if (threads > 0xFFFFFFFFLL)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "the batch has too many rows for one launch");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16))
    return fail(LAQ_ERR_MISALIGNED, fn, "q, out and workspace must be 16-byte aligned");
  return LAQ_OK;
}

// Some element lies both in the rows [a + i as, + V) and in the rows [b + j bs, + V),
// i and j below `rows`; strides of V and more (or one row), so that rows of either
// follow one another.  Steps past the rows that end first, as far as they meet
// others: no more than 2 rows steps, and one where the arrays lie apart.
bool overlap(const uint16_t* a, int64_t as, const uint16_t* b, int64_t bs, int64_t rows, int64_t V) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  auto row = [](uintptr_t p, int64_t stride, int64_t i) { return p + 2 * (uintptr_t)(i * stride); };
  const uintptr_t width = 2 * (uintptr_t)V;
  if (row(x, as, rows - 1) + width <= y || row(y, bs, rows - 1) + width <= x) return false;
  for (int64_t i = 0, j = 0; i < rows && j < rows;) {
    const uintptr_t p = row(x, as, i), q = row(y, bs, j);
    if (p + width <= q) ++i;
    else if (q + width <= p) ++j;
    else return true;
  }
  return false;
}

}  // namespace

extern "C" {

laq_status laq_paged_append_f16(const laq_paged_batch* batch, const void* qkv, int64_t qkv_stride,
                                const void* q_norm_weight, const void* k_norm_weight, const float* cos_sin,
                                int64_t rope_rows, int64_t Hq, int64_t Hkv, int64_t head_dim, float eps, void* q_out,
                                void* stream) {
  const char* fn = "laq_paged_append_f16";
  const laq::LaunchEvents ev = take_events();
  bool nothing = false;
  const laq_status st = check_append(fn, batch, qkv, qkv_stride, q_norm_weight, k_norm_weight, cos_sin, rope_rows, Hq, Hkv,
                                     head_dim, eps, q_out, 2, &nothing);
  if (st != LAQ_OK) return st;
  if (nothing) return ok();
  return hip_status(fn, laq::launch_paged_append(
                            internal_batch(*batch), static_cast<const uint16_t*>(qkv), qkv_stride,
                            static_cast<const uint16_t*>(q_norm_weight), static_cast<const uint16_t*>(k_norm_weight),
                            cos_sin, rope_rows, Hq, Hkv, eps, static_cast<uint16_t*>(q_out),
                            static_cast<hipStream_t>(stream), ev));
}

laq_status laq_paged_append_e4m3(const laq_paged_batch* batch, uint8_t* k_scales, uint8_t* v_scales, const void* qkv,
                                 int64_t qkv_stride, const void* q_norm_weight, const void* k_norm_weight,
                                 const float* cos_sin, int64_t rope_rows, int64_t Hq, int64_t Hkv, int64_t head_dim,
                                 float eps, void* q_out, void* stream) {
  const char* fn = "laq_paged_append_e4m3";
  const laq::LaunchEvents ev = take_events();
  bool nothing = false;
  const laq_status st = check_append(fn, batch, qkv, qkv_stride, q_norm_weight, k_norm_weight, cos_sin, rope_rows, Hq, Hkv,
                                     head_dim, eps, q_out, 1, &nothing);
  if (st != LAQ_OK) return st;
  if (nothing) return ok();
  if (!k_scales || !v_scales) return fail(LAQ_ERR_NULL_POINTER, fn, "null scales");
  return hip_status(fn, laq::launch_paged_append_codes(
                            internal_codes(*batch, k_scales, v_scales, Hkv), static_cast<const uint16_t*>(qkv),
                            qkv_stride, static_cast<const uint16_t*>(q_norm_weight),
                            static_cast<const uint16_t*>(k_norm_weight), cos_sin, rope_rows, Hq, Hkv, eps,
                            static_cast<uint16_t*>(q_out), static_cast<hipStream_t>(stream), ev));
}

static bool attention_sizes(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  return !(B < 1 || B > (1 << 20) || T < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || Hq > 4096 || T > (1LL << 30) ||
           T * Hq > (1LL << 30) || capacity < 1 || capacity > (1LL << 30));
}

int64_t laq_paged_attention_workspace_bytes(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  return attention_sizes(B, T, Hq, Hkv, capacity) ? laq::paged_attention_workspace(B, T, Hq, Hkv, capacity) : 0;
}

int64_t laq_paged_attention_e4m3_workspace_bytes(int64_t B, int64_t T, int64_t Hq, int64_t Hkv, int64_t capacity) {
  return attention_sizes(B, T, Hq, Hkv, capacity) ? laq::paged_attention_codes_workspace(B, T, Hq, Hkv, capacity) : 0;
}

laq_status laq_paged_attention_f16(const laq_paged_batch* batch, const void* q, int64_t Hq, int64_t Hkv,
                                   int64_t head_dim, int64_t window, void* out, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  const char* fn = "laq_paged_attention_f16";
  const laq::LaunchEvents ev = take_events();
  bool nothing = false;
  const laq_status st = check_attention(fn, batch, q, Hq, Hkv, head_dim, window, out, workspace, workspace_bytes, 2, &nothing);
  if (st != LAQ_OK) return st;
  if (nothing) return ok();
  return hip_status(fn, laq::launch_paged_attention(internal_batch(*batch), static_cast<const uint16_t*>(q), Hq, Hkv,
                                                    window, static_cast<uint16_t*>(out),
                                                    static_cast<float*>(workspace), static_cast<hipStream_t>(stream),
                                                    ev));
}

laq_status laq_paged_attention_e4m3(const laq_paged_batch* batch, const uint8_t* k_scales, const uint8_t* v_scales,
                                    const void* q, int64_t Hq, int64_t Hkv, int64_t head_dim, int64_t window, void* out,
                                    void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "laq_paged_attention_e4m3";
  const laq::LaunchEvents ev = take_events();
  bool nothing = false;
  const laq_status st = check_attention(fn, batch, q, Hq, Hkv, head_dim, window, out, workspace, workspace_bytes, 1, &nothing);
  if (st != LAQ_OK) return st;
  if (nothing) return ok();
  if (!k_scales || !v_scales) return fail(LAQ_ERR_NULL_POINTER, fn, "null scales");
  return hip_status(fn, laq::launch_paged_attention_codes(
                            internal_codes(*batch, const_cast<uint8_t*>(k_scales), const_cast<uint8_t*>(v_scales), Hkv),
                            static_cast<const uint16_t*>(q), Hq, Hkv, window, static_cast<uint16_t*>(out),
                            static_cast<float*>(workspace), static_cast<hipStream_t>(stream), ev));
}

laq_status laq_adjust_logits_f16(const laq_logits_adjust* adjust, const void* logits, int64_t logits_stride, int64_t rows,
                                 int64_t V, void* out, int64_t out_stride, void* stream) {
  const char* fn = "laq_adjust_logits_f16";
  const laq::LaunchEvents ev = take_events();
  if (!adjust) return fail(LAQ_ERR_NULL_POINTER, fn, "null adjust");
  const laq_logits_adjust& a = *adjust;
  if (rows < 0 || rows >= (1LL << 22)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 0 <= rows < 2^22");
  if (V < 1 || V > (1 << 24)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= V <= 2^24");
  for (int64_t s : {logits_stride, out_stride}) {
    if (s < V && rows > 1) return fail(LAQ_ERR_BAD_SHAPE, fn, "strides of logits and out must be at least V");
    if (s < 0 || s > (1LL << 32)) return fail(LAQ_ERR_BAD_SHAPE, fn, "strides must be in 0..2^32");
  }
  if (a.history) {
    if (a.history_room < 0 || a.history_room >= (1 << 20)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 0 <= history_room < 2^20");
    if (a.history_stride < 0 || a.history_stride > (1LL << 32)) return fail(LAQ_ERR_BAD_SHAPE, fn, "strides must be in 0..2^32");
    if (!a.history_len) return fail(LAQ_ERR_NULL_POINTER, fn, "null history_len");
  }
  if (a.bias_token) {
    if (a.biases < 0 || a.biases > LAQ_MAX_BIASES) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 0 <= biases <= 2047");
    if (a.bias_stride < 0 || a.bias_stride > (1LL << 32)) return fail(LAQ_ERR_BAD_SHAPE, fn, "strides must be in 0..2^32");
    if (!a.bias_value) return fail(LAQ_ERR_NULL_POINTER, fn, "null bias_value");
  }
  if (a.mask && (a.mask_stride < 0 || a.mask_stride > (1LL << 32)))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "strides must be in 0..2^32");
  if (rows == 0) return ok();
  if (!logits || !out) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if (!aligned(logits, 2) || !aligned(out, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "logits and out must be 2-byte aligned");
  for (const void* p : {(const void*)a.history, (const void*)a.history_len, (const void*)a.prompt_len,
                        (const void*)a.repetition, (const void*)a.frequency, (const void*)a.presence,
                        (const void*)a.bias_token, (const void*)a.bias_value, (const void*)a.mask})
    if (!aligned(p, 4)) return fail(LAQ_ERR_MISALIGNED, fn, "the arrays of adjust must be 4-byte aligned");
  const bool same = out == logits && (rows == 1 || out_stride == logits_stride);
  if (!same && overlap(static_cast<const uint16_t*>(logits), logits_stride, static_cast<const uint16_t*>(out), out_stride, rows, V))
    return fail(LAQ_ERR_BAD_SHAPE, fn, "out must be logits itself or share no element with it");
  laq::Adjust d{};
  d.logits = static_cast<const uint16_t*>(logits);
  d.out = static_cast<uint16_t*>(out);
  d.stride = logits_stride;
  d.out_stride = out_stride;
  if (a.history && a.history_room > 0 && (a.repetition || a.frequency || a.presence)) {
    d.history = a.history;
    d.history_len = a.history_len;
    d.prompt_len = a.prompt_len;
    d.history_stride = a.history_stride;
    d.room = (int)a.history_room;
    d.repetition = a.repetition;
    d.frequency = a.frequency;
    d.presence = a.presence;
  }
  if (a.bias_token && a.biases > 0) {
    d.bias_token = a.bias_token;
    d.bias_value = a.bias_value;
    d.bias_stride = a.bias_stride;
    d.biases = (int)a.biases;
  }
  d.mask = a.mask;
  d.mask_stride = a.mask_stride;
  d.V = (int)V;
  d.in_place = same;
  if (laq::adjust_logits_threads(d, rows) > 0xFFFFFFFFLL)
    return fail(LAQ_ERR_BAD_SHAPE, fn, "too many logits for one launch");
  return hip_status(fn, laq::launch_adjust_logits(d, rows, static_cast<hipStream_t>(stream), ev));
}

laq_status laq_sample_f16(const void* logits, int64_t logits_stride, int64_t rows, int64_t V, const float* u,
                          const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                          int32_t* token, float* prob, void* stream) {
  const char* fn = "laq_sample_f16";
  const laq::LaunchEvents ev = take_events();
  // (1024 threads a row: 2^22 rows would be 2^32 threads, more than one launch may have)
  if (rows < 0 || rows >= (1LL << 22)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 0 <= rows < 2^22");
  if (V < 1 || V > (1 << 24)) return fail(LAQ_ERR_BAD_SHAPE, fn, "need 1 <= V <= 2^24");
  if (logits_stride < V && rows > 1) return fail(LAQ_ERR_BAD_SHAPE, fn, "logits_stride must be at least V");
  if (logits_stride < 0 || logits_stride > (1LL << 32)) return fail(LAQ_ERR_BAD_SHAPE, fn, "logits_stride must be in 0..2^32");
  if (rows == 0) return ok();
  if (!logits || !u || !token) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  if (!aligned(logits, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "logits must be 2-byte aligned");
  if (!aligned(u, 4) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) ||
      !aligned(token, 4) || !aligned(prob, 4))
    return fail(LAQ_ERR_MISALIGNED, fn, "per-row arrays must be 4-byte aligned");
  return hip_status(fn, laq::launch_sample(static_cast<const uint16_t*>(logits), logits_stride, rows, V, u, temperature,
                                           top_k, top_p, min_p, token, prob, static_cast<hipStream_t>(stream), ev));
}

}  // extern "C"

// ---------------------------------------------------------------------------
// The linear without a caller workspace and without allocation: split-K
// partial sums in a scratch array the library holds on each GPU.
// ---------------------------------------------------------------------------
namespace {

// Each GPU the library runs on holds its own copy of this array until the
// process ends.  In host code the name is only a symbol handle, never an
// address: the device address comes from hipGetSymbolAddress, per device.
static __device__ __align__(256) float scratch[LAQ_NOALLOC_SCRATCH_BYTES / sizeof(float)];

constexpr int kScratchDevices = 64;
std::atomic<float*> g_scratch_ptr[kScratchDevices];
std::mutex g_scratch_mutex;

// Device address of `scratch` on the device that runs `stream` (looked up
// once per device, with that device current).
laq_status scratch_on_stream_device(const char* fn, hipStream_t stream, float** out) {
  int cur = 0;
  hipError_t e = hipGetDevice(&cur);
  if (e != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e));
  int dev = cur;
  if (stream) {
    hipDevice_t d = 0;
    e = hipStreamGetDevice(stream, &d);
    if (e != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e));
    dev = (int)d;
  }
  if (dev < 0 || dev >= kScratchDevices) return fail(LAQ_ERR_HIP, fn, "device index beyond the scratch table");
  float* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (!p) {
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    p = g_scratch_ptr[dev].load(std::memory_order_relaxed);
    if (!p) {
      if (dev != cur && (e = hipSetDevice(dev)) != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e));
      void* addr = nullptr;
      e = hipGetSymbolAddress(&addr, HIP_SYMBOL(scratch));
      const hipError_t e2 = dev != cur ? hipSetDevice(cur) : hipSuccess;
      if (e != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e));
      if (e2 != hipSuccess) return fail(LAQ_ERR_HIP, fn, hipGetErrorString(e2));
      if (!addr) return fail(LAQ_ERR_HIP, fn, "no device address for the scratch array");
      p = static_cast<float*>(addr);
      g_scratch_ptr[dev].store(p, std::memory_order_release);
    }
  }
  *out = p;
  return LAQ_OK;
}

}  // namespace

extern "C" laq_status laq_linear_noalloc_w3g128(const void* x, const uint32_t* qweight, const void* scales,
                                                const uint8_t* zeros, void* y, int64_t M, int64_t N, int64_t K,
                                                void* stream) {
  const char* fn = "laq_linear_noalloc_w3g128";
  const laq::LaunchEvents ev = take_events();  // consumed whether or not the call launches
  if (!x || !qweight || !scales || !zeros || !y) return fail(LAQ_ERR_NULL_POINTER, fn, "null pointer argument");
  laq_status st = check_shape(fn, N, K);
  if (st != LAQ_OK) return st;
  if (M < 1 || M > LAQ_MAX_M) return fail(LAQ_ERR_BAD_M, fn, "M must be in 1..16");
  if (!aligned(x, 16) || !aligned(qweight, 16)) return fail(LAQ_ERR_MISALIGNED, fn, "x and qweight must be 16-byte aligned");
  if (!aligned(scales, 2) || !aligned(y, 2)) return fail(LAQ_ERR_MISALIGNED, fn, "scales and y must be 2-byte aligned");
  const size_t need = laq::split_workspace_bytes(laq::mfma_split_plan((int)M, N, (int)(K / 128)), (int)M, N);
  if (need > (size_t)LAQ_NOALLOC_SCRATCH_BYTES)
    return fail(LAQ_ERR_BAD_SHAPE, fn,
                "the split-K partial sums of this shape exceed the scratch array (LAQ_NOALLOC_SCRATCH_BYTES)");
  float* ws = nullptr;
  if (need > 0) {
    st = scratch_on_stream_device(fn, static_cast<hipStream_t>(stream), &ws);
    if (st != LAQ_OK) return st;
  }
  return hip_status(fn, laq::launch_linear<3>(static_cast<const uint16_t*>(x), qweight,
                                              static_cast<const uint16_t*>(scales), zeros,
                                              static_cast<uint16_t*>(y), (int)M, N, K,
                                              static_cast<hipStream_t>(stream), ev, ws, need));
}

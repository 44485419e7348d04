// Driver for a sanitizer build (AddressSanitizer + UndefinedBehaviorSanitizer
// on the host code) of the entry points that abi_sanitize.cpp does not call: the
// batched serving ones (paged append, paged attention and its workspace size,
// sampling; their forms over caches of 8 bits; the logits' adjustment), the
// linears that update the residual stream, and the MLP block.
// Arguments that their host-side validation must reject, sizes at and past every
// limit and extreme integers among them, checking the returned status and the
// last-error text; and the workspace sizes over grids of sizes, valid and not.
// Nothing here passes validation, so no HIP call is reached and no GPU is
// needed.  Any sanitizer report aborts the run; a wrong status returns 1.
// Prints "ok N" (N checks) on success.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <limits>
#include <vector>

#include "laq.h"

namespace {

int g_checks = 0, g_bad = 0;

void expect(int line, laq_status got, laq_status want, const char* fn) {
  ++g_checks;
  const char* msg = laq_last_error();
  if (got != want || (fn && !std::strstr(msg, fn))) {
    std::printf("line %d: status %d (want %d), last error \"%s\"\n", line, got, want, msg);
    ++g_bad;
  }
}
#define EXPECT(call, want, fn) expect(__LINE__, (call), (want), (fn))

void* const P = reinterpret_cast<void*>(0x100000);  // aligned, never dereferenced
float* const F = static_cast<float*>(P);
int32_t* const I = static_cast<int32_t*>(P);
uint32_t* const Q = static_cast<uint32_t*>(P);
uint8_t* const Z = static_cast<uint8_t*>(P);
const int64_t kMax = std::numeric_limits<int64_t>::max();
const int64_t kMin = std::numeric_limits<int64_t>::min();

template <typename T>
T* off(T* p, int bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<char*>(p) + bytes);
}

laq_paged_batch batch() {
  laq_paged_batch b;
  b.k_pages = b.v_pages = P;
  b.page_table = b.token_start = b.seq_len = I;
  b.num_pages = 10;
  b.page_size = 16;
  b.page_stride = 8 * 16 * 128;
  b.head_stride = 16 * 128;
  b.slot_stride = 128;
  b.table_pages = b.table_stride = 1000;
  b.B = 2;
  b.T = 3;
  return b;
}

laq_status append(const laq_paged_batch* b, int64_t Hq = 32, int64_t Hkv = 8, int64_t stride = (int64_t)1 << 40,
                  int64_t rope = 100, float eps = 1e-6f, int64_t d = 128) {
  return laq_paged_append_f16(b, P, stride, P, P, F, rope, Hq, Hkv, d, eps, P, nullptr);
}
laq_status attention(const laq_paged_batch* b, int64_t Hq = 32, int64_t Hkv = 8, int64_t window = 0,
                     int64_t bytes = 0, int64_t d = 128) {
  return laq_paged_attention_f16(b, P, Hq, Hkv, d, window, P, P, bytes, nullptr);
}

// What both calls check of a batch: a member set to each of some values.
void members(int64_t laq_paged_batch::*m, std::initializer_list<int64_t> values, laq_status want) {
  for (int64_t v : values) {
    laq_paged_batch b = batch();
    b.*m = v;
    EXPECT(append(&b), want, "laq_paged_append_f16");
    EXPECT(attention(&b), want, "laq_paged_attention_f16");
  }
}

}  // namespace

int main() {
  const laq_paged_batch good = batch();
  EXPECT(append(nullptr), LAQ_ERR_NULL_POINTER, "laq_paged_append_f16");
  EXPECT(attention(nullptr), LAQ_ERR_NULL_POINTER, "laq_paged_attention_f16");
  members(&laq_paged_batch::num_pages, {kMin, -1, 0, (int64_t)1 << 31, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::page_size, {kMin, -16, 0, 1, 8, 17, 24, 1 << 21, (int64_t)1 << 62, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::page_stride, {kMin, -128, 0, 64, (int64_t)1 << 31, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::head_stride, {kMin, -8, 0, 120, ((int64_t)1 << 40) + 8, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::slot_stride, {kMin, -128, 0, 64, (1 << 26) + 8, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::table_pages, {kMin, -1, 0, ((int64_t)1 << 26) + 1, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::table_stride, {kMin, -1, 999, ((int64_t)1 << 40) + 1, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::B, {kMin, -1, (1 << 20) + 1, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::T, {kMin, -1, (int64_t)1 << 26, ((int64_t)1 << 30) / 32 + 1, kMax}, LAQ_ERR_BAD_SHAPE);
  members(&laq_paged_batch::page_stride, {8 * 16 * 128 + 4}, LAQ_ERR_MISALIGNED);
  members(&laq_paged_batch::head_stride, {16 * 128 + 1}, LAQ_ERR_MISALIGNED);
  members(&laq_paged_batch::slot_stride, {130}, LAQ_ERR_MISALIGNED);
  for (int which = 0; which < 5; ++which) {
    for (int bytes : {-1, 1, 2}) {  // -1: null
      laq_paged_batch b = batch();
      if (which < 2)
        (which ? b.v_pages : b.k_pages) = bytes < 0 ? nullptr : off(P, bytes);
      else
        (which == 2 ? b.page_table : which == 3 ? b.token_start : b.seq_len) = bytes < 0 ? nullptr : off(I, bytes);
      const laq_status want = bytes < 0 ? LAQ_ERR_NULL_POINTER : LAQ_ERR_MISALIGNED;
      EXPECT(append(&b), want, "laq_paged_append_f16");
      // (alignment counts for a call that is right otherwise)
      EXPECT(attention(&b, 32, 8, 0, (int64_t)1 << 40), want, "laq_paged_attention_f16");
    }
  }
  const int64_t heads[][2] = {{0, 1}, {8, 0}, {8, 3}, {-8, -8}, {4104, 8}, {kMax, 1}, {8, kMin}, {kMin, 1}, {kMin, -1}};
  for (const auto& h : heads) {
    EXPECT(append(&good, h[0], h[1]), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
    EXPECT(attention(&good, h[0], h[1]), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_f16");
  }
  for (int64_t d : {kMin, (int64_t)0, (int64_t)64, (int64_t)129, kMax}) {
    EXPECT(append(&good, 32, 8, (int64_t)1 << 40, 100, 1e-6f, d), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
    EXPECT(attention(&good, 32, 8, 0, 0, d), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_f16");
  }
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)48 * 128 - 8, ((int64_t)1 << 40) + 8, kMax})
    EXPECT(append(&good, 32, 8, v), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
  EXPECT(append(&good, 32, 8, 48 * 128 + 4), LAQ_ERR_MISALIGNED, "laq_paged_append_f16");
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, ((int64_t)1 << 31) + 1, kMax})
    EXPECT(append(&good, 32, 8, (int64_t)1 << 40, v), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
  for (float e : {-1e-6f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity()})
    EXPECT(append(&good, 32, 8, (int64_t)1 << 40, 100, e), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
  for (int64_t v : {kMin, (int64_t)-1, ((int64_t)1 << 30) + 1, kMax})
    EXPECT(attention(&good, 32, 8, v), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_f16");
  EXPECT(laq_paged_append_f16(&good, nullptr, (int64_t)1 << 40, P, P, F, 100, 32, 8, 128, 1e-6f, P, nullptr),
         LAQ_ERR_NULL_POINTER, "laq_paged_append_f16");
  EXPECT(laq_paged_append_f16(&good, P, (int64_t)1 << 40, off(P, 2), P, F, 100, 32, 8, 128, 1e-6f, P, nullptr),
         LAQ_ERR_MISALIGNED, "laq_paged_append_f16");
  EXPECT(laq_paged_attention_f16(&good, P, 32, 8, 128, 0, nullptr, P, (int64_t)1 << 40, nullptr), LAQ_ERR_NULL_POINTER,
         "laq_paged_attention_f16");
  EXPECT(laq_paged_attention_f16(&good, P, 32, 8, 128, 0, P, nullptr, (int64_t)1 << 40, nullptr), LAQ_ERR_NULL_POINTER,
         "laq_paged_attention_f16");
  EXPECT(laq_paged_attention_f16(&good, P, 32, 8, 128, 0, P, off(P, 8), (int64_t)1 << 40, nullptr), LAQ_ERR_MISALIGNED,
         "laq_paged_attention_f16");

  // sizes at their limits: a workspace one byte short, launches of 2^32 threads
  const std::vector<int64_t> sizes = {kMin, -1, 0, 1, 2, 3, 63, 64, 65, 4096, 1 << 20, (1 << 20) + 1, ((int64_t)1 << 26) - 1,
                                      (int64_t)1 << 26, (int64_t)1 << 30, ((int64_t)1 << 30) + 1, kMax};
  for (int64_t B : sizes)
    for (int64_t T : sizes)
      for (int64_t Hkv : {kMin, (int64_t)0, (int64_t)1, (int64_t)8, (int64_t)511, (int64_t)512, (int64_t)4096, kMax})
        for (int64_t R : {1, 2, 16, 512, 4096})
          for (int64_t capacity : {kMin, (int64_t)0, (int64_t)16, (int64_t)128, (int64_t)129, (int64_t)4096, (int64_t)1 << 30, kMax}) {
            const int64_t Hq = Hkv > 0 && Hkv <= 4096 ? Hkv * R : Hkv;
            const int64_t n = laq_paged_attention_workspace_bytes(B, T, Hq, Hkv, capacity);
            const int64_t n8 = laq_paged_attention_e4m3_workspace_bytes(B, T, Hq, Hkv, capacity);
            g_checks += 2;
            if (n8 < 0 || n8 > n) {
              std::printf("laq_paged_attention_e4m3_workspace_bytes(%lld, %lld, %lld, %lld, %lld) = %lld\n", (long long)B,
                          (long long)T, (long long)Hq, (long long)Hkv, (long long)capacity, (long long)n8);
              ++g_bad;
            }
            if (n < 0 || n > 140 * 1000 * 1000) {
              std::printf("laq_paged_attention_workspace_bytes(%lld, %lld, %lld, %lld, %lld) = %lld\n", (long long)B,
                          (long long)T, (long long)Hq, (long long)Hkv, (long long)capacity, (long long)n);
              ++g_bad;
            }
            if (n > 0) {
              laq_paged_batch b = batch();
              b.B = B;
              b.T = T;
              b.table_pages = b.table_stride = (capacity + 15) / 16;
              const int64_t need = laq_paged_attention_workspace_bytes(B, T, Hq, Hkv, b.table_pages * 16);
              EXPECT(attention(&b, Hq, Hkv, 0, need - 1), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_f16");
            }
          }
  for (int64_t below : {1, 2, 3}) {
    laq_paged_batch b = batch();
    b.T = ((int64_t)1 << 26) - below;
    EXPECT(append(&b, 1, 1), LAQ_ERR_BAD_SHAPE, "laq_paged_append_f16");
  }

  typedef laq_status (*residual_fn)(const void*, const uint32_t*, const void*, const uint8_t*, void*, const float*,
                                    float*, int64_t, int64_t, void*);
  const residual_fn residual[] = {laq_linear_residual_w3g128, laq_linear_residual_w4g128};
  const char* const residual_name[] = {"laq_linear_residual_w3g128", "laq_linear_residual_w4g128"};
  for (int i = 0; i < 2; ++i) {
    const residual_fn f = residual[i];
    const char* fn = residual_name[i];
    EXPECT(f(nullptr, Q, P, Z, P, F, F, 64, 2560, nullptr), LAQ_ERR_NULL_POINTER, fn);
    EXPECT(f(P, nullptr, P, Z, P, F, F, 64, 2560, nullptr), LAQ_ERR_NULL_POINTER, fn);
    EXPECT(f(P, Q, P, Z, nullptr, nullptr, F, 64, 2560, nullptr), LAQ_ERR_NULL_POINTER, fn);
    EXPECT(f(P, Q, P, Z, nullptr, F, nullptr, 64, 2560, nullptr), LAQ_ERR_NULL_POINTER, fn);
    for (int64_t n : {kMin, (int64_t)-1, (int64_t)0, (int64_t)1 << 31, kMax})
      EXPECT(f(P, Q, P, Z, P, F, F, n, 2560, nullptr), LAQ_ERR_BAD_SHAPE, fn);
    for (int64_t k : {kMin, (int64_t)-128, (int64_t)0, (int64_t)200, (int64_t)1920, (int64_t)1 << 20, (int64_t)(kMax - 127)})
      EXPECT(f(P, Q, P, Z, P, F, F, 64, k, nullptr), LAQ_ERR_BAD_SHAPE, fn);
    EXPECT(f(P, Q, P, Z, P, F, F + 1, 64, 2560, nullptr), LAQ_ERR_BAD_SHAPE, fn);
    EXPECT(f(P, Q, P, Z, P, F + 63, F, 64, 2560, nullptr), LAQ_ERR_BAD_SHAPE, fn);
    EXPECT(f(off(P, 8), Q, P, Z, P, F, F, 64, 2560, nullptr), LAQ_ERR_MISALIGNED, fn);
    EXPECT(f(P, Q, off(P, 1), Z, P, F, F, 64, 2560, nullptr), LAQ_ERR_MISALIGNED, fn);
    EXPECT(f(P, Q, P, Z, P, off(F, 2), off(F, 2), 64, 2560, nullptr), LAQ_ERR_MISALIGNED, fn);
  }

  const char* fn = "laq_add_rmsnorm_mlp_w3g128";
  auto mlp = [](const float* r, float* r_out, int64_t D, int64_t width, void* ws, int64_t bytes, float eps = 1e-6f,
                const void* y_scales = P) {
    return laq_add_rmsnorm_mlp_w3g128(r, P, P, eps, r_out, Q, y_scales, Z, Q, P, Z, P, D, width, ws, bytes, nullptr);
  };
  const int64_t need = laq_mlp_workspace_bytes(2560, 9728);
  const int64_t plenty = (int64_t)1 << 40;
  EXPECT(mlp(nullptr, nullptr, 2560, 9728, P, plenty), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(mlp(F, nullptr, 2560, 9728, nullptr, plenty), LAQ_ERR_NULL_POINTER, fn);
  for (int64_t d : {kMin, (int64_t)-128, (int64_t)0, (int64_t)64, (int64_t)2688, (int64_t)(kMax - 127), kMax})
    EXPECT(mlp(F, nullptr, d, 9728, P, plenty), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t i : {kMin, (int64_t)-128, (int64_t)0, (int64_t)200, ((int64_t)1 << 20) + 128, (int64_t)(kMax - 127), kMax})
    EXPECT(mlp(F, nullptr, 2560, i, P, plenty), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t b : {need - 1, (int64_t)0, (int64_t)-1, kMin}) EXPECT(mlp(F, nullptr, 2560, 9728, P, b), LAQ_ERR_BAD_SHAPE, fn);
  for (float e : {-1e-6f, std::numeric_limits<float>::quiet_NaN(), std::numeric_limits<float>::infinity()})
    EXPECT(mlp(F, nullptr, 2560, 9728, P, plenty, e), LAQ_ERR_BAD_SHAPE, fn);
  EXPECT(mlp(F, F, 2560, 9728, P, plenty), LAQ_ERR_BAD_SHAPE, fn);
  EXPECT(mlp(off(F, 8), nullptr, 2560, 9728, P, plenty), LAQ_ERR_MISALIGNED, fn);
  EXPECT(mlp(F, nullptr, 2560, 9728, off(P, 8), plenty), LAQ_ERR_MISALIGNED, fn);
  EXPECT(mlp(F, nullptr, 2560, 9728, P, plenty, 1e-6f, off(P, 1)), LAQ_ERR_MISALIGNED, fn);
  for (int64_t d : {kMin, (int64_t)-1, (int64_t)0, (int64_t)100, (int64_t)128, (int64_t)2560, (int64_t)2688, kMax})
    for (int64_t i : {kMin, (int64_t)-1, (int64_t)0, (int64_t)100, (int64_t)128, (int64_t)9728, (int64_t)1 << 20, kMax}) {
      const int64_t b = laq_mlp_workspace_bytes(d, i);
      ++g_checks;
      const bool valid = d >= 128 && d <= 2560 && d % 128 == 0 && i >= 128 && i <= (1 << 20) && i % 128 == 0;
      if (b < 0 || (!valid && b != 0)) {
        std::printf("laq_mlp_workspace_bytes(%lld, %lld) = %lld\n", (long long)d, (long long)i, (long long)b);
        ++g_bad;
      }
    }

  fn = "laq_sample_f16";
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)1 << 22, kMax})
    EXPECT(laq_sample_f16(P, 1000, v, 1000, F, F, I, F, F, I, F, nullptr), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)(1 << 24) + 1, kMax})
    EXPECT(laq_sample_f16(P, 1000, 4, v, F, F, I, F, F, I, F, nullptr), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)999, ((int64_t)1 << 32) + 1, kMax})
    EXPECT(laq_sample_f16(P, v, 4, 1000, F, F, I, F, F, I, F, nullptr), LAQ_ERR_BAD_SHAPE, fn);
  EXPECT(laq_sample_f16(nullptr, 1000, 4, 1000, F, F, I, F, F, I, F, nullptr), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(laq_sample_f16(P, 1000, 4, 1000, nullptr, F, I, F, F, I, F, nullptr), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(laq_sample_f16(P, 1000, 4, 1000, F, F, I, F, F, nullptr, F, nullptr), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(laq_sample_f16(off(P, 1), 1000, 4, 1000, F, F, I, F, F, I, F, nullptr), LAQ_ERR_MISALIGNED, fn);
  EXPECT(laq_sample_f16(P, 1000, 4, 1000, off(F, 2), F, I, F, F, I, F, nullptr), LAQ_ERR_MISALIGNED, fn);
  EXPECT(laq_sample_f16(P, 1000, 4, 1000, F, F, off(I, 1), F, F, I, F, nullptr), LAQ_ERR_MISALIGNED, fn);
  EXPECT(laq_sample_f16(P, 1000, 4, 1000, F, F, I, F, F, I, off(F, 3), nullptr), LAQ_ERR_MISALIGNED, fn);

  // caches of 8 bits: what the fp16 calls check, strides of whole 16 bytes, and the scales
  uint8_t* const S = static_cast<uint8_t*>(P);
  auto append8 = [&](const laq_paged_batch* b, uint8_t* ks, uint8_t* vs, int64_t Hq = 32, int64_t Hkv = 8,
                     int64_t stride = (int64_t)1 << 40) {
    return laq_paged_append_e4m3(b, ks, vs, P, stride, P, P, F, 100, Hq, Hkv, 128, 1e-6f, P, nullptr);
  };
  auto attention8 = [&](const laq_paged_batch* b, const uint8_t* ks, const uint8_t* vs, int64_t Hq = 32, int64_t Hkv = 8,
                        int64_t window = 0, int64_t bytes = (int64_t)1 << 40) {
    return laq_paged_attention_e4m3(b, ks, vs, P, Hq, Hkv, 128, window, P, P, bytes, nullptr);
  };
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)8, (int64_t)24, (int64_t)130, kMax}) {
    const auto each = [&](int64_t laq_paged_batch::*m, laq_status want) {
      laq_paged_batch b = batch();
      b.*m = v;
      EXPECT(append8(&b, S, S), want, "laq_paged_append_e4m3");
      EXPECT(attention8(&b, S, S), want, "laq_paged_attention_e4m3");
    };
    each(&laq_paged_batch::page_size, LAQ_ERR_BAD_SHAPE);
    each(&laq_paged_batch::slot_stride, v == 130 ? LAQ_ERR_MISALIGNED : LAQ_ERR_BAD_SHAPE);
    each(&laq_paged_batch::head_stride, v == 130 ? LAQ_ERR_MISALIGNED : LAQ_ERR_BAD_SHAPE);
    each(&laq_paged_batch::page_stride, v == 130 ? LAQ_ERR_MISALIGNED : LAQ_ERR_BAD_SHAPE);
    if (v == 8 || v == 24) continue;
    EXPECT(append8(&good, S, S, v, 8), LAQ_ERR_BAD_SHAPE, "laq_paged_append_e4m3");
    EXPECT(attention8(&good, S, S, v, 8), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_e4m3");
  }
  EXPECT(append8(nullptr, S, S), LAQ_ERR_NULL_POINTER, "laq_paged_append_e4m3");
  EXPECT(append8(&good, nullptr, S), LAQ_ERR_NULL_POINTER, "laq_paged_append_e4m3");
  EXPECT(append8(&good, S, nullptr), LAQ_ERR_NULL_POINTER, "laq_paged_append_e4m3");
  EXPECT(attention8(nullptr, S, S), LAQ_ERR_NULL_POINTER, "laq_paged_attention_e4m3");
  EXPECT(attention8(&good, nullptr, S), LAQ_ERR_NULL_POINTER, "laq_paged_attention_e4m3");
  EXPECT(attention8(&good, S, nullptr), LAQ_ERR_NULL_POINTER, "laq_paged_attention_e4m3");
  for (int64_t v : {kMin, (int64_t)-1, ((int64_t)1 << 30) + 1, kMax})
    EXPECT(attention8(&good, S, S, 32, 8, v), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_e4m3");
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0})
    EXPECT(attention8(&good, S, S, 32, 8, 0, v), LAQ_ERR_BAD_SHAPE, "laq_paged_attention_e4m3");
  {
    laq_paged_batch b = batch();
    b.T = (int64_t)1 << 18;  // 2^14 windows of 2 x 4096 + 512 waves, 2^33 threads
    EXPECT(append8(&b, S, S, 4096, 4096), LAQ_ERR_BAD_SHAPE, "laq_paged_append_e4m3");
  }

  fn = "laq_adjust_logits_f16";
  const uint32_t* const M = static_cast<const uint32_t*>(P);
  const laq_logits_adjust all = {I, I, I, 100, 100, F, F, F, I, F, 5, 5, M, 32};
  void* const O = off(P, 1 << 24);
  auto adjust = [&](const laq_logits_adjust* a, int64_t rows = 4, int64_t V = 1000, int64_t stride = 1000,
                    int64_t out_stride = 1000, const void* x = P, void* y = nullptr) {
    return laq_adjust_logits_f16(a, x, stride, rows, V, y ? y : O, out_stride, nullptr);
  };
  EXPECT(adjust(nullptr), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(adjust(&all, 4, 1000, 1000, 1000, nullptr), LAQ_ERR_NULL_POINTER, fn);
  EXPECT(laq_adjust_logits_f16(&all, P, 1000, 4, 1000, nullptr, 1000, nullptr), LAQ_ERR_NULL_POINTER, fn);
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)1 << 22, kMax}) EXPECT(adjust(&all, v), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)1001, (int64_t)(1 << 24) + 1, kMax})
    EXPECT(adjust(&all, 4, v), LAQ_ERR_BAD_SHAPE, fn);
  for (int64_t v : {kMin, (int64_t)-1, (int64_t)0, (int64_t)999, ((int64_t)1 << 32) + 1, kMax}) {
    EXPECT(adjust(&all, 4, 1000, v), LAQ_ERR_BAD_SHAPE, fn);
    EXPECT(adjust(&all, 4, 1000, 1000, v), LAQ_ERR_BAD_SHAPE, fn);
  }
  for (int64_t v : {kMin, (int64_t)-1, ((int64_t)1 << 32) + 1, kMax})
    for (int64_t laq_logits_adjust::*m : {&laq_logits_adjust::history_stride, &laq_logits_adjust::history_room,
                                          &laq_logits_adjust::bias_stride, &laq_logits_adjust::biases,
                                          &laq_logits_adjust::mask_stride}) {
      laq_logits_adjust a = all;
      a.*m = v;
      EXPECT(adjust(&a), LAQ_ERR_BAD_SHAPE, fn);
    }
  {
    laq_logits_adjust a = all;
    a.history_len = nullptr;
    EXPECT(adjust(&a), LAQ_ERR_NULL_POINTER, fn);
    a = all;
    a.bias_value = nullptr;
    EXPECT(adjust(&a), LAQ_ERR_NULL_POINTER, fn);
    a = all;
    a.mask = off(const_cast<uint32_t*>(M), 2);
    EXPECT(adjust(&a), LAQ_ERR_MISALIGNED, fn);
    a = all;
    a.repetition = off(F, 1);
    EXPECT(adjust(&a), LAQ_ERR_MISALIGNED, fn);
  }
  EXPECT(adjust(&all, 4, 1000, 1000, 1000, off(P, 1)), LAQ_ERR_MISALIGNED, fn);
  EXPECT(adjust(&all, 4, 1000, 1000, 1000, P, off(P, 1 << 12)), LAQ_ERR_BAD_SHAPE, fn);
  EXPECT(adjust(&all, 4, 1000, 1000, 1001, P, P), LAQ_ERR_BAD_SHAPE, fn);
  EXPECT(adjust(&all, (1 << 22) - 1, 1 << 24, (int64_t)1 << 32, (int64_t)1 << 32, P,
                reinterpret_cast<void*>((uintptr_t)1 << 62)), LAQ_ERR_BAD_SHAPE, fn);

  if (g_bad) {
    std::printf("%d of %d checks failed\n", g_bad, g_checks);
    return 1;
  }
  std::printf("ok %d\n", g_checks);
  return 0;
}

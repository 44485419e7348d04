// Driver for a ThreadSanitizer build of the batched serving entry points (host
// code), beside abi_threads.cpp: eight host threads call them at the same time, each with its own
// argument that the host-side validation must reject, check that the status and
// the calling thread's last-error text are those of its own call, and query the
// workspace size, which must not depend on what other threads do.  Nothing
// passes validation, so no HIP call is reached and no GPU is needed.  Prints
// "ok N" (N checks) on success; a wrong result returns 1, a report aborts.
#include <atomic>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <thread>
#include <vector>

#include "laq.h"

namespace {

std::atomic<int> g_checks{0}, g_bad{0};
void* const P = reinterpret_cast<void*>(0x100000);  // aligned, never dereferenced
float* const F = static_cast<float*>(P);
int32_t* const I = static_cast<int32_t*>(P);

void check(bool cond, int thread, const char* what) {
  g_checks.fetch_add(1, std::memory_order_relaxed);
  if (!cond) {
    if (g_bad.fetch_add(1) < 10) std::printf("thread %d: %s (last error \"%s\")\n", thread, what, laq_last_error());
  }
}

void call(int kind, int thread) {
  const laq_paged_batch good = {P, P, I, I, I, 10, 16, 8 * 16 * 128, 16 * 128, 128, 1000, 1000, 2, 3};
  laq_paged_batch b = good;
  laq_status st, want = LAQ_ERR_BAD_SHAPE;
  const char* fn = kind < 3 ? "laq_paged_append_f16" : kind < 6 ? "laq_paged_attention_f16" : "laq_sample_f16";
  switch (kind) {
    case 0: b.page_size = 24; st = laq_paged_append_f16(&b, P, 6144, P, P, F, 100, 32, 8, 128, 1e-6f, P, nullptr); break;
    case 1: st = laq_paged_append_f16(&b, P, 6144, P, P, F, 0, 32, 8, 128, 1e-6f, P, nullptr); break;
    case 2: b.seq_len = nullptr; want = LAQ_ERR_NULL_POINTER;
      st = laq_paged_append_f16(&b, P, 6144, P, P, F, 100, 32, 8, 128, 1e-6f, P, nullptr); break;
    case 3: st = laq_paged_attention_f16(&b, P, 32, 8, 128, -1, P, P, 1LL << 40, nullptr); break;
    case 4: st = laq_paged_attention_f16(&b, P, 32, 8, 128, 0, P, P, 16, nullptr); break;
    case 5: b.slot_stride = 132; want = LAQ_ERR_MISALIGNED;
      st = laq_paged_attention_f16(&b, P, 32, 8, 128, 0, P, P, 1LL << 40, nullptr); break;
    case 6: st = laq_sample_f16(P, 1000, 4, 0, F, F, I, F, F, I, F, nullptr); break;
    default: want = LAQ_ERR_NULL_POINTER; st = laq_sample_f16(P, 1000, 4, 1000, F, F, I, F, F, nullptr, F, nullptr); break;
  }
  check(st == want, thread, "wrong status");
  check(std::strstr(laq_last_error(), fn) != nullptr, thread, "last error names another call");
}

}  // namespace

int main() {
  const int64_t small = laq_paged_attention_workspace_bytes(16, 16, 32, 8, 8192);
  const int64_t large = laq_paged_attention_workspace_bytes(300, 9000, 40, 8, 1 << 20);
  std::vector<std::thread> threads;
  for (int t = 0; t < 8; ++t) {
    threads.emplace_back([t, small, large] {
      for (int i = 0; i < 3000; ++i) {
        call(t, t);
        if (i % 7 == 0) {
          check(laq_paged_attention_workspace_bytes(16, 16, 32, 8, 8192) == small, t, "workspace size changed");
          check(laq_paged_attention_workspace_bytes(300, 9000, 40, 8, 1 << 20) == large, t, "workspace size changed");
        }
      }
    });
  }
  for (auto& th : threads) th.join();
  if (g_bad.load() != 0) {
    std::printf("%d of %d checks failed\n", g_bad.load(), g_checks.load());
    return 1;
  }
  std::printf("ok %d\n", g_checks.load());
  return 0;
}

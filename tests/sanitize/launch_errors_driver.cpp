// Launches that fail: each call of the scores of tokens and of the embedding has to report
// it, whichever of its launches it was. This program's own hipLaunchKernel,
// hipGetLastError and the two calls around a <<< >>> stand before the runtime's; nothing reaches a GPU, and the addresses
// below are never dereferenced. Exit status: failed checks.
#include <cstdint>
#include <cstdio>

#include "tkef.h"

static int g_fail = 0;
static int g_launches = 0, g_failing = 0;  // the g_failing-th launch of a call fails; 0: none
static hipError_t g_last = hipSuccess;

extern "C" __attribute__((visibility("default"))) hipError_t hipLaunchKernel(
    const void*, dim3, dim3, void**, size_t, hipStream_t) {
  if (++g_launches != g_failing) return hipSuccess;
  g_last = hipErrorInvalidConfiguration;
  return g_last;
}

extern "C" __attribute__((visibility("default"))) hipError_t __hipPushCallConfiguration(
    dim3, dim3, size_t, hipStream_t) {
  return hipSuccess;
}
extern "C" __attribute__((visibility("default"))) hipError_t __hipPopCallConfiguration(
    dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = *block = dim3(1);
  *lds = 0;
  *stream = nullptr;
  return hipSuccess;
}

// the last failure, once
extern "C" __attribute__((visibility("default"))) hipError_t hipGetLastError(void) {
  const hipError_t e = g_last;
  g_last = hipSuccess;
  return e;
}

template <typename T>
static T* at(uintptr_t a) {
  return reinterpret_cast<T*>(a);
}

template <typename F>
static void check(const char* name, F call) {
  g_failing = g_launches = 0;
  int rc = call();
  const int launches = g_launches;
  if (rc != TKEF_OK || launches < 1) {
    std::fprintf(stderr, "%s: %d with %d launches\n", name, rc, launches);
    ++g_fail;
  }
  for (int i = 1; i <= launches; ++i) {
    g_failing = i;
    g_launches = 0;
    g_last = hipSuccess;
    rc = call();
    if (rc != TKEF_EHIP) {
      std::fprintf(stderr, "%s: launch %d of %d fails, the call returns %d\n", name, i, launches,
                   rc);
      ++g_fail;
    }
  }
  g_failing = 0;
  g_last = hipSuccess;
}

int main() {
  const int32_t* t = at<int32_t>(0x1000);
  float* f = at<float>(0x100000);
  int32_t* i = at<int32_t>(0x3000);
  void* w = at<void>((uintptr_t)1 << 40);
  void* x = at<void>((uintptr_t)1 << 41);
  void* y = at<void>((uintptr_t)1 << 42);

  for (int32_t dtype = 0; dtype < 3; ++dtype)
    for (int64_t v : {1000, 200000})
      for (int64_t k : {0, 20}) {
        tkef_score_plan p = nullptr;
        size_t ws = 0;
        if (tkef_score_plan_create(64, v, k, dtype, 1.0, &p) != TKEF_OK) return 100;
        (void)tkef_score_plan_info(p, &ws);
        check("score forward", [&] {
          return tkef_score_forward(p, x, v, 64, t, f, f, k > 0 ? i : nullptr,
                                    k > 0 ? f : nullptr, f, w, ws, nullptr, nullptr);
        });
        check("score backward",
              [&] { return tkef_score_backward(p, x, v, 64, t, f, f, f, y, v, nullptr, nullptr); });
        (void)tkef_score_plan_destroy(p);
      }

  for (int32_t out = 0; out < 3; ++out)
    for (int32_t grad = 0; grad < 3; ++grad)
      for (int64_t n : {5, 300, 5000, 20000})
        for (int64_t width : {3, 512}) {
          tkef_embed_plan p = nullptr;
          size_t ws = 0;
          if (tkef_embed_plan_create(n, 1000, width, grad, out, grad,
                                     grad == TKEF_DTYPE_F16 ? TKEF_VAL_F16 : TKEF_VAL_F32, 1.0,
                                     &p) != TKEF_OK)
            return 100;
          (void)tkef_embed_plan_info(p, &ws);
          check("embed forward", [&] {
            return tkef_embed_forward(p, x, width, t, n, y, width, nullptr, nullptr);
          });
          check("embed backward", [&] {
            return tkef_embed_backward(p, t, n, x, width, nullptr, 0, y, width, w, ws, nullptr,
                                       nullptr);
          });
          check("embed lists", [&] {
            return tkef_embed_lists(p, t, n, x, width, 0, i, f, i, w, ws, nullptr, nullptr);
          });
          // no tokens: a list has no entries, so nothing has to hold them
          check("embed lists of no tokens", [&] {
            return tkef_embed_lists(p, nullptr, 0, nullptr, width, 0, nullptr, nullptr, i, w, ws,
                                    nullptr, nullptr);
          });
          (void)tkef_embed_plan_destroy(p);
        }
  std::printf("%d failed checks\n", g_fail);
  return g_fail > 99 ? 99 : g_fail;
}

// Drives the row operators' host code (plans, workspace sizes, argument checks)
// through the C ABI without a GPU. Addresses below are never dereferenced: every
// call ends in an argument error, or in zero rows. Exit status: failed checks.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "tkef.h"

static int g_fail = 0;
#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      std::fprintf(stderr, "line %d: failed: %s\n", __LINE__, #x);  \
      ++g_fail;                                                     \
    }                                                               \
  } while (0)

static void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }

static void lists() {
  const int64_t rows[] = {1, 7, 1 << 20}, vocab[] = {1, 7, 1000, 16385, 131073, 1 << 20};
  const int64_t ks[] = {1, 5, 64, 256, 1024};
  for (int64_t n : rows)
    for (int64_t v : vocab)
      for (int64_t k : ks)
        for (int32_t dtype = 0; dtype < 3; ++dtype)
          for (int32_t val = 0; val < 2; ++val) {
            const int want = k <= v ? TKEF_OK : TKEF_ERANGE;
            tkef_top_plan t = nullptr;
            tkef_distill_plan d = nullptr;
            CHECK(tkef_top_plan_create(n, v, k, dtype, val, 0.7, &t) == want);
            CHECK(tkef_distill_plan_create(n, v, k, dtype, val, 0.7, &d) == want);
            if (want != TKEF_OK) {
              CHECK(t == nullptr && d == nullptr);
              continue;
            }
            size_t wt = 1, wd = 1;
            CHECK(tkef_top_plan_info(t, &wt) == TKEF_OK && wt % 256 == 0);
            CHECK(tkef_distill_plan_info(d, &wd) == TKEF_OK && wd % 256 == 0);
            CHECK(tkef_top_plan_info(t, nullptr) == TKEF_OK);
            int32_t* idx = static_cast<int32_t*>(at(0x10000));
            float* f = static_cast<float*>(at(0x20000));
            if (wt > 0)
              CHECK(tkef_top_execute(t, at(0x1000), v, n, idx, f, f, nullptr, 0, nullptr,
                                     nullptr) == TKEF_EWORKSPACE);
            CHECK(tkef_top_execute(t, nullptr, v, 0, nullptr, nullptr, nullptr, at(0x1000), wt,
                                   nullptr, nullptr) == TKEF_OK);
            CHECK(tkef_top_execute(t, at(0x1000), v - 1, n, idx, f, f, at(0x1000), wt, nullptr,
                                   nullptr) == TKEF_EINVAL);
            CHECK(tkef_distill_step(d, at(0x1000), v, n, idx, f, nullptr, nullptr, nullptr, f,
                                    at(0x1000), v + 1, at(0x1000), wd, nullptr,
                                    nullptr) == TKEF_EINVAL);  // the logits' address, other rows
            CHECK(tkef_distill_forward(d, at(0x1000), v, n + 1, idx, f, nullptr, nullptr, nullptr,
                                       f, nullptr, at(0x1000), wd, nullptr,
                                       nullptr) == TKEF_ERANGE);
            CHECK(tkef_distill_backward(d, at(0x1000), v, n, nullptr, f, nullptr, nullptr, nullptr,
                                        f, nullptr, f, v, at(0x1000), wd, nullptr,
                                        nullptr) == TKEF_EINVAL);
            CHECK(tkef_top_plan_destroy(t) == TKEF_OK);
            CHECK(tkef_distill_plan_destroy(d) == TKEF_OK);
          }
  tkef_top_plan t = nullptr;
  for (double bad : {0.0, -1.0, 1e7, (double)NAN, (double)INFINITY})
    CHECK(tkef_top_plan_create(1, 10, 1, 0, 0, bad, &t) == TKEF_ERANGE);
  CHECK(tkef_top_plan_create(1, 10, 1, 0, 0, 1.0, nullptr) == TKEF_EINVAL);
}

static void drafts() {
  for (int64_t b : {1, 37, 32768})
    for (int64_t n : {1, 8, 63})
      for (int64_t v : {1, 1000, 32000, 1 << 20}) {
        tkef_verify_plan p = nullptr;
        const int rc = tkef_verify_plan_create(b, n, v, TKEF_DTYPE_F32, 1.0, &p);
        const int64_t pieces = b * (n + 1) * ((v / 4 + 4095) / 4096 > 0 ? (v / 4 + 4095) / 4096 : 1);
        CHECK(rc == (pieces <= 1 << 21 ? TKEF_OK : TKEF_ERANGE));
        if (rc != TKEF_OK) continue;
        size_t ws = 0;
        CHECK(tkef_verify_plan_info(p, &ws) == TKEF_OK && ws > 0 && ws % 256 == 0);
        CHECK(tkef_verify_plan_bind(p, nullptr, ws, nullptr) == TKEF_EWORKSPACE);
        CHECK(tkef_verify_plan_bind(p, at(0x1000), ws - 1, nullptr) == TKEF_EWORKSPACE);
        int32_t* i = static_cast<int32_t*>(at(0x10000));
        float* f = static_cast<float*>(at(0x20000));
        CHECK(tkef_verify_execute(p, at(0x1000), 0, v, at(0x2000), 0, v, 0, i, f, f, v, nullptr, i,
                                  i, f, at(0x1000), ws, nullptr, nullptr) == TKEF_OK);
        CHECK(tkef_verify_execute(p, at(0x1000), 0, v, at(0x2000), 0, v, b, i, f, f, v - 1, nullptr,
                                  i, i, f, at(0x1000), ws, nullptr, nullptr) == TKEF_EINVAL);
        CHECK(tkef_verify_execute(p, at(0x1000), 0, v, at(0x2000), 0, v, b, i, f, f, v, nullptr, i,
                                  i, f, at(0x1040), ws, nullptr, nullptr) == TKEF_EWORKSPACE);
        CHECK(tkef_verify_plan_destroy(p) == TKEF_OK);
      }
}

int main() {
  lists();
  drafts();
  std::printf("%d failed checks\n", g_fail);
  return g_fail != 0;
}

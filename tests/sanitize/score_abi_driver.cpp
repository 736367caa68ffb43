// Drives the host code of the scores of tokens and of the embedding (plans, workspace
// sizes, argument checks) through the C ABI without a GPU. Addresses below are never
// dereferenced: every call ends in an argument error, or in zero rows. Exit status: failed
// checks.
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

template <typename T>
static T* at(uintptr_t a) {
  return reinterpret_cast<T*>(a);
}

static void scores() {
  const int64_t rows[] = {1, 7, 1 << 20}, vocab[] = {1, 7, 1000, 16385, 131073, 1 << 20};
  const int64_t ks[] = {0, 1, 5, 64};
  for (int64_t n : rows)
    for (int64_t v : vocab)
      for (int64_t k : ks)
        for (int32_t dtype = 0; dtype < 3; ++dtype) {
          tkef_score_plan p = nullptr;
          const int want = k <= v ? TKEF_OK : TKEF_ERANGE;
          CHECK(tkef_score_plan_create(n, v, k, dtype, 0.7, &p) == want);
          CHECK((p != nullptr) == (want == TKEF_OK));
          if (p == nullptr) continue;
          size_t ws = 1;
          CHECK(tkef_score_plan_info(p, &ws) == TKEF_OK && ws % 256 == 0);
          CHECK(tkef_score_plan_info(p, nullptr) == TKEF_OK);
          const int32_t* t = at<int32_t>(0x1000);
          float* f = at<float>(0x2000);
          int32_t* i = at<int32_t>(0x3000);
          void* w = at<void>(0x10000);
          if (ws > 0)
            CHECK(tkef_score_forward(p, f, v, n, t, f, f, i, f, f, nullptr, 0, nullptr,
                                     nullptr) == TKEF_EWORKSPACE);
          CHECK(tkef_score_forward(p, nullptr, v, 0, nullptr, nullptr, nullptr, nullptr, nullptr,
                                   nullptr, w, ws, nullptr, nullptr) == TKEF_OK);
          CHECK(tkef_score_forward(p, f, v - 1, n, t, f, f, i, f, f, w, ws, nullptr, nullptr) ==
                TKEF_EINVAL);
          CHECK(tkef_score_forward(p, f, v, n + 1, t, f, f, i, f, f, w, ws, nullptr, nullptr) ==
                TKEF_ERANGE);
          CHECK(tkef_score_backward(p, f, v, n, t, f, f, f, f, v + 1, nullptr, nullptr) ==
                TKEF_EINVAL);  // the logits' address, other rows
          CHECK(tkef_score_plan_destroy(p) == TKEF_OK);
        }
}

static void embeddings() {
  const int64_t rows[] = {1, 9, 40000, 1 << 20}, vocab[] = {1, 1000, 131073, 1 << 20};
  const int64_t width[] = {1, 515, 1 << 16};
  for (int64_t n : rows)
    for (int64_t v : vocab)
      for (int64_t d : width)
        for (int32_t dtype = 0; dtype < 3; ++dtype) {
          tkef_embed_plan p = nullptr;
          CHECK(tkef_embed_plan_create(n, v, d, dtype, 2 - dtype, dtype, dtype % 2, -3.5, &p) ==
                TKEF_OK);
          if (p == nullptr) continue;
          size_t ws = 1;
          CHECK(tkef_embed_plan_info(p, &ws) == TKEF_OK && ws % 256 == 0 && ws > 0);
          CHECK(tkef_embed_plan_info(p, nullptr) == TKEF_OK);
          const int32_t* t = at<int32_t>(0x1000);
          void* x = at<void>(0x100000);
          int32_t* i = at<int32_t>(0x3000);
          void* w = at<void>(0x10000);
          CHECK(tkef_embed_forward(p, x, d, t, 0, nullptr, 0, nullptr, nullptr) == TKEF_OK);
          CHECK(tkef_embed_forward(p, x, d, t, n, x, d, nullptr, nullptr) == TKEF_EINVAL);
          CHECK(tkef_embed_forward(p, x, (int64_t)1 << 40, t, n, x, d, nullptr, nullptr) ==
                TKEF_EINVAL);
          CHECK(tkef_embed_forward(p, x, INT64_MAX, t, n, x, d, nullptr, nullptr) == TKEF_ERANGE);
          CHECK(tkef_embed_forward(p, x, INT64_MIN, t, n, x, d, nullptr, nullptr) == TKEF_EINVAL);
          CHECK(tkef_embed_backward(p, t, n, x, d, nullptr, 0, x, d, w, ws, nullptr, nullptr) ==
                TKEF_EINVAL);
          CHECK(tkef_embed_backward(p, t, n, x, d, nullptr, 0, nullptr, d, w, ws - 1, nullptr,
                                    nullptr) == TKEF_EWORKSPACE);
          CHECK(tkef_embed_lists(p, t, n, x, d, INT64_MAX, i, x, i, w, ws, nullptr, nullptr) ==
                TKEF_ERANGE);
          CHECK(tkef_embed_lists(p, t, n, x, d, INT64_MIN, i, x, i, w, ws, nullptr, nullptr) ==
                TKEF_ERANGE);
          CHECK(tkef_embed_lists(p, t, n + 1, x, d, 0, i, x, i, w, ws, nullptr, nullptr) ==
                TKEF_ERANGE);
          CHECK(tkef_embed_plan_destroy(p) == TKEF_OK);
        }
  tkef_embed_plan p = nullptr;
  CHECK(tkef_embed_plan_create(1, 1, 1, 0, 0, 0, 0, 1e300, &p) == TKEF_ERANGE && p == nullptr);
  CHECK(tkef_embed_plan_create(INT64_MAX, 1, 1, 0, 0, 0, 0, 1.0, &p) == TKEF_ERANGE);
  CHECK(tkef_embed_plan_create(1, 1, INT64_MIN, 0, 0, 0, 0, 1.0, &p) == TKEF_ERANGE);
}

int main() {
  scores();
  embeddings();
  std::printf("%d failed checks\n", g_fail);
  return g_fail != 0;
}

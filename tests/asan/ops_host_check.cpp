// Host paths of the operators in paged_attn_ops.h under the sanitizers: valid
// and random arguments, with launchers that launch nothing (a call whose checks
// pass returns PA_EHIP).
#include "paged_attn_ops.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      std::printf("%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, pa_last_error()); \
      return 1;                                                         \
    }                                                                   \
  } while (0)

int main() {
  void* dev = reinterpret_cast<void*>(0x10000);
  float* fdev = static_cast<float*>(dev);
  int32_t* idev = static_cast<int32_t*>(dev);
  std::mt19937 rng(7);
  auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };

  for (int r = 0; r <= 256; r += 2)
    for (int kind = 0; kind < 5; ++kind) {
      double* freqs = static_cast<double*>(std::malloc(r / 2 * sizeof(double) + 1));
      double magnitude = 0;
      CHECK(pa_rope_frequencies(r, 10000.0, kind, 8.0, 4096.0, 1.0, 32.0, freqs, &magnitude) == PA_OK);
      for (int layout = 0; layout < 2; ++layout) {
        pa_rope* rope = nullptr;
        const int rc = pa_rope_create(256, r, layout, freqs, magnitude, &rope);
        CHECK(rc == (r % 16 == 0 ? PA_OK : PA_EUNSUPPORTED) && (rope != nullptr) == (rc == PA_OK));
        CHECK(pa_rope_destroy(rope) == PA_OK);
      }
      std::free(freqs);
    }

  double freqs[64];
  for (double& f : freqs) f = 0.5;
  pa_rope* rope = nullptr;
  CHECK(pa_rope_create(128, 128, PA_ROPE_HALF, freqs, 1.0, &rope) == PA_OK);
  pa_kv_pool* pool = nullptr;
  CHECK(kv_pool_create(100, 16, 8, 128, dev, dev, &pool) == PA_OK);
  CHECK(paged_attn_norm_rope(rope, dev, 4096, 32, fdev, dev, 1024, 8, fdev, 1e-6f, PA_BF16, idev, 7, dev, 4096, dev,
                             1024, nullptr) == PA_EHIP);
  CHECK(paged_attn_rope_append(pool, rope, dev, 4096, 32, fdev, dev, 1024, fdev, dev, 1024, 1e-6f, PA_FP32, nullptr,
                               idev, 9, idev, 10, idev, 3, dev, nullptr) == PA_EHIP);
  size_t bytes = 0;
  CHECK(paged_attn_biased_workspace_size(pool, 1, 32, 100000, 1, 0, &bytes) == PA_OK && bytes > 0);
  CHECK(paged_attn_decode_biased(pool, dev, idev, 6250, idev, 1, 32, 0.1f, 30.f, fdev, 0, idev, 100000, dev, bytes, dev,
                                 nullptr) == PA_EHIP);
  CHECK(paged_attn_decode_biased(pool, dev, idev, 6250, idev, 1, 32, 0.1f, 30.f, fdev, 0, idev, 100000, dev, bytes - 1,
                                 dev, nullptr) == PA_EINVAL);

  const int64_t big = 2147483647;
  int launched = 0;
  for (int i = 0; i < 200000; ++i) {
    const int32_t hq = (int32_t)pick({0, 8, 32, 64, 7, -1, big, 8 * 100000}), batch = (int32_t)pick({0, 1, 3, 1000, big, -5});
    const int32_t ctx = (int32_t)pick({0, 1, 100, 8192, 100000, big, -1}), chunk = (int32_t)pick({0, 1, 7, 100, 8192, big, -1});
    const int32_t stride = (int32_t)pick({0, 1, 10, 6250, 134217727, 134217728, big, -1});
    const int32_t window = (int32_t)pick({0, 1, 4096, big, -1}), total = (int32_t)pick({0, 1, 50, big, -1});
    const float scale = (float)pick({0, 1, -1}), cap = (float)pick({0, 30, 1, -1, 2000000000});
    const int64_t qs = pick({0, 4096, 4100, -4096, big, (int64_t)1 << 62, (int64_t)-1 << 62});
    void* p = reinterpret_cast<void*>(pick({0, 0x10000, 0x10004, 0x10001}));
    size_t need = 0;
    int rc = paged_attn_biased_workspace_size(pool, batch, hq, ctx, chunk, window, &need);
    CHECK(rc == PA_OK || rc == PA_EINVAL);
    rc = paged_attn_decode_biased(pool, p, idev, stride, idev, batch, hq, scale, cap, nullptr, window, nullptr, ctx, dev,
                                  (size_t)1 << 60, dev, nullptr);
    CHECK(rc == PA_OK || rc == PA_EINVAL || rc == PA_EHIP);
    launched += rc == PA_EHIP;
    rc = paged_attn_extend_biased(pool, dev, idev, total, idev, stride, idev, batch, hq, scale, cap, fdev, window, idev,
                                  static_cast<int32_t*>(p), ctx, chunk, dev, need, dev, nullptr);
    CHECK(rc == PA_OK || rc == PA_EINVAL || rc == PA_EHIP);
    launched += rc == PA_EHIP;
    rc = paged_attn_norm_rope(rope, p, qs, hq, nullptr, dev, 1024, (int32_t)pick({0, 8, -1, big}), nullptr, scale, chunk,
                              idev, total, dev, 4096, dev, qs, nullptr);
    CHECK(rc == PA_OK || rc == PA_EINVAL || rc == PA_EHIP);
    launched += rc == PA_EHIP;
    rc = paged_attn_rope_append(pool, rope, dev, qs, hq, fdev, dev, 1024, nullptr, p, 1024, cap, window, nullptr, idev,
                                total, idev, stride, idev, batch, dev, nullptr);
    CHECK(rc == PA_OK || rc == PA_EINVAL || rc == PA_EHIP);
    launched += rc == PA_EHIP;
  }
  CHECK(launched > 1000);
  CHECK(pa_rope_destroy(rope) == PA_OK && kv_pool_destroy(pool) == PA_OK);
  std::printf("host operator checks passed\n");
  return 0;
}

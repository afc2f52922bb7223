// The rotary entry points' host code against the HIP stand-in: handles of every kind, and calls
// of every operator, which allocate nothing and reach their launches with the caller's
// arguments.  Launches are stubbed here and in stubs.cpp.
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>

#include "fake_hip.h"
#include "rotary_calls.h"

#define CHECK(cond)                                                          \
  do {                                                                       \
    if (!(cond)) {                                                           \
      std::fprintf(stderr, "check failed: %s (line %d)\n", #cond, __LINE__); \
      return 1;                                                              \
    }                                                                        \
  } while (0)

namespace libra {
namespace {
int g_rotary = 0, g_append = 0, g_write = 0, g_decode = 0, g_chunk = 0;
}
hipError_t launch_rotary(const Rotary&, const RotaryRows&, hipStream_t) { return ++g_rotary, hipSuccess; }
hipError_t launch_kv_append(const KvLayout&, const NewRows&, const int64_t*, int64_t, int32_t, void*,
                            hipStream_t) { return ++g_append, hipSuccess; }
hipError_t launch_cache_write_rotary(const KvLayout&, const Plan&, const void*, const NewRows&,
                                     const int32_t*, int32_t, hipStream_t) { return ++g_write, hipSuccess; }
hipError_t launch_decode_rotary(const KvLayout&, const Plan&, void*, const NewRows&, const int32_t*,
                                int32_t, float, void*, float*, bool, hipStream_t) { return ++g_decode, hipSuccess; }
hipError_t launch_chunk_rotary(const KvLayout&, const Plan&, void*, const NewRows&, const int32_t*,
                               int32_t, float, void*, float*, hipStream_t) { return ++g_chunk, hipSuccess; }
}  // namespace libra

using namespace libra;

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](int n) { return int(rng() % uint64_t(n)); };
  int made = 0;
  for (int i = 0; i < 3000; ++i) {
    std::vector<double> f(128);
    for (double& x : f) x = std::ldexp(double(rng() >> 11) / (1ull << 53) - 0.5, pick(30) - 8);
    libra_rotary_desc d{};
    d.head_dim = pick(520);
    d.rotary_dim = pick(3) ? 0 : pick(260);
    d.pairing = pick(3) ? pick(2) : pick(4) - 1;
    d.scaling = pick(5);
    d.base = std::exp(double(pick(40)) - 5);
    d.factor = pick(10);
    d.original_length = pick(4) ? 1 << pick(20) : -1;
    d.slow = pick(3);
    d.fast = pick(40);
    d.amplitude = pick(4) ? 0 : 0.5 * pick(5);
    d.frequencies = pick(3) ? nullptr : f.data();
    libra_rotary h = nullptr;
    if (libra_rotary_create(&d, &h) != LIBRA_OK) {
      CHECK(!h);
      continue;
    }
    ++made;
    int32_t R = 0;
    double theta[128], amp = 0;
    CHECK(libra_rotary_get(h, nullptr, &R, theta, &amp) == LIBRA_OK && R >= 2 && R <= 256 && amp > 0);
    for (int j = 0; j < R / 2; ++j) CHECK(std::isfinite(theta[j]));
    libra_rotary_destroy(h);
  }
  CHECK(made > 100);

  const int B = 4, hq = 8, hkv = 2;
  const int32_t lens[B] = {300, 17, 90, 2048}, news[B] = {1, 17, 80, 1};
  const int rows = 99, pages = 200;
  std::vector<unsigned char> cache(size_t(pages) * hkv * 4096 + 16), buf(1 << 20);
  auto al = [](std::vector<unsigned char>& v, size_t n) {
    return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(v.data()) + n - 1) & ~uintptr_t(n - 1));
  };
  libra_kv_layout_desc ld{pages, 16, hkv, 128, LIBRA_DTYPE_BF16, al(cache, 16), al(cache, 16)};
  libra_kv_layout lay = nullptr;
  CHECK(libra_kv_layout_create(&ld, &lay) == LIBRA_OK);
  libra_rotary_desc rd{};
  rd.head_dim = 128;
  rd.base = 1e4;
  libra_rotary rot = nullptr;
  CHECK(libra_rotary_create(&rd, &rot) == LIBRA_OK);
  libra_plan_desc pd{LIBRA_MODE_APPEND, B, hq, hkv};
  libra_plan plan = nullptr;
  CHECK(libra_splitkv_plan(&pd, lens, news, nullptr, &plan) == LIBRA_OK);
  std::vector<unsigned char> wsv(libra_plan_workspace_bytes(plan) + 256);
  void* ws = al(wsv, 256);
  const size_t ws_bytes = libra_plan_workspace_bytes(plan);
  void* p = al(buf, 16);
  const int32_t* i32 = static_cast<const int32_t*>(p);
  const int64_t* i64 = static_cast<const int64_t*>(p);
  const long before = g_fake_hip.allocations();
  long copies = 0;
  for (int i = 0; i < 3; ++i) {
    CHECK(libra_rotary_apply(rot, LIBRA_DTYPE_FP32, p, 1024, 128, i32, rows, hq, 128, i & 1, p, 1024, 128,
                             nullptr) == LIBRA_OK);
    CHECK(libra_kv_append(lay, rot, i32, i64, rows, p, 1536, hq, p, 1536, p, 1536, hkv, p, nullptr) ==
          LIBRA_E_INVAL);  // in place, but q's rows are not dense
    CHECK(libra_kv_append(lay, rot, i32, i64, rows, p, 1024, hq, p, 1536, p, 1536, hkv, p, nullptr) ==
          LIBRA_OK);
    CHECK(libra_append_attn_rotary(lay, plan, rot, nullptr, rows, p, 1536, p, 1536, p, 1536, hkv, i32, 200, B,
                                   hq, 0.1f, i & 1, ws, ws_bytes, p, nullptr, nullptr) == LIBRA_OK);
    if (i == 0) copies = g_fake_hip.memcpy_async;
  }
  CHECK(g_rotary == 3 && g_append == 3 && g_write == 3 && g_decode == 3 && g_chunk == 3);
  CHECK(g_fake_hip.allocations() == before);
  CHECK(copies > 0 && g_fake_hip.memcpy_async == copies);  // the tables go up once
  libra_plan_destroy(plan);
  libra_rotary_destroy(rot);
  libra_kv_layout_destroy(lay);
  std::printf("rotary host ok (%d handles)\n", made);
  return 0;
}

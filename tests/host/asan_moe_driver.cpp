// Host-only exercise of the argument checks of the router, the 8-bit calls and the experts under
// AddressSanitizer and UndefinedBehaviorSanitizer: random sizes up to the types' ends, some
// pointers missing or unaligned.  No call gets as far as a launch: it holds no row, lacks a
// pointer, or its workspace is a byte short.  Addresses are made up and never read.
#include <cstdint>
#include <cstdio>
#include <limits>
#include <random>

#include "mla_online.h"

static std::mt19937_64 rng(11);

template <class T>
static T pick(std::initializer_list<T> v) {
  return v.begin()[rng() % v.size()];
}

static int32_t any32() {
  switch (rng() % 4) {
    case 0: return (int32_t)rng();
    case 1: return pick<int32_t>({std::numeric_limits<int32_t>::min(), -1, 0, 1, std::numeric_limits<int32_t>::max()});
    default: return (int32_t)(rng() % 512);
  }
}

static int64_t any64() {
  switch (rng() % 3) {
    case 0: return (int64_t)rng();
    case 1: return pick<int64_t>({std::numeric_limits<int64_t>::min(), -1, 0, 1, int64_t(1) << 31, int64_t(1) << 62, std::numeric_limits<int64_t>::max()});
    default: return any32();
  }
}

// an address of this alignment, now and then another or none
template <class T = void>
static T* at(uintptr_t align) {
  const int k = rng() % 16;
  return k == 0 ? nullptr : reinterpret_cast<T*>(align * (1 + rng() % 99) + (k == 1 ? 1 + rng() % align : 0));
}

static float anyf() {
  return pick<float>({0.f, 1.f, -2.5f, 0.9f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN(), 1e30f});
}

int main() {
  int64_t met[8] = {0};
  auto count = [&](mla_status s) {
    if (s < MLA_OK || s >= MLA_ERR_HIP || (s != MLA_OK) != (mla_last_error_detail()[0] != 0)) {
      printf("status %d, detail '%s'\n", (int)s, mla_last_error_detail());
      return false;
    }
    ++met[s];
    return true;
  };
  for (int it = 0; it < 200000; ++it) {
    const int32_t experts = rng() % 3 ? pick({1, 8, 60, 256, 1024}) : any32();
    mla_route_cfg cfg{(int32_t)(rng() % 2), 1, 1, 1, 1 + (int32_t)(rng() % 8), 1, (int32_t)(rng() % 2), 1.f, 0.9f};
    switch (rng() % 10) {
      case 0: cfg.scoring = any32(); break;
      case 1: cfg.n_groups = any32(); break;
      case 2: cfg.n_groups = 8; cfg.top_groups = rng() % 2 ? 1 + (int32_t)(rng() % 9) : any32(); break;
      case 3: cfg.group_best = any32(); break;
      case 4: cfg.top_k = any32(); break;
      case 5: cfg.min_k = any32(); break;
      case 6: cfg.scale = anyf(); break;
      case 7: cfg.tau = anyf(); break;
      default: break;
    }
    const mla_route_cfg* cp = rng() % 64 ? &cfg : nullptr;
    const int32_t type = rng() % 4 ? (int32_t)(rng() % 2) : any32();
    const int64_t stride = rng() % 3 ? (int64_t)experts + (int64_t)(rng() % 5) : any64();
    // no row, or some and nowhere to write them
    if (!count(mla_moe_route(0, experts, at(16), type, stride, at<float>(4), cp, at<int32_t>(4), at<float>(4), at<int32_t>(4), nullptr, nullptr)) ||
        !count(mla_moe_route(any64() | 1, experts, at(16), type, stride, nullptr, cp, nullptr, at<float>(4), nullptr, nullptr, nullptr)))
      return 1;
    const int32_t cols = rng() % 3 ? 16 * (int32_t)(rng() % 1200) : any32();
    const int64_t xs = rng() % 3 ? cols + 8 * (int64_t)(rng() % 3) : any64();
    const int64_t rows = rng() % 3 ? 0 : -1 - (int64_t)(rng() >> 2);
    if (!count(mla_i8_quantize(rows, cols, at(16), xs, at(16), at<float>(4), nullptr)) ||
        !count(mla_i8_dequantize(rows, cols, at(16), at<float>(4), at(16), xs, nullptr)) ||
        !count(mla_i8_quantize((int64_t)(rng() >> 1) | 1, cols, at(16), xs, nullptr, at<float>(4), nullptr)) ||
        !count(mla_i8_dequantize((int64_t)(rng() >> 1) | 1, cols, nullptr, at<float>(4), at(16), xs, nullptr)))
      return 1;
    const int32_t d_in = rng() % 3 ? 64 * (int32_t)(rng() % 300) : any32(), d_out = rng() % 2 ? any32() : 1 + (int32_t)(rng() % 100000);
    if (!count(mla_shared_wb_i8(0, d_in, d_out, at(16), at<float>(4), at(16), at<float>(4), type, at(16), nullptr)) ||
        !count(mla_shared_wb_i8(any64() | 1, d_in, d_out, nullptr, at<float>(4), at(16), at<float>(4), type, at(16), nullptr)))
      return 1;
    mla_moe_layer layer{64 * (1 + (int32_t)(rng() % 256)), 64 * (1 + (int32_t)(rng() % 256)), 1 + (int32_t)(rng() % 1024), (int32_t)(rng() % 99), 1 + (int32_t)(rng() % 16)};
    switch (rng() % 10) {
      case 0: layer.d_model = any32(); break;
      case 1: layer.d_ffn = any32(); break;
      case 2: layer.n_experts = any32(); break;
      case 3: layer.first_expert = any32(); break;
      case 4: layer.top_k = any32(); break;
      default: break;
    }
    const mla_moe_layer* lp = rng() % 64 ? &layer : nullptr;
    const int64_t n = rng() % 3 ? (int64_t)(rng() % 100000) : any64();
    size_t ws = 0;
    const mla_status q = mla_moe_experts_i8_query(lp, n, type, rng() % 64 ? &ws : nullptr);
    if (!count(q)) return 1;
    if (q == MLA_OK && (ws == 0 || ws > (size_t(1) << 38))) {
      printf("workspace of %zu bytes\n", ws);
      return 1;
    }
    const size_t given = q == MLA_OK ? ws - 1 : rng() % 1000;
    const int64_t x_stride = rng() % 3 ? layer.d_model : any64();
    const mla_status e = mla_moe_experts_i8(lp, n, at(16), x_stride, at<int32_t>(4), at<float>(4), at<int32_t>(4), at(16), at<float>(16), at(16),
                                            at<float>(16), type, at(16), at(256), given, nullptr);
    if (!count(e)) return 1;
    if (e == MLA_OK && n != 0) {
      printf("a workspace of %zu of %zu bytes was accepted\n", given, ws);
      return 1;
    }
  }
  printf("calls: %lld accepted without a row, refused %lld NULL %lld shape %lld unsupported %lld workspace\n", (long long)met[MLA_OK],
         (long long)met[MLA_ERR_NULL], (long long)met[MLA_ERR_SHAPE], (long long)met[MLA_ERR_UNSUPPORTED], (long long)met[MLA_ERR_WORKSPACE]);
  return met[MLA_OK] && met[MLA_ERR_NULL] && met[MLA_ERR_SHAPE] && met[MLA_ERR_UNSUPPORTED] && met[MLA_ERR_WORKSPACE] ? 0 : 1;
}

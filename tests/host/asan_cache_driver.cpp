// Host-only exercise of the argument checks of the 4-bit and cache entry points under
// AddressSanitizer and UndefinedBehaviorSanitizer: random sizes up to the types' ends, some
// pointers missing or unaligned.  No call gets as far as a launch: it holds no row, or its
// workspace is a byte short.  Addresses are made up and never read.
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

static mla_geom geom() {
  const int heads = pick({1, 8, 16, 20, 64, 128});
  mla_geom g{heads, 1, 512, 64, 4096, 1, 0.07f, 10000.0, 0};
  switch (rng() % 12) {
    case 0: g.n_heads = any32(); break;
    case 1: g.n_groups = any32(); break;
    case 2: g.d_latent = any32(); break;
    case 3: g.d_rope = pick({16, 0, -64, 128}); break;
    case 4: g.softmax_scale = pick({0.f, -1.f, std::numeric_limits<float>::infinity(), std::numeric_limits<float>::quiet_NaN()}); break;
    case 5: g.rope_base = pick({1.0, 0.5, -3.0, std::numeric_limits<double>::infinity(), std::numeric_limits<double>::quiet_NaN()}); break;
    case 6: g.value_rope = any32(); break;
    default: break;
  }
  return g;
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
    const mla_geom g = geom();
    const mla_geom* gp = rng() % 64 ? &g : nullptr;
    const int32_t page_rows = rng() % 4 ? pick({64, 128, 192, 65536}) : any32();
    const int64_t pages = rng() % 4 ? 1 + (int64_t)(rng() % 1000) : any64();
    const int32_t n_seqs = rng() % 4 ? (int32_t)(rng() % 300) : any32(), n_q = rng() % 4 ? 1 + (int32_t)(rng() % 40) : any32();
    const int32_t most = rng() % 4 ? (int32_t)(rng() % 5000) : any32();
    size_t ws = 0;
    const mla_status q = mla_cache_attend_query(gp, n_seqs, n_q, most, page_rows, rng() % 64 ? &ws : nullptr);
    if (!count(q)) return 1;
    if (q == MLA_OK && (ws == 0 || ws > (size_t(1) << 30))) {
      printf("workspace of %zu bytes\n", ws);
      return 1;
    }
    const size_t given = q == MLA_OK ? ws - 1 : rng() % 1000;
    const mla_status a = mla_cache_attend(gp, n_seqs, n_q, at(16), at<int32_t>(4), at<mla_page>(16), at<int32_t>(4), most, pages, page_rows, at(16),
                                          at(16), at<float>(4), at(256), given, nullptr);
    if (!count(a)) return 1;
    if (a == MLA_OK && n_seqs != 0) {
      printf("a workspace of %zu of %zu bytes was accepted\n", given, ws);
      return 1;
    }
    // no row, or one and no address to read it from
    const int64_t stride = rng() % 3 ? pick<int64_t>({576, 584, 640, 2112}) : any64();
    if (!count(mla_cache_append(gp, 0, at(16), stride, at<int32_t>(4), at<int32_t>(4), pages, page_rows, at(16), nullptr)) ||
        !count(mla_cache_gather(gp, 0, at<int32_t>(4), pages, page_rows, at(16), at(16), stride, nullptr)) ||
        !count(mla_cache_append(gp, (int64_t)(rng() >> 2) + 1, at(16), stride, nullptr, nullptr, pages,
                                page_rows, at(16), nullptr)) ||
        !count(mla_cache_gather(gp, (int64_t)(rng() >> 2) + 1, nullptr, pages, page_rows, at(16), at(16), stride, nullptr)))
      return 1;
    const int32_t cols = rng() % 3 ? 32 * (int32_t)(rng() % 300) : any32();
    const int64_t xs = rng() % 3 ? cols + 8 * (int64_t)(rng() % 3) : any64();
    const int64_t rows = rng() % 3 ? 0 : -1 - (int64_t)(rng() >> 2);
    if (!count(mla_mx4_quantize(rows, cols, at(16), xs, at(16), at(1), nullptr)) ||
        !count(mla_mx4_dequantize(rows, cols, at(16), at(1), at(16), xs, nullptr)) ||
        !count(mla_mx4_quantize((int64_t)(rng() >> 1), cols, at(16), xs, nullptr, at(1), nullptr)))
      return 1;
    const int32_t d_in = rng() % 3 ? 64 * (int32_t)(rng() % 300) : any32(), d_out = any32(), type = rng() % 4 ? (int32_t)(rng() % 2) : any32();
    if (!count(mla_shared_wb_mx4(0, d_in, d_out, at(16), at(16), at(4), type, at(16), nullptr)) ||
        !count(mla_shared_wb_mx4(any64() | 1, d_in, d_out, nullptr, at(16), at(4), type, at(16), nullptr)))
      return 1;
  }
  printf("calls: %lld accepted without a row, refused %lld NULL %lld shape %lld unsupported %lld workspace\n", (long long)met[MLA_OK],
         (long long)met[MLA_ERR_NULL], (long long)met[MLA_ERR_SHAPE], (long long)met[MLA_ERR_UNSUPPORTED], (long long)met[MLA_ERR_WORKSPACE]);
  return met[MLA_OK] && met[MLA_ERR_NULL] && met[MLA_ERR_SHAPE] && met[MLA_ERR_UNSUPPORTED] && met[MLA_ERR_WORKSPACE] ? 0 : 1;
}

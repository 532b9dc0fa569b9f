// Host-only checks of the KV cache's ABI layer (nq_kv_api.cpp), built with a plain host compiler
// under AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_kv_host.py.  The kernels and
// the HIP runtime are replaced by stubs that record every launch, so that no GPU is needed and no
// pointer is read.
//
// Exit status 0 when every check passes; each failure prints its line.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <random>
#include <string>
#include <vector>

#include "nestquant.h"
#include "nq_kernels.hpp"

extern "C" {
hipError_t hipStreamGetDevice(hipStream_t, hipDevice_t* dev) {
  *dev = 0;
  return hipSuccess;
}
hipError_t hipGetDevice(int* dev) {
  *dev = 0;
  return hipSuccess;
}
hipError_t hipSetDevice(int) { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "stub HIP error"; }
}

static std::vector<std::string> g_calls;
static std::string g_error;
static nq::AttendArgs g_attend;

namespace nq {
static hipError_t rec(const char* name) {
  g_calls.push_back(name);
  return hipSuccess;
}
nq_status set_error(nq_status s, const char* fmt, ...) {
  char text[512];
  va_list args;
  va_start(args, fmt);
  std::vsnprintf(text, sizeof text, fmt, args);
  va_end(args);
  g_error = text;
  return s;
}
nq_status check_code(const nq_params*, int64_t, const char*) { return NQ_OK; }
EncodeArgs code_args(const nq_params* p) {
  EncodeArgs e{};
  e.q = p->q;
  e.k = p->k;
  e.mtab = 0x04030201u;
  return e;
}
hipError_t launch_kv_append(const KVAppendArgs&, int, int, hipStream_t) { return rec("append"); }
hipError_t launch_attend(const AttendArgs& a, const AttendPlan&, int, int, hipStream_t) {
  g_attend = a;
  return rec("few");
}
hipError_t launch_prompt(const AttendArgs& a, int, int, hipStream_t) {
  g_attend = a;
  return rec("many");
}
hipError_t attend_set_attributes() { return hipSuccess; }
hipError_t prompt_set_attributes() { return hipSuccess; }
}  // namespace nq

static int g_fail = 0;
#define CHECK(cond)                                                   \
  do {                                                                \
    if (!(cond)) {                                                    \
      std::fprintf(stderr, "FAIL line %d: %s\n", __LINE__, #cond);    \
      ++g_fail;                                                       \
    }                                                                 \
  } while (0)

static void* const DEV = reinterpret_cast<void*>(0x10000);     // never dereferenced

static nq_kv_cache cache(int heads = 8, int dim = 128) {
  nq_kv_cache c{};
  c.k.q = c.v.q = 14;
  c.k.k = c.v.k = 4;
  c.k.base = c.v.base = 10.0 / 56;
  c.k_codes = c.k_beta = c.v_codes = c.v_beta = static_cast<uint32_t*>(DEV);
  c.k_scales = c.v_scales = static_cast<float*>(DEV);
  c.pages = 1 << 20;
  c.heads = heads;
  c.dim = dim;
  c.page = 64;
  return c;
}

// The size query of a call's arguments.
static int64_t size(int heads, int dim, int q_heads, int64_t seqs, int64_t tokens, int64_t queries, int64_t length,
                    int64_t window = 0, int64_t sinks = 0) {
  return nq_attend_workspace_size(heads, dim, tokens, q_heads, seqs, queries, length, window, sinks);
}

struct Attend {
  int heads = 8, dim = 128, q_heads = 32;
  int64_t seqs = 1, tokens = 1, queries = 1, length = 100;
  bool starts = true;
  double scale = 0.1;
  nq_status operator()() const {
    g_calls.clear();
    const nq_kv_cache c = cache(heads, dim);
    const nq_heads x = {DEV, (int64_t)q_heads * dim, dim};
    return nq_attend(&c, static_cast<int32_t*>(DEV), 1 << 20, static_cast<int32_t*>(DEV), seqs,
                     starts ? static_cast<int32_t*>(DEV) : nullptr, queries, length, 0, 0, scale, NQ_BF16, &x,
                     tokens, q_heads, &x, nullptr, DEV, (int64_t)1 << 60, nullptr);
  }
};

static nq_status append(int64_t tokens, int heads, int dim, int q_heads) {
  g_calls.clear();
  const nq_kv_cache c = cache(heads, dim);
  const nq_kv_prep prep{};
  const nq_heads x = {DEV, 0, 0};
  return nq_kv_append(&c, &prep, tokens, static_cast<int64_t*>(DEV), nullptr, NQ_BF16, &x, q_heads, &x, &x, &x,
                      NQ_BF16, nullptr);
}

// A launch takes fewer than 2^32 threads.
static void launches() {
  Attend a;
  CHECK(a() == NQ_OK && g_calls.size() == 1 && g_calls[0] == "few");
  // 128 rows of a KV head a workgroup of 256 threads: 2^24 of them and one fewer
  a = {.seqs = 2048, .tokens = 32768, .queries = 32768, .length = 64};
  CHECK(a() == NQ_ERR_UNSUPPORTED && g_calls.empty());
  CHECK(g_error.find("nq_attend: more workgroups") == 0);
  a.seqs = 2047;
  CHECK(a() == NQ_OK && g_calls.size() == 1 && g_calls[0] == "many");
  CHECK((int64_t)g_attend.chunks * g_attend.blocks * g_attend.heads * g_attend.seqs * 256 < (int64_t)1 << 32);
  // records of 64 tokens
  a = {.seqs = 2048, .tokens = 4096, .queries = 17, .length = 1024 * 64};
  CHECK(a() == NQ_ERR_UNSUPPORTED && g_calls.empty());
  a.length -= 64;
  CHECK(a() == NQ_OK);
  // chunks of the cache of single tokens: 16 steps of 32 tokens each
  a = {.seqs = 16384, .tokens = 16384, .queries = 1, .length = 128 * 512};
  CHECK(a() == NQ_ERR_UNSUPPORTED && g_calls.empty());
  a.length -= 512;
  CHECK(a() == NQ_OK);
  CHECK((int64_t)g_attend.chunks * g_attend.blocks * g_attend.heads * g_attend.seqs * 256 < (int64_t)1 << 32);

  // 256 blocks a workgroup of 64 threads
  CHECK(append(5, 8, 128, 32) == NQ_OK && g_calls.size() == 1);
  CHECK(append((int64_t)1 << 28, 1, 256, 0) == NQ_ERR_UNSUPPORTED && g_calls.empty());
  CHECK(g_error.find("nq_kv_append: more workgroups") == 0);
  CHECK(append(((int64_t)1 << 28) - 8, 1, 256, 0) == NQ_OK);
  CHECK(append(((int64_t)1 << 28) - 8, 1, 256, 7) == NQ_OK);      // the queries in a launch of their own
}

// The size query refuses what the call refuses, however large.
static void sizes() {
  CHECK(size(8, 128, 32, 2048, 32768, 32768, 64) == -1);
  CHECK(size(8, 128, 32, 2047, 32768, 32768, 64) > 0);
  CHECK(size(8, 128, 32, 16384, 16384, 1, 128 * 512) == -1);
  CHECK(size(1024, 256, 1024, 65535, 65535, 65, (1 << 30) - 1) == -1);
  CHECK(size(1024, 256, 16384, 65535, 65535, 4, (1 << 30) - 1) == -1);
  CHECK(size(1, 256, 1, 65535, 65535, 65535, (1 << 30) - 1) == -1);
}

// A workspace of the bound serves every smaller call, and the bound stays near the size.
static void bounds() {
  std::mt19937_64 rng(1);
  auto up_to = [&](int64_t most) {   // spread over the logarithm, 0 and the largest now and then
    if (rng() % 8 == 0) return rng() % 2 ? most : (int64_t)0;
    const double x = std::exp(std::log((double)most + 1) * ((double)(rng() >> 11) * 0x1p-53));
    return std::min((int64_t)x, most);
  };
  int compared = 0;
  for (int i = 0; i < 400000; ++i) {
    const int dims[] = {64, 128, 256}, groups[] = {1, 2, 3, 4, 5, 8, 12, 16, 17, 40};
    const int dim = dims[rng() % 3], heads = 1 + (int)up_to(15), q_heads = heads * groups[rng() % 10];
    const int64_t tokens = up_to(40000), seqs = up_to(300), queries = up_to(tokens), length = up_to(300000);
    const int64_t window = rng() % 2 ? 0 : up_to(5000), sinks = up_to(300);
    const int64_t bound = nq_attend_workspace_bound(heads, dim, tokens, q_heads, seqs, queries, length, window, sinks);
    const int64_t own = size(heads, dim, q_heads, seqs, tokens, queries, length, window, sinks);
    CHECK((bound < 0) == (own < 0));
    CHECK(bound >= own);
    if (bound < 0) continue;
    // beside the records: 1022 workgroups of 128 rows, or 2048 and four a pair and 512 tokens of 32
    CHECK(bound <= own + (1022 * 128 + 2048 * 32 + seqs * heads * 4 * (2 + length / 512) * 32) * 4 * (dim + 4));
    for (int j = 0; j < 8; ++j) {
      const int64_t t = up_to(tokens), w = window ? std::max<int64_t>(up_to(window), 1) : up_to(5000);
      const int64_t s = up_to(seqs), q = up_to(std::min(t, queries)), l = up_to(length), k = up_to(sinks);
      const int64_t smaller = size(heads, dim, q_heads, s, t, q, l, w, k);
      if (smaller < 0) continue;
      if (smaller > bound) {
        std::fprintf(stderr, "%d heads of %d, %d query heads: %lld of %lld for tokens %lld/%lld seqs %lld/%lld "
                     "queries %lld/%lld length %lld/%lld window %lld/%lld sinks %lld/%lld\n", heads, dim, q_heads,
                     (long long)smaller, (long long)bound, (long long)t, (long long)tokens, (long long)s,
                     (long long)seqs, (long long)q, (long long)queries, (long long)l, (long long)length,
                     (long long)w, (long long)window, (long long)k, (long long)sinks);
        ++g_fail;
        return;
      }
      ++compared;
      const int64_t b = nq_attend_workspace_bound(heads, dim, t, q_heads, s, q, l, w, k);
      CHECK(b <= bound);
    }
  }
  CHECK(compared > 1000000);
}

// No tokens and no sequences: nothing to do, whatever the bounds.
static void nothing() {
  Attend a;
  a = {.seqs = 0, .tokens = 0, .queries = 1, .starts = false};
  CHECK(a() == NQ_OK && g_calls.empty());
  a = {.seqs = 3, .tokens = 0, .queries = 4};
  CHECK(a() == NQ_OK && g_calls.empty());
  CHECK(nq_attend_workspace_size(8, 128, 0, 32, 0, 1, 100, 0, 0) == 0);
  CHECK(nq_attend_workspace_size(8, 128, 0, 32, 3, 4, 100, 0, 0) == 0);
  a = {.seqs = 3, .tokens = 3, .queries = 4};
  CHECK(a() == NQ_ERR_INVALID_ARG && g_calls.empty());
  a = {.seqs = 0, .tokens = 0, .queries = -1};
  CHECK(a() == NQ_ERR_INVALID_ARG && g_calls.empty());
}

// The scale reaches the kernels in fp32.
static void scales() {
  Attend a;
  a = {.scale = 1e38};
  CHECK(a() == NQ_OK && std::isfinite(g_attend.k_scale));
  a = {.scale = -1e40};
  CHECK(a() == NQ_ERR_INVALID_ARG && g_calls.empty());
  CHECK(g_error.find("nq_attend: scale") == 0);
}

int main() {
  launches();
  scales();
  sizes();
  bounds();
  nothing();
  if (g_fail) return 1;
  std::puts("all host KV cache checks passed");
  return 0;
}

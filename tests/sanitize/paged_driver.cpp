// Drives the paged caches' host code on a machine without a GPU, built with the
// host sanitizers: a stand-in HIP runtime (host memory, no device work) lets
// plans exist, and launch stand-ins keep the parameters they are given. Checks
// every refusal of the C ABI, and over random dimensions that the work split
// covers all keys, fits the launchers' variants and stays inside the workspace.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>

#include "bifattn.h"
#include "bifattn_paged.h"

using namespace bifattn;

static size_t g_alloc = 0;          // bytes of the last allocation
static char* g_base = nullptr;
static int g_stream_device = 0;     // device that every stream belongs to
static PagedAttnParams g_stream, g_wide;
static PagedCombineParams g_combine;
static PagedAppendParams g_append;
static PagedGatherParams g_gather;
static int g_launches, g_ctx_tiles, g_dec_tiles, g_wide_tiles;

extern "C" {
hipError_t hipGetDeviceCount(int* n) { return *n = 1, hipSuccess; }
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipStreamGetDevice(hipStream_t, hipDevice_t* d) { return *d = g_stream_device, hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
hipError_t hipStreamCreateWithFlags(hipStream_t* s, unsigned) { return *s = (hipStream_t)16, hipSuccess; }
hipError_t hipStreamDestroy(hipStream_t) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipMallocAsync(void** p, size_t n, hipStream_t) {
  g_alloc = n;
  if (n > (size_t(1) << 33)) return hipErrorOutOfMemory;
  *p = g_base = (char*)aligned_alloc(256, (n + 255) & ~size_t(255));
  return *p ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipMalloc(void**, size_t) { return hipErrorOutOfMemory; }
hipError_t hipFreeAsync(void* p, hipStream_t) { return free(p), hipSuccess; }
hipError_t hipFree(void* p) { return free(p), hipSuccess; }
hipError_t hipMemsetAsync(void* p, int v, size_t n, hipStream_t) { return memset(p, v, n), hipSuccess; }
hipError_t hipMemset(void* p, int v, size_t n) { return memset(p, v, n), hipSuccess; }
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind) { return memcpy(d, s, n), hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return *e = (hipEvent_t)16, hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
}
namespace bifattn {
hipError_t launch_paged_stream(const PagedAttnParams& P, int, int, int tc, int td, hipStream_t) {
  return g_stream = P, g_ctx_tiles = tc, g_dec_tiles = td, g_launches |= 1, hipSuccess;
}
hipError_t launch_paged_wide(const PagedAttnParams& P, int, int, int td, hipStream_t) {
  return g_wide = P, g_wide_tiles = td, g_launches |= 2, hipSuccess;
}
hipError_t launch_paged_combine(const PagedCombineParams& C, int, hipStream_t, hipEvent_t) {
  return g_combine = C, g_launches |= 4, hipSuccess;
}
hipError_t launch_paged_whole(const PagedWholeParams& W, int, int, int tiles, hipStream_t, hipEvent_t) {
  return g_stream = W.A, g_combine = W.C, g_dec_tiles = tiles, g_launches |= 32, hipSuccess;
}
hipError_t launch_paged_append(const PagedAppendParams& A, int, hipStream_t, hipEvent_t) {
  return g_append = A, g_launches |= 8, hipSuccess;
}
hipError_t launch_paged_gather(const PagedGatherParams& G, int, hipStream_t, hipEvent_t) {
  return g_gather = G, g_launches |= 16, hipSuccess;
}
}  // namespace bifattn

#define CHECK(x)                                                              \
  do {                                                                        \
    if (!(x)) {                                                               \
      std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #x);              \
      std::exit(1);                                                           \
    }                                                                         \
  } while (0)

static bifattn_paged_dims_t dims() {
  bifattn_paged_dims_t d{};
  d.b = 3, d.h = 8, d.g = 2, d.d = 128, d.m_c = 100, d.m_d_max = 40, d.page = 16, d.num_pages = 50, d.n = 1;
  return d;
}
static bifattn_status_t create(const bifattn_paged_dims_t& d) {
  bifattn_paged_plan_t p = (bifattn_paged_plan_t)16;
  const bifattn_status_t st = bifattn_paged_plan_create(&d, &p);
  CHECK((st == BIFATTN_OK) == (p != nullptr));
  if (p) CHECK(bifattn_paged_plan_destroy(p) == BIFATTN_OK);
  return st;
}

static void refused_dims() {
  CHECK(bifattn_paged_plan_create(nullptr, nullptr) == BIFATTN_EINVAL);
  bifattn_paged_plan_t p = (bifattn_paged_plan_t)16;
  CHECK(bifattn_paged_plan_create(nullptr, &p) == BIFATTN_EINVAL && !p);
  CHECK(bifattn_paged_plan_destroy(nullptr) == BIFATTN_OK);
  CHECK(create(dims()) == BIFATTN_OK);
#define BAD(field, value, want)    \
  {                                \
    bifattn_paged_dims_t d = dims(); \
    d.field = value;               \
    CHECK(create(d) == want);      \
  }
  BAD(b, 0, BIFATTN_EINVAL) BAD(h, 0, BIFATTN_EINVAL) BAD(g, 0, BIFATTN_EINVAL) BAD(g, 3, BIFATTN_EINVAL)
  BAD(d, 96, BIFATTN_EUNSUPPORTED) BAD(d, 256, BIFATTN_EUNSUPPORTED) BAD(m_c, -1, BIFATTN_EINVAL)
  BAD(m_d_max, -1, BIFATTN_EINVAL) BAD(page, 0, BIFATTN_EINVAL) BAD(page, 8, BIFATTN_EUNSUPPORTED)
  BAD(page, 24, BIFATTN_EUNSUPPORTED) BAD(page, 512, BIFATTN_EUNSUPPORTED) BAD(num_pages, 0, BIFATTN_EINVAL)
  BAD(scale, INFINITY, BIFATTN_EINVAL) BAD(scale, NAN, BIFATTN_EINVAL) BAD(n, -1, BIFATTN_EINVAL)
  BAD(n, 17, BIFATTN_EUNSUPPORTED) BAD(maps, 3, BIFATTN_EINVAL) BAD(maps, -1, BIFATTN_EINVAL)
  BAD(kv_type, BIFATTN_KV_INT8, BIFATTN_EUNSUPPORTED) BAD(kv_type, BIFATTN_KV_INT4, BIFATTN_EUNSUPPORTED)
  BAD(kv_type, 5, BIFATTN_EINVAL) BAD(kv_type, -1, BIFATTN_EINVAL) BAD(m_c, (1 << 30) + 1, BIFATTN_EUNSUPPORTED)
  BAD(b, 1 << 30, BIFATTN_EINVAL)
  {
    bifattn_paged_dims_t d = dims();
    d.m_c = d.m_d_max = 0;
    CHECK(create(d) == BIFATTN_EINVAL);
    d = dims();
    d.maps = 2, d.n = 9;  // 2 * 4 * 9 query rows
    CHECK(create(d) == BIFATTN_EUNSUPPORTED);
    d.n = 8;
    CHECK(create(d) == BIFATTN_OK);
    d = dims();
    d.num_pages = INT32_MAX, d.h = d.g = 1 << 28, d.b = 1;
    CHECK(create(d) == BIFATTN_EINVAL);
  }
}

static void refused_calls() {
  alignas(16) static char mem[256];
  void* a = mem;
  void* odd = mem + 8;  // not 16-byte aligned
  int32_t* i = (int32_t*)mem;
  int32_t* iodd = (int32_t*)(mem + 2);
  float* f = (float*)mem;
  float* fodd = (float*)(mem + 2);
  for (int maps = 1; maps <= 2; ++maps)
    for (int kv : {0, 1, 4}) {
      bifattn_paged_dims_t d = dims();
      d.maps = maps, d.kv_type = kv;
      bifattn_paged_plan_t P;
      CHECK(bifattn_paged_plan_create(&d, &P) == BIFATTN_OK);
      bifattn_pages_t pg{};
      pg.K = a, pg.V = a;
      if (kv == 4) pg.K_exp = pg.V_exp = (uint8_t*)a;
      auto run = [&](const void* q, const bifattn_pages_t* p, const int32_t* c, const int32_t* t, const int32_t* l,
                     void* out) {
        g_launches = 0;
        const bifattn_status_t st =
            maps == 1 ? bifattn_paged_decode(P, q, p, c, t, l, out, nullptr)
                      : bifattn_paged_decode_diff(P, q, p, c, t, l, f, nullptr, 0.f, 1.f, out, nullptr);
        CHECK((st == BIFATTN_OK) == (g_launches != 0));
        return st;
      };
      CHECK(run(a, &pg, i, i, i, a) == BIFATTN_OK);
      CHECK(run(nullptr, &pg, i, i, i, a) == BIFATTN_EINVAL);
      CHECK(run(a, nullptr, i, i, i, a) == BIFATTN_EINVAL);
      CHECK(run(a, &pg, nullptr, i, i, a) == BIFATTN_EINVAL);
      CHECK(run(a, &pg, i, nullptr, i, a) == BIFATTN_EINVAL);
      CHECK(run(a, &pg, i, i, nullptr, a) == BIFATTN_EINVAL);
      CHECK(run(a, &pg, i, i, i, nullptr) == BIFATTN_EINVAL);
      CHECK(run(odd, &pg, i, i, i, a) == BIFATTN_EALIGN);
      CHECK(run(a, &pg, iodd, i, i, a) == BIFATTN_EALIGN);
      CHECK(run(a, &pg, i, iodd, i, a) == BIFATTN_EALIGN);
      CHECK(run(a, &pg, i, i, iodd, a) == BIFATTN_EALIGN);
      CHECK(run(a, &pg, i, i, i, odd) == BIFATTN_EALIGN);
      auto pool = [&](auto change) {
        bifattn_pages_t x = pg;
        change(x);
        return run(a, &x, i, i, i, a);
      };
      CHECK(pool([&](bifattn_pages_t& x) { x.K = nullptr; }) == BIFATTN_EINVAL);
      CHECK(pool([&](bifattn_pages_t& x) { x.V = odd; }) == BIFATTN_EALIGN);
      CHECK(pool([&](bifattn_pages_t& x) { x.K_exp = kv == 4 ? nullptr : (uint8_t*)a; }) == BIFATTN_EINVAL);
      CHECK(pool([&](bifattn_pages_t& x) { x.k_scale = f; }) == (kv == 1 ? BIFATTN_OK : BIFATTN_EINVAL));
      if (kv == 1) CHECK(pool([&](bifattn_pages_t& x) { x.v_scale = fodd; }) == BIFATTN_EALIGN);
      g_stream_device = 1;
      CHECK(bifattn_paged_plan_status(P, nullptr) == BIFATTN_OK);
      CHECK((maps == 1 ? bifattn_paged_decode(P, a, &pg, i, i, i, a, (hipStream_t)32)
                       : bifattn_paged_decode_diff(P, a, &pg, i, i, i, f, nullptr, 0.f, 1.f, a, (hipStream_t)32)) ==
            BIFATTN_EINVAL);
      g_stream_device = 0;
      // the other kind's entry point
      CHECK((maps == 2 ? bifattn_paged_decode(P, a, &pg, i, i, i, a, nullptr)
                       : bifattn_paged_decode_diff(P, a, &pg, i, i, i, f, nullptr, 0.f, 1.f, a, nullptr)) ==
            BIFATTN_EINVAL);
      if (maps == 2) {
        auto diff = [&](const float* lam, const float* w, float eps, float s) {
          return bifattn_paged_decode_diff(P, a, &pg, i, i, i, lam, w, eps, s, a, nullptr);
        };
        CHECK(diff(nullptr, nullptr, 0.f, 1.f) == BIFATTN_EINVAL);
        CHECK(diff(f, f, -1.f, 1.f) == BIFATTN_EINVAL);
        CHECK(diff(f, f, NAN, 1.f) == BIFATTN_EINVAL);
        CHECK(diff(f, f, 0.f, INFINITY) == BIFATTN_EINVAL);
        CHECK(diff(fodd, f, 0.f, 1.f) == BIFATTN_EALIGN);
        CHECK(diff(f, (float*)odd, 0.f, 1.f) == BIFATTN_EALIGN);
        CHECK(diff(f, f, 0.f, 1.f) == BIFATTN_OK);
      }
      bifattn_new_rows_t r{};
      r.samples = 3, r.n = 5, r.k = a, r.v = a, r.q = a, r.q_out = a, r.rot = 32, r.freqs = f;
      auto app = [&](auto change) {
        bifattn_new_rows_t x = r;
        change(x);
        g_launches = 0;
        const bifattn_status_t st = bifattn_paged_append(P, &pg, i, &x, i, i, nullptr);
        CHECK((st == BIFATTN_OK) == (g_launches == 8));
        return st;
      };
      typedef bifattn_new_rows_t R;
      CHECK(app([](R&) {}) == BIFATTN_OK);
      CHECK(g_append.position0 == d.m_c && g_append.max_rows == 40 && g_append.table_pages == 3);
      CHECK(app([](R& x) { x.context = 1, x.samples = 1; }) == BIFATTN_OK);
      CHECK(g_append.position0 == 0 && g_append.max_rows == 100 && g_append.table_pages == 7);
      CHECK(app([](R& x) { x.context = 1; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.samples = 4; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.samples = 0; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.n = (1 << 29) + 1; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.n = 0; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.k = nullptr; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.v = nullptr; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.q = nullptr; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.q_out = nullptr; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.q = x.q_out = nullptr; }) == BIFATTN_OK && g_append.h == 0);
      CHECK(app([](R& x) { x.freqs = nullptr; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.freqs = nullptr, x.rot = 0; }) == BIFATTN_OK);
      CHECK(app([](R& x) { x.rot = 24; }) == BIFATTN_EUNSUPPORTED);
      CHECK(app([](R& x) { x.rot = -16; }) == BIFATTN_EINVAL);
      CHECK(app([](R& x) { x.rot = 128; }) == (maps == 1 ? BIFATTN_OK : BIFATTN_EINVAL));
      CHECK(app([](R& x) { x.rot = 144; }) == BIFATTN_EINVAL);
      CHECK(app([&](R& x) { x.k = odd; }) == BIFATTN_EALIGN);
      CHECK(app([&](R& x) { x.q_out = odd; }) == BIFATTN_EALIGN);
      CHECK(app([&](R& x) { x.counts = iodd; }) == BIFATTN_EALIGN);
      CHECK(app([](R& x) { x.v_stride[1] = 4; }) == BIFATTN_EALIGN);
      CHECK(app([](R& x) { x.q_stride[2] = 129; }) == BIFATTN_EALIGN);
      CHECK(bifattn_paged_append(nullptr, &pg, i, &r, i, i, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, nullptr, i, &r, i, i, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, &pg, nullptr, &r, i, i, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, &pg, i, nullptr, i, i, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, &pg, i, &r, nullptr, i, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, &pg, i, &r, i, nullptr, nullptr) == BIFATTN_EINVAL);
      CHECK(bifattn_paged_append(P, &pg, i, &r, i, iodd, nullptr) == BIFATTN_EALIGN);
      auto gat = [&](const int32_t* t, const int32_t* l, int s, int n, int c, void* k) {
        return bifattn_paged_gather(P, &pg, t, nullptr, l, s, n, c, k, a, nullptr);
      };
      CHECK(gat(i, i, 3, 7, 0, a) == BIFATTN_OK && g_gather.max_rows == 40);
      CHECK(gat(i, i, 1, 7, 1, a) == BIFATTN_OK && g_gather.max_rows == 100);
      CHECK(gat(i, i, 2, 7, 1, a) == BIFATTN_EINVAL);
      CHECK(gat(i, i, 4, 7, 0, a) == BIFATTN_EINVAL);
      CHECK(gat(i, i, 3, 0, 0, a) == BIFATTN_EINVAL);
      CHECK(gat(nullptr, i, 3, 7, 0, a) == BIFATTN_EINVAL);
      CHECK(gat(i, nullptr, 3, 7, 0, a) == BIFATTN_EINVAL);
      CHECK(gat(i, i, 3, 7, 0, nullptr) == BIFATTN_EINVAL);
      CHECK(gat(i, i, 3, 7, 0, odd) == BIFATTN_EALIGN);
      CHECK(bifattn_paged_plan_destroy(P) == BIFATTN_OK);
    }
  bifattn_plan_info_t info;
  CHECK(bifattn_paged_plan_get_info(nullptr, &info) == BIFATTN_EINVAL);
  CHECK(bifattn_paged_plan_status(nullptr, nullptr) == BIFATTN_EINVAL);
  CHECK(bifattn_paged_decode(nullptr, a, nullptr, i, i, i, a, nullptr) == BIFATTN_EINVAL);
  CHECK(bifattn_paged_decode_diff(nullptr, a, nullptr, i, i, i, f, f, 0.f, 1.f, a, nullptr) == BIFATTN_EINVAL);
  CHECK(bifattn_paged_gather(nullptr, nullptr, i, i, i, 1, 1, 0, a, a, nullptr) == BIFATTN_EINVAL);
  // a sequence kind that the plan does not have
  for (int own = 0; own < 2; ++own) {
    bifattn_paged_dims_t d = dims();
    (own ? d.m_c : d.m_d_max) = 0;
    bifattn_paged_plan_t P;
    CHECK(bifattn_paged_plan_create(&d, &P) == BIFATTN_OK);
    bifattn_pages_t pg{};
    pg.K = pg.V = a;
    bifattn_new_rows_t r{};
    r.samples = 1, r.n = 1, r.k = r.v = a, r.context = own;
    CHECK(bifattn_paged_append(P, &pg, i, &r, i, i, nullptr) == BIFATTN_EINVAL);
    CHECK(bifattn_paged_gather(P, &pg, i, nullptr, i, 1, 1, own, a, a, nullptr) == BIFATTN_EINVAL);
    CHECK(bifattn_paged_decode(P, a, &pg, own ? nullptr : i, own ? i : nullptr, own ? i : nullptr, a, nullptr) ==
          BIFATTN_OK);
    CHECK(bifattn_paged_plan_destroy(P) == BIFATTN_OK);
  }
}

// Over random dimensions: what the kernels assume of their parameters.
static void splits() {
  std::mt19937 rng(5);
  auto pick = [&](int lo, int hi) { return (int)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng))); };
  alignas(16) static char mem[64];
  int32_t* i = (int32_t*)mem;
  int seen = 0, whole = 0;
  while (seen < 4000) {
    bifattn_paged_dims_t d{};
    d.g = pick(1, 40), d.h = d.g * pick(1, 32), d.b = pick(1, 600), d.n = pick(1, 8), d.d = rng() % 2 ? 64 : 128;
    d.m_c = rng() % 8 ? pick(1, 60000) : 0, d.m_d_max = rng() % 8 ? pick(1, 5000) : 0;
    d.page = 16 << rng() % 5, d.num_pages = 10, d.maps = 1 + rng() % 2;
    if (d.maps * d.h / d.g * d.n > 64 || d.m_c + d.m_d_max == 0) continue;
    bifattn_paged_plan_t P;
    const bifattn_status_t st = bifattn_paged_plan_create(&d, &P);
    if (st == BIFATTN_ENOMEM) continue;
    CHECK(st == BIFATTN_OK);
    ++seen;
    bifattn_pages_t pg{};
    pg.K = pg.V = mem;
    g_launches = 0;
    CHECK((d.maps == 1 ? bifattn_paged_decode(P, mem, &pg, i, i, i, mem, nullptr)
                       : bifattn_paged_decode_diff(P, mem, &pg, i, i, i, (float*)mem, nullptr, 0.f, 1.f, mem, nullptr)) == BIFATTN_OK);
    const int R = d.maps * d.h / d.g * d.n, M = d.b * R;
    const int64_t units = (int64_t)d.b * d.g;
    const PagedCombineParams& C = g_combine;
    bifattn_plan_info_t info;
    CHECK(bifattn_paged_plan_get_info(P, &info) == BIFATTN_OK);
    CHECK((info.path == BIFATTN_PATH_STANDARD) == (g_launches == 32));
    if (g_launches == 32) {  // small steps: the unit fits two query tiles
      CHECK(g_dec_tiles <= 2 && g_dec_tiles * 16 >= R && units <= 1536 && d.m_c + d.m_d_max <= 4000);
      CHECK(g_stream.R == R && C.R == R && C.pn * d.maps == R && C.hn == d.h * d.n);
      ++whole;
      CHECK(bifattn_paged_plan_destroy(P) == BIFATTN_OK);
      continue;
    }
    const PagedAttnParams& K = g_launches & 2 ? g_wide : g_stream;
    CHECK(g_launches & 4);
    CHECK(K.R == R && K.M == M && K.M == K.maps * K.Mh && K.R == K.maps * K.pn && C.M == M && C.R == R);
    CHECK((1 << K.pool.shift) == d.page && K.table_pages == (d.m_d_max + d.page - 1) / d.page);
    // own rows: whole tiles per chunk, chunks cover the capacity, tiles hold the unit
    int dec = g_launches & 1 ? g_stream.n_dec_blocks : 0;
    if (g_launches & 2) dec += g_wide.n_dec_blocks;
    CHECK(dec == units * K.S_d && C.S_d == 4 * K.S_d);
    if (d.m_d_max) CHECK(K.dec_keys % 128 == 0 && (int64_t)K.S_d * K.dec_keys >= d.m_d_max && (int64_t)(K.S_d - 1) * K.dec_keys < d.m_d_max);
    if (g_launches & 1) CHECK(g_dec_tiles * 16 >= R && (g_dec_tiles == 1 || g_dec_tiles == 2 || g_dec_tiles == 4));
    // context: one of the launchers' variants, splits cover it
    CHECK(C.S_c == K.S_c);
    if (!d.m_c) {
      CHECK(K.S_c == 0 && g_launches == 5 && g_ctx_tiles == 0);
    } else if (g_launches & 2) {
      CHECK(K.ctx_wide == 4 || K.ctx_wide == 8);
      CHECK(K.ctx_keys % (16 * K.ctx_wide) == 0 && (int64_t)K.S_c * K.ctx_keys >= d.m_c && (int64_t)(K.S_c - 1) * K.ctx_keys < d.m_c);
      CHECK(K.ctx_row_blocks % K.maps == 0 && (int64_t)K.ctx_row_blocks / K.maps * 32 * K.ctx_wide >= K.Mh);
      CHECK(g_wide.n_ctx_blocks == (int64_t)d.g * K.S_c * K.ctx_row_blocks);
      if (g_wide.n_dec_blocks) CHECK(g_wide_tiles <= 2 && g_wide_tiles * 16 >= R);
      if (g_launches & 1) CHECK(g_ctx_tiles == 0 && g_stream.n_ctx_small_blocks == 0 && g_wide.n_dec_blocks == 0);
    } else {
      CHECK(g_ctx_tiles * 16 >= M && g_stream.n_ctx_small_blocks == d.g * K.S_c && K.S_c >= 1);
      const int tc = g_ctx_tiles, td = g_dec_tiles;
      CHECK((td == 4 && tc == 4) || (td == 2 && tc == 2) || (td == 1 && (tc == 1 || tc == 2)));
    }
    // the partials lie inside the workspace, one behind the other
    const size_t ctx = (size_t)d.g * K.S_c * M, own = (size_t)dec * 4 * R;
    CHECK((char*)K.ctx_acc == g_base && (char*)K.ctx_ml >= g_base + ctx * d.d * 4);
    CHECK((char*)K.dec_acc >= (char*)K.ctx_ml + ctx * 8 && (char*)K.dec_ml >= (char*)K.dec_acc + own * d.d * 4);
    CHECK((char*)K.status >= (char*)K.dec_ml + own * 8 + 4 * (size_t)d.b && (char*)K.status + 4 <= g_base + g_alloc);
    // appends of any size: every token and head in one work-group's share
    bifattn_new_rows_t r{};
    r.samples = 1 + rng() % d.b, r.n = pick(1, 20000), r.context = d.m_d_max == 0, r.k = r.v = mem;
    if (r.context) r.samples = 1;
    if (rng() % 2) r.q = r.q_out = mem;
    CHECK(bifattn_paged_append(P, &pg, i, &r, i, i, nullptr) == BIFATTN_OK);
    const PagedAppendParams& A = g_append;
    const int heads = (r.q ? d.h : 0) + 2 * d.g;
    CHECK((int64_t)A.token_blocks * A.tokens_per_block >= r.n && (int64_t)(A.token_blocks - 1) * A.tokens_per_block < r.n);
    CHECK((int64_t)A.head_blocks * A.heads_per_block >= heads && (int64_t)(A.head_blocks - 1) * A.heads_per_block < heads);
    CHECK(A.tickets + d.b == K.status && A.tokens_per_block <= 8);
    CHECK(bifattn_paged_plan_destroy(P) == BIFATTN_OK);
  }
  CHECK(whole > 100 && whole < 3000);
}

int main() {
  refused_dims();
  refused_calls();
  splits();
  std::printf("all checks passed\n");
  return 0;
}

// Host side of the paged caches: argument validation, work splitting, the
// plan's workspace, launches and the C ABI declared in include/bifattn.h.
#include "bifattn.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdlib>
#include <new>

#include "bifattn_paged.h"

using namespace bifattn;

struct bifattn_paged_plan_s {
  bifattn_paged_dims_t dims{};
  float scale = 0.f;
  int ntok = 1, maps = 1, shift = 4;
  int pn = 0, R = 0, Mh = 0, M = 0;
  int dec_tiles = 1, ctx_tiles = 0;  // ctx_tiles 0: no context, or the many-row kernel
  int ctx_wide = 0;                  // many-row kernel: waves of a work-group, else 0
  int ctx_keys = 0, S_c = 0, ctx_row_blocks = 1, n_ctx_blocks = 0, n_ctx_small_blocks = 0;
  int dec_keys = 0, S_d = 0, n_dec_blocks = 0;
  int whole = 0;                     // one launch, without partials (small steps)
  // The plan's own stream orders the workspace's allocation and freeing;
  // done_ev marks the end of its last call.
  hipStream_t own = nullptr;
  hipEvent_t done_ev = nullptr;
  bool ws_async = false;
  int device = 0;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  float* ctx_acc = nullptr;
  float2* ctx_ml = nullptr;
  float* dec_acc = nullptr;
  float2* dec_ml = nullptr;
  int* tickets = nullptr;
  int* status = nullptr;
};

namespace {

constexpr unsigned kOrderEventFlags = hipEventDisableTiming | hipEventDisableSystemFence;
constexpr int kCUs = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
bool aligned(const void* ptr, uintptr_t a) { return ((uintptr_t)ptr & (a - 1)) == 0; }

// Tuning overrides from the environment: a positive integer, else `fallback`.
int env_int(const char* name, int fallback) {
  const char* v = std::getenv(name);
  if (!v || !*v) return fallback;
  char* end = nullptr;
  const long x = std::strtol(v, &end, 10);
  return (end && *end == 0 && x > 0 && x < (1 << 30)) ? (int)x : fallback;
}

bool on_plan_device(const bifattn_paged_plan_s* P, hipStream_t stream) {
  int dev = -1;
  if (stream) {
    hipDevice_t d = -1;
    if (hipStreamGetDevice(stream, &d) != hipSuccess) {
      (void)hipGetLastError();
      return false;
    }
    dev = d;
  } else if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return dev == P->device;
}

bifattn_status_t check_dims(const bifattn_paged_dims_t* d) {
  if (!d) return BIFATTN_EINVAL;
  if (d->b < 1 || d->h < 1 || d->g < 1 || d->m_c < 0 || d->m_d_max < 0 || d->n < 0 || d->num_pages < 1)
    return BIFATTN_EINVAL;
  if (d->h % d->g || (d->m_c == 0 && d->m_d_max == 0) || !std::isfinite(d->scale)) return BIFATTN_EINVAL;
  if (d->maps < 0 || d->maps > 2) return BIFATTN_EINVAL;
  if (d->kv_type == BIFATTN_KV_INT8 || d->kv_type == BIFATTN_KV_INT4) return BIFATTN_EUNSUPPORTED;
  if (d->kv_type != BIFATTN_KV_BF16 && d->kv_type != BIFATTN_KV_FP8_E4M3 && d->kv_type != BIFATTN_KV_MXFP4)
    return BIFATTN_EINVAL;
  if (d->d != 64 && d->d != 128) return BIFATTN_EUNSUPPORTED;
  if (d->page < 1) return BIFATTN_EINVAL;
  if (d->page < 16 || d->page > 256 || (d->page & (d->page - 1))) return BIFATTN_EUNSUPPORTED;
  const double ntok = d->n > 0 ? d->n : 1, maps = d->maps == 2 ? 2 : 1;
  if (maps * (d->h / d->g) * ntok > kMaxP) return BIFATTN_EUNSUPPORTED;
  // row numbers up to three strides past the end stay within 32 bits
  if (d->m_c > (1 << 29) || d->m_d_max > (1 << 29)) return BIFATTN_EUNSUPPORTED;
  if (maps * d->b * d->h * ntok > INT32_MAX / 2 || (double)d->b * d->g > INT32_MAX / 2) return BIFATTN_EINVAL;
  if ((double)d->num_pages * d->g * d->page * d->d * 2 > 4.0e18 ||
      (double)d->b * (d->m_c + (double)d->m_d_max) * d->g * d->d > 4.0e18)
    return BIFATTN_EINVAL;
  return BIFATTN_OK;
}

// Partials' loads that a combine wave issues together, at most (three work-groups
// of four waves per CU hold 16).
int64_t combine_loads(const bifattn_paged_plan_s* P) {
  return (int64_t)P->maps * P->dims.b * P->dims.h * P->ntok > 12 * kCUs ? 8 : 16;
}

// Keys of an own-row work-group: the whole capacity up to 1024 keys, halved
// (not below 256) while fewer than half as many work-groups as CUs would exist.
int own_chunk(int64_t units, int64_t rows) {
  int keys = (int)std::min<int64_t>(1024, std::max<int64_t>(128, round_up(rows, 128)));
  while (keys / 2 >= 256 && units * ceil_div(rows, keys) < kCUs / 2) keys /= 2;
  return keys;
}

// Waves per work-group (8 or 4) and key splits of a many-row context part: the
// least of an estimate of the step's time over both and over the splits. Its
// terms are the parts of a step (a context work-group's start and keys, the
// own-row work-groups beside the last round of context ones, the partials and
// the combine's loads), its constants a fit of whole steps: 1500 random layers
// (33 to 10^4 rows per group, 0.1k to 40k keys, every type, both head kinds) at
// about ten settings each. Over 1500 others the choice is 1.8% slower than the
// best of those settings on average, 8% at the 95th percentile, 29% at worst; a fixed number
// of work-groups (160 of eight waves, 256 of four) 12%, 37% and up to 2.8 times.
struct ManySplit {
  int waves = 4;
  int64_t splits = 1;
};
int many_step(int waves) { return waves == 8 ? 128 : 64; }  // keys of a stage
ManySplit many_row_split(const bifattn_paged_plan_s* P) {
  const bifattn_paged_dims_t& d = P->dims;
  const bool half = d.d == 64;
  const int64_t units = (int64_t)d.b * d.g;
  const int64_t own = P->dec_tiles <= 2 ? units * P->S_d : 0;  // own-row work-groups in the launch
  const double codes = d.kv_type == BIFATTN_KV_BF16 ? 1.0 : d.kv_type == BIFATTN_KV_FP8_E4M3 ? 0.6 : 0.4;
  const double bytes = 2.0 * d.g * paged_row_bytes(d.d, d.kv_type) * ((double)d.m_c + 0.75 * (double)d.b * d.m_d_max);
  const double kv = d.kv_type == BIFATTN_KV_BF16 ? 1.41 : d.kv_type == BIFATTN_KV_FP8_E4M3 ? 0.84 : 1.08;
  const double td = 2.93 + 1.69 * (half ? 0.5 : 1.0) * codes * std::min(P->dec_keys, d.m_d_max) / 128.0;
  ManySplit best;
  double least = -1.0;
  for (int waves = 4; waves <= 8; waves += 4) {
    const int64_t slots = waves == 8 ? kCUs : (half ? 3 : 2) * kCUs;
    const int64_t per_split = (int64_t)d.g * P->maps * ceil_div(P->Mh, 32 * waves);
    const int64_t own_wgs = ceil_div(own, waves / kWaves);
    const int64_t most = std::max<int64_t>(1, std::min(ceil_div(d.m_c, many_step(waves)), 4 * kCUs / per_split));
    for (int64_t S = 1; S <= most; S += 1 + S / 8) {
      const int64_t keys = round_up(ceil_div(d.m_c, S), many_step(waves));
      const int64_t parts = ceil_div(d.m_c, keys), wgs = per_split * parts;
      // the clock gives way as more than five eighths of the CUs run context
      // work-groups; those that share a CU slow each other
      const double busy = (1.0 + 0.06 * (double)std::max<int64_t>(0, std::min<int64_t>(wgs, kCUs) - 160) / 96.0) *
                          (1.0 + 0.38 * (double)(ceil_div(std::min(wgs, slots), kCUs) - 1));
      const double tc = (waves == 8 ? 4.5 : 3.0) + (waves == 8 ? 0.0198 : 0.0194) * (half ? 0.58 : 1.0) *
                                                       (P->maps == 2 ? 0.89 : 1.0) * kv * (double)keys * busy;
      const int64_t rem = wgs % slots;
      const double tr = rem ? tc : 0.0, alone = (double)ceil_div(own_wgs, slots - rem) * td;
      const double beside = own_wgs == 0       ? 0.0
                            : alone <= tr + td ? alone
                                               : ((double)rem * tc + (double)own_wgs * td) / (double)slots + 0.23 * td;
      double t = (double)(wgs / slots) * tc + std::max(tr, beside) + 0.05 * std::min(tr, beside);
      t = std::max(t, bytes / 7.5e6);
      const int64_t loads = ceil_div(parts * d.d, 256) + ceil_div(4 * (int64_t)P->S_d * d.d, 256);
      t += 1.66 * (double)(ceil_div(loads, combine_loads(P)) - 1) +
           (double)(parts + 4 * P->S_d) * P->M * d.g * (d.d * 4 + 16) / 2.1e6;
      if (least < 0.0 || t < least) {
        least = t;
        best.waves = waves;
        best.splits = S;
      }
    }
  }
  return best;
}

// Keys of a few-row context work-group: the least of an estimate of the step's
// time. A step is as long as its longest work-group (whose keys take longer as
// the GPU fills), the work over the slots, or the bytes, with the partials and
// the combine behind it. The constants are a fit of whole steps: 1500 random
// layers (up to 32 rows per group, 0.5k to 40k keys) at about nine chunks each;
// over 1500 others the choice is 2.1% slower than the best chunk on average, 10%
// at the 95th percentile (chunks of twice an even share over 512 slots, within
// 256 and 2048: 4.4%, 16%).
int64_t few_row_keys(const bifattn_paged_plan_s* P) {
  const bifattn_paged_dims_t& d = P->dims;
  const bool bf16 = d.kv_type == BIFATTN_KV_BF16, fp8 = d.kv_type == BIFATTN_KV_FP8_E4M3;
  const double slots = kCUs * (bf16 ? 2.95 : fp8 ? 1.65 : 1.51) * (d.d == 64 ? 1.5 : 1.0);
  const double key = (bf16 ? 7.4e-3 : fp8 ? 7.2e-3 : 6.6e-3) * (d.d == 64 ? 0.51 : 1.0);
  const int64_t units = (int64_t)d.b * d.g;
  const double td =
      P->S_d ? 3.52 + key * (P->R > 16 ? 1.87 : 1.0) * (double)round_up(std::min(P->dec_keys, d.m_d_max), 128) : 0.0;
  const double bytes = 2.0 * paged_row_bytes(d.d, d.kv_type) * ((double)d.g * d.m_c + 0.75 * (double)units * d.m_d_max);
  int64_t best = 128;
  double least = -1.0;
  for (int64_t keys = 128; keys <= 2560; keys += keys < 768 ? 128 : keys < 1536 ? 256 : 512) {
    const int64_t S = ceil_div(d.m_c, keys), wgs = d.g * S + units * P->S_d;
    // whole tiles of the group's 4 S waves
    const double tc = 3.52 + key * (P->M > 16 ? 1.87 : 1.0) * (double)(128 * ceil_div(d.m_c, 128 * S));
    const double chain = std::max(tc, td);
    const double filled = std::max(((double)d.g * S * tc + (double)units * P->S_d * td) / slots, bytes / 6.09e6);
    const int64_t loads = ceil_div(S * d.d, 256) + ceil_div(4 * (int64_t)P->S_d * d.d, 256);
    double t = std::max(chain * (1.0 + 0.24 * std::min(1.0, (double)wgs / slots)), filled) + 0.15 * std::min(chain, filled);
    t += 8.1e-7 * (double)(S + kWaves * P->S_d) * P->M * d.g * (d.d * 4 + 16) +
         1.58 * (double)(ceil_div(loads, combine_loads(P)) - 1) + (loads > 8 ? 0.66 : 0.0);
    if (least < 0.0 || t < least) least = t, best = keys;
  }
  return best;
}

// Whether a step runs as one launch without partials (whole_kernel): where the
// estimate of its time, us, is below that of the parts and the combine. Both are
// fits to 1500 random layers timed either way (up to 1536 units of at most 32
// query rows, 4000 keys); over 1500 others the choice is 0.6% slower than the
// faster way on average, 3% at the 95th percentile (always in parts: 21%).
//   one launch: a start, the unit's keys, which take longer as units share a
//     CU, and their bytes; never below a launch's own cost;
//   in parts: a start, the longest work-group's keys, partials, work-groups
//     beyond the GPU's slots, bytes; never below two launches'.
bool takes_one_launch(const bifattn_paged_plan_s* P) {
  const bifattn_paged_dims_t& d = P->dims;
  const int64_t units = (int64_t)d.b * d.g;
  const int env = env_int("BIFATTN_WHOLE", 0);  // 1: where it can, 2: never
  if (P->dec_tiles > 2 || env == 2) return false;
  if (env == 1) return true;
  if (units > 1536 || (int64_t)d.m_c + d.m_d_max > 4000) return false;
  const bool two = P->R > 16;
  const double half = d.d == 64 ? 0.52 : 1.0;
  const double code = d.kv_type == BIFATTN_KV_BF16 ? 7.4e-3 : d.kv_type == BIFATTN_KV_FP8_E4M3 ? 8.0e-3 : 7.6e-3;
  const double key = code * half * (two ? 1.7 : 1.0);
  const double row = 2.0 * paged_row_bytes(d.d, d.kv_type);
  const double keys = (double)d.m_c + d.m_d_max;
  const double one = std::max(6.5, 5.4 + (two ? 0.6 : 0.0) +
                                       key * keys * (1.0 + 1.84 * std::max(0.0, (double)units / 368.0 - 1.0)) +
                                       row * (double)units * keys / 26.5e6);
  double parts = row * ((double)units * d.m_d_max + (double)d.g * d.m_c) / 10.3e6 +
                 6.7e-7 * (double)(P->S_c + kWaves * P->S_d) * P->M * d.g * (d.d * 4 + 16) +
                 1.1 * std::max(0.0, (double)(P->n_ctx_blocks + P->n_ctx_small_blocks + P->n_dec_blocks) / 512.0 - 1.0);
  if (P->ctx_wide)
    parts += 7.7 + 0.023 * half * P->ctx_keys;
  else
    parts += 7.2 + key * std::max(P->S_c ? (double)d.m_c / P->S_c : 0.0, (double)std::min(P->dec_keys, d.m_d_max));
  return one <= std::max(8.7, parts);
}

bifattn_status_t split_work(bifattn_paged_plan_s* P) {
  const bifattn_paged_dims_t& d = P->dims;
  P->ntok = d.n > 0 ? d.n : 1;
  P->maps = d.maps == 2 ? 2 : 1;
  while ((1 << P->shift) < d.page) ++P->shift;
  P->pn = d.h / d.g * P->ntok;
  P->R = P->maps * P->pn;
  P->Mh = d.b * P->pn;
  P->M = P->maps * P->Mh;
  P->dec_tiles = P->R <= 16 ? 1 : (P->R <= 32 ? 2 : 4);
  const int64_t units = (int64_t)d.b * d.g, M = P->M;
  if (d.m_d_max > 0) {
    P->dec_keys = (int)round_up(env_int("BIFATTN_DEC_KEYS", own_chunk(units, d.m_d_max)), kWaves * kTileKeys);
    P->S_d = (int)ceil_div(d.m_d_max, P->dec_keys);
  }
  if (units * P->S_d > INT32_MAX / 4) return BIFATTN_EINVAL;
  P->n_dec_blocks = (int)(units * P->S_d);
  if (d.m_c == 0) return BIFATTN_OK;
  // Few rows per group (the streaming kernel): what its variants hold, two query
  // tiles, four where a unit has as many. Against the many-row kernel with 8 to 32
  // rows (13 layers of every type) 8 to 60% faster in 35 of 39 and 3 to 8% slower in
  // the others, all grouped ones of 32 rows; with 64 rows per unit and one unit per
  // group (4 layers of every type) 37 to 51% faster.
  if (M <= 32 || (M <= 64 && P->dec_tiles == 4)) {
    P->ctx_tiles = M <= 16 ? 1 : (M <= 32 ? 2 : 4);
    if (P->ctx_tiles < P->dec_tiles) P->ctx_tiles = P->dec_tiles;
    const int64_t keys = few_row_keys(P);
    P->ctx_keys = (int)round_up(env_int("BIFATTN_CTX_KEYS", (int)keys), kWaves * kTileKeys);
    P->S_c = (int)ceil_div(d.m_c, P->ctx_keys);
    if ((int64_t)d.g * P->S_c > INT32_MAX / 4) return BIFATTN_EINVAL;
    P->n_ctx_small_blocks = d.g * P->S_c;
  } else {
    ManySplit split = many_row_split(P);
    const int wgs = env_int("BIFATTN_CTX_WGS", 0);
    if (wgs > 0) {
      split.waves = env_int("BIFATTN_CTX_WIDE", split.waves) == 8 ? 8 : 4;
      split.splits = ceil_div(wgs, (int64_t)d.g * P->maps * ceil_div(P->Mh, 32 * split.waves));
    }
    P->ctx_wide = split.waves;
    P->ctx_row_blocks = P->maps * (int)ceil_div(P->Mh, 32 * P->ctx_wide);
    P->ctx_keys = (int)round_up(ceil_div(d.m_c, split.splits), many_step(P->ctx_wide));
    P->S_c = (int)ceil_div(d.m_c, P->ctx_keys);
    if ((int64_t)d.g * P->S_c * P->ctx_row_blocks > INT32_MAX / 4) return BIFATTN_EINVAL;
    P->n_ctx_blocks = d.g * P->S_c * P->ctx_row_blocks;
  }
  return BIFATTN_OK;
}

struct Layout {
  size_t ctx_acc = 0, ctx_ml = 0, dec_acc = 0, dec_ml = 0, tickets = 0, bytes = 0;
};
Layout layout(const bifattn_paged_plan_s* P) {
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  const size_t ctx = (size_t)P->dims.g * P->S_c * P->M;
  const size_t dec = (size_t)P->n_dec_blocks * kWaves * P->R;
  Layout L;
  size_t off = up(ctx * P->dims.d * 4);
  L.ctx_ml = off;
  off = up(off + ctx * 8);
  L.dec_acc = off;
  off = up(off + dec * P->dims.d * 4);
  L.dec_ml = off;
  off = up(off + dec * 8);
  L.tickets = off;  // b tickets, then the status word
  L.bytes = up(off + 4 * ((size_t)P->dims.b + 1));
  return L;
}

bool release(bifattn_paged_plan_s* P) {
  bool ok = true;
  if (P->done_ev) (void)hipEventDestroy(P->done_ev);
  if (P->ws) {
    if (P->ws_async)
      ok = hipFreeAsync(P->ws, P->own) == hipSuccess && hipStreamSynchronize(P->own) == hipSuccess;
    else
      ok = hipFree(P->ws) == hipSuccess;
  }
  if (P->own) (void)hipStreamDestroy(P->own);
  if (!ok) (void)hipGetLastError();
  delete P;
  return ok;
}

bifattn_status_t check_pages(const bifattn_paged_plan_s* P, const bifattn_pages_t* pages, PagePool* pool) {
  if (!pages || !pages->K || !pages->V) return BIFATTN_EINVAL;
  const bool mx = P->dims.kv_type == BIFATTN_KV_MXFP4, fp8 = P->dims.kv_type == BIFATTN_KV_FP8_E4M3;
  if (mx != (pages->K_exp != nullptr) || mx != (pages->V_exp != nullptr)) return BIFATTN_EINVAL;
  if (!fp8 && (pages->k_scale || pages->v_scale)) return BIFATTN_EINVAL;
  if (!aligned(pages->K, 16) || !aligned(pages->V, 16) || !aligned(pages->K_exp, 4) ||
      !aligned(pages->V_exp, 4) || !aligned(pages->k_scale, 4) || !aligned(pages->v_scale, 4))
    return BIFATTN_EALIGN;
  pool->K = static_cast<uint8_t*>(pages->K);
  pool->V = static_cast<uint8_t*>(pages->V);
  pool->K_exp = pages->K_exp;
  pool->V_exp = pages->V_exp;
  pool->k_scale = pages->k_scale;
  pool->v_scale = pages->v_scale;
  pool->num_pages = P->dims.num_pages;
  pool->g = P->dims.g;
  pool->shift = P->shift;
  return BIFATTN_OK;
}

// The two parts and the combine of one attention step; maps from the plan.
bifattn_status_t attend(bifattn_paged_plan_s* P, const void* q, const bifattn_pages_t* pages,
                        const int32_t* ctx_table, const int32_t* tables, const int32_t* lens,
                        const float* lambda, const float* weight, float eps, float out_scale, void* out,
                        hipStream_t stream) {
  const bifattn_paged_dims_t& d = P->dims;
  PagedAttnParams K{};
  const bifattn_status_t st = check_pages(P, pages, &K.pool);
  if (!q || !out || (d.m_c > 0 && !ctx_table) || (d.m_d_max > 0 && (!tables || !lens)) ||
      !on_plan_device(P, stream))
    return BIFATTN_EINVAL;
  if (st != BIFATTN_OK) return st;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ctx_table, 4) || !aligned(tables, 4) || !aligned(lens, 4))
    return BIFATTN_EALIGN;
  K.q = static_cast<const uint16_t*>(q);
  K.ctx_table = ctx_table;
  K.tables = tables;
  K.lens = d.m_d_max > 0 ? lens : nullptr;
  K.ctx_acc = P->ctx_acc;
  K.ctx_ml = P->ctx_ml;
  K.dec_acc = P->dec_acc;
  K.dec_ml = P->dec_ml;
  K.status = P->status;
  K.b = d.b;
  K.hn = d.h * P->ntok;
  K.g = d.g;
  K.pn = P->pn;
  K.maps = P->maps;
  K.R = P->R;
  K.Mh = P->Mh;
  K.M = P->M;
  K.ntok = P->ntok;
  K.m_c = d.m_c;
  K.m_d_max = d.m_d_max;
  K.table_pages = (int)ceil_div(d.m_d_max, d.page);
  K.ctx_keys = P->ctx_keys;
  K.S_c = P->S_c;
  K.ctx_row_blocks = P->ctx_row_blocks;
  K.ctx_wide = P->ctx_wide;
  K.dec_keys = P->dec_keys;
  K.S_d = P->S_d;
  // scale * (q . k) = |scale| * ((-q) . k): the kernels see a positive scale
  K.scale_log2 = std::fabs(P->scale) * 1.4426950408889634f;
  K.q_sign = P->scale < 0.f ? 0x80008000u : 0u;
  PagedCombineParams C{};
  C.ctx_acc = P->ctx_acc;
  C.ctx_ml = P->ctx_ml;
  C.dec_acc = P->dec_acc;
  C.dec_ml = P->dec_ml;
  C.lens = K.lens;
  C.k_scale = pages->k_scale;
  C.v_scale = pages->v_scale;
  C.lambda = lambda;
  C.weight = weight;
  C.eps = eps;
  C.out_scale = out_scale;
  C.out = static_cast<uint16_t*>(out);
  C.status = P->status;
  C.b = d.b;
  C.hn = K.hn;
  C.g = d.g;
  C.pn = P->pn;
  C.maps = P->maps;
  C.R = P->R;
  C.Mh = P->Mh;
  C.M = P->M;
  C.ntok = P->ntok;
  C.m_d_max = d.m_d_max;
  C.S_c = P->S_c;
  C.S_d = P->S_d * kWaves;
  hipError_t e = hipSuccess;
  if (P->whole) {
    const PagedWholeParams W{K, C};
    e = launch_paged_whole(W, d.d, d.kv_type, P->dec_tiles, stream, P->done_ev);
    return e == hipSuccess ? BIFATTN_OK : BIFATTN_EHIP;
  }
  if (P->ctx_wide) {
    // Units of more than 32 rows need more registers than two waves per SIMD
    // have: their own rows follow in a launch of their own.
    const bool one = P->dec_tiles <= 2;
    K.n_ctx_blocks = P->n_ctx_blocks;
    K.n_dec_blocks = one ? P->n_dec_blocks : 0;
    e = launch_paged_wide(K, d.d, d.kv_type, P->dec_tiles, stream);
    K.n_dec_blocks = one ? 0 : P->n_dec_blocks;
    if (e == hipSuccess && K.n_dec_blocks) e = launch_paged_stream(K, d.d, d.kv_type, 0, P->dec_tiles, stream);
  } else {
    K.n_ctx_small_blocks = P->n_ctx_small_blocks;
    K.n_dec_blocks = P->n_dec_blocks;
    e = launch_paged_stream(K, d.d, d.kv_type, P->ctx_tiles, P->dec_tiles, stream);
  }
  if (e != hipSuccess) return BIFATTN_EHIP;
  return launch_paged_combine(C, d.d, stream, P->done_ev) == hipSuccess ? BIFATTN_OK : BIFATTN_EHIP;
}

// The sequence kind that a call names: its row capacity, 0 when the plan has none.
int capacity(const bifattn_paged_plan_s* P, int32_t context) { return context ? P->dims.m_c : P->dims.m_d_max; }

}  // namespace

extern "C" {

bifattn_status_t bifattn_paged_plan_create(const bifattn_paged_dims_t* dims, bifattn_paged_plan_t* plan) {
  if (!plan) return BIFATTN_EINVAL;
  *plan = nullptr;
  bifattn_status_t st = check_dims(dims);
  if (st != BIFATTN_OK) return st;
  bifattn_paged_plan_s* P = new (std::nothrow) bifattn_paged_plan_s();
  if (!P) return BIFATTN_ENOMEM;
  P->dims = *dims;
  st = split_work(P);
  if (st != BIFATTN_OK) {
    delete P;
    return st;
  }
  P->whole = takes_one_launch(P);
  P->scale = dims->scale != 0.f ? dims->scale : 1.0f / std::sqrt((float)dims->d / (float)P->maps);
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1 || hipGetDevice(&P->device) != hipSuccess) {
    (void)hipGetLastError();
    delete P;
    return BIFATTN_EHIP;
  }
  const Layout L = layout(P);
  if (hipStreamCreateWithFlags(&P->own, hipStreamNonBlocking) != hipSuccess) {
    (void)hipGetLastError();
    delete P;
    return BIFATTN_EHIP;
  }
  if (hipMallocAsync(&P->ws, L.bytes, P->own) == hipSuccess) {
    P->ws_async = true;
  } else {
    (void)hipGetLastError();
    P->ws = nullptr;
    if (hipMalloc(&P->ws, L.bytes) != hipSuccess) {
      (void)hipGetLastError();
      P->ws = nullptr;
      release(P);
      return BIFATTN_ENOMEM;
    }
  }
  char* base = static_cast<char*>(P->ws);
  P->ws_bytes = L.bytes;
  P->ctx_acc = reinterpret_cast<float*>(base + L.ctx_acc);
  P->ctx_ml = reinterpret_cast<float2*>(base + L.ctx_ml);
  P->dec_acc = reinterpret_cast<float*>(base + L.dec_acc);
  P->dec_ml = reinterpret_cast<float2*>(base + L.dec_ml);
  P->tickets = reinterpret_cast<int*>(base + L.tickets);
  P->status = P->tickets + dims->b;
  if (hipMemsetAsync(P->tickets, 0, 4 * ((size_t)dims->b + 1), P->own) != hipSuccess ||
      hipStreamSynchronize(P->own) != hipSuccess ||
      hipEventCreateWithFlags(&P->done_ev, kOrderEventFlags) != hipSuccess) {
    (void)hipGetLastError();
    release(P);
    return BIFATTN_EHIP;
  }
  *plan = P;
  return BIFATTN_OK;
}

bifattn_status_t bifattn_paged_plan_destroy(bifattn_paged_plan_t P) {
  if (!P) return BIFATTN_OK;
  // an event that was never recorded is complete
  bifattn_status_t st = hipEventSynchronize(P->done_ev) == hipSuccess ? BIFATTN_OK : BIFATTN_EHIP;
  if (!release(P)) st = BIFATTN_EHIP;
  return st;
}

bifattn_status_t bifattn_paged_plan_get_info(bifattn_paged_plan_t P, bifattn_plan_info_t* info) {
  if (!P || !info) return BIFATTN_EINVAL;
  *info = bifattn_plan_info_t{};
  info->ctx_keys_per_block = P->ctx_keys;
  info->ctx_splits = P->S_c;
  info->ctx_row_blocks = P->ctx_row_blocks;
  info->ctx_blocks = P->n_ctx_blocks + P->n_ctx_small_blocks;
  info->dec_keys_per_block = P->dec_keys;
  info->dec_splits = P->S_d * kWaves;
  info->dec_blocks = P->n_dec_blocks;
  info->fused = !P->ctx_wide || P->dec_tiles <= 2;
  info->path = P->whole ? BIFATTN_PATH_STANDARD : BIFATTN_PATH_BIFURCATED;
  info->workspace_bytes = P->ws_bytes;
  info->ctx_kernel = P->ctx_wide ? 2 : 0;
  return BIFATTN_OK;
}

bifattn_status_t bifattn_paged_plan_status(bifattn_paged_plan_t P, hipStream_t stream) {
  if (!P) return BIFATTN_EINVAL;
  if (hipStreamSynchronize(stream) != hipSuccess) return BIFATTN_EHIP;
  int flag = 0;
  if (hipMemcpy(&flag, P->status, sizeof flag, hipMemcpyDeviceToHost) != hipSuccess) return BIFATTN_EHIP;
  if (!flag) return BIFATTN_OK;
  if (hipMemset(P->status, 0, sizeof flag) != hipSuccess) return BIFATTN_EHIP;
  return flag & kStatusPage ? BIFATTN_EPAGE : flag & kStatusScale ? BIFATTN_ESCALE : BIFATTN_ELENS;
}

bifattn_status_t bifattn_paged_append(bifattn_paged_plan_t P, const bifattn_pages_t* pages, const int32_t* table,
                                      const bifattn_new_rows_t* rows, const int32_t* lens, int32_t* lens_out,
                                      hipStream_t stream) {
  if (!P || !table || !rows || !lens || !lens_out || !rows->k || !rows->v) return BIFATTN_EINVAL;
  const bifattn_paged_dims_t& d = P->dims;
  PagedAppendParams A{};
  bifattn_status_t st = check_pages(P, pages, &A.pool);
  if (st == BIFATTN_EINVAL) return st;
  A.max_rows = capacity(P, rows->context);
  if (rows->samples < 1 || rows->samples > (rows->context ? 1 : d.b) || rows->n < 1 || rows->n > (1 << 29) || A.max_rows < 1 ||
      (rows->q != nullptr) != (rows->q_out != nullptr) || rows->rot < 0 || rows->rot > d.d / P->maps ||
      (rows->rot > 0 && !rows->freqs) || !on_plan_device(P, stream))
    return BIFATTN_EINVAL;
  if (rows->rot % 16) return BIFATTN_EUNSUPPORTED;
  if (st != BIFATTN_OK) return st;
  if (!aligned(rows->q, 16) || !aligned(rows->k, 16) || !aligned(rows->v, 16) || !aligned(rows->q_out, 16) ||
      !aligned(rows->freqs, 4) || !aligned(rows->counts, 4) || !aligned(table, 4) || !aligned(lens, 4) ||
      !aligned(lens_out, 4))
    return BIFATTN_EALIGN;
  for (int k = 0; k < 3; ++k) {
    if ((rows->q && rows->q_stride[k] % 8) || rows->k_stride[k] % 8 || rows->v_stride[k] % 8) return BIFATTN_EALIGN;
    A.qs[k] = rows->q_stride[k];
    A.ks[k] = rows->k_stride[k];
    A.vs[k] = rows->v_stride[k];
  }
  // lens_out may be lens or counts, whose elements the kernel then replaces when
  // all have been read; a part of one would be another sample's input.
  for (const int32_t* in : {lens, rows->counts}) {
    if (!in) continue;
    const uintptr_t a = (uintptr_t)in, z = (uintptr_t)lens_out, bytes = 4 * (uintptr_t)rows->samples;
    if (a == z)
      A.in_place = 1;
    else if (a < z + bytes && z < a + bytes)
      return BIFATTN_EINVAL;
  }
  A.table = table;
  A.lens = lens;
  A.counts = rows->counts;
  A.lens_out = lens_out;
  A.tickets = P->tickets;
  A.status = P->status;
  A.q = static_cast<const uint16_t*>(rows->q);
  A.k = static_cast<const uint16_t*>(rows->k);
  A.v = static_cast<const uint16_t*>(rows->v);
  A.q_out = static_cast<uint16_t*>(rows->q_out);
  A.freqs = rows->freqs;
  A.h = rows->q ? d.h : 0;
  A.g = d.g;
  A.n = rows->n;
  A.d = d.d;
  A.maps = P->maps;
  A.rot = rows->rot;
  A.neighbours = rows->neighbours != 0;
  A.table_pages = (int)ceil_div(A.max_rows, d.page);
  A.position0 = rows->context ? 0 : d.m_c;
  A.samples = rows->samples;
  // A pass of a work-group takes 32 rows of 128 elements (64 of 64). Few tokens:
  // one pass a work-group. Many: whole tokens, as many (up to 8) as fill their
  // passes best, while four work-groups per CU remain.
  const int heads = A.h + 2 * A.g, pass = 256 / (d.d / 16);
  const bool many = (int64_t)A.samples * A.n * ceil_div(heads, pass) > 8 * kCUs;
  A.heads_per_block = many ? heads : std::min(heads, pass);
  A.tokens_per_block = 1;
  double fill = 0.0;
  for (int T = 1; many && T <= 8 && (T == 1 || A.samples * ceil_div(A.n, T) >= 4 * kCUs); ++T) {
    const double f = (double)(T * heads) / (double)round_up(T * heads, pass);
    if (f > fill + 0.02) fill = f, A.tokens_per_block = T;
  }
  A.head_blocks = (int)ceil_div(heads, A.heads_per_block);
  const int64_t token_blocks = ceil_div(A.n, A.tokens_per_block);
  if ((double)A.samples * (double)token_blocks * A.head_blocks > INT32_MAX / 2) return BIFATTN_EINVAL;
  A.token_blocks = (int)token_blocks;
  return launch_paged_append(A, d.kv_type, stream, P->done_ev) == hipSuccess ? BIFATTN_OK : BIFATTN_EHIP;
}

bifattn_status_t bifattn_paged_gather(bifattn_paged_plan_t P, const bifattn_pages_t* pages, const int32_t* table,
                                      const int32_t* first, const int32_t* lens, int32_t samples, int32_t rows,
                                      int32_t context, void* k_out, void* v_out, hipStream_t stream) {
  if (!P || !table || !lens || !k_out || !v_out) return BIFATTN_EINVAL;
  PagedGatherParams G{};
  const bifattn_status_t st = check_pages(P, pages, &G.pool);
  if (st == BIFATTN_EINVAL) return st;
  G.max_rows = capacity(P, context);
  if (samples < 1 || samples > (context ? 1 : P->dims.b) || rows < 1 || G.max_rows < 1 || !on_plan_device(P, stream))
    return BIFATTN_EINVAL;
  if (st != BIFATTN_OK) return st;
  if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(table, 4) || !aligned(first, 4) || !aligned(lens, 4))
    return BIFATTN_EALIGN;
  G.table = table;
  G.first = first;
  G.lens = lens;
  G.k_out = static_cast<uint16_t*>(k_out);
  G.v_out = static_cast<uint16_t*>(v_out);
  G.status = P->status;
  G.d = P->dims.d;
  G.samples = samples;
  G.rows = rows;
  G.table_pages = (int)ceil_div(G.max_rows, P->dims.page);
  return launch_paged_gather(G, P->dims.kv_type, stream, P->done_ev) == hipSuccess ? BIFATTN_OK : BIFATTN_EHIP;
}

bifattn_status_t bifattn_paged_decode(bifattn_paged_plan_t P, const void* q, const bifattn_pages_t* pages,
                                      const int32_t* ctx_table, const int32_t* tables, const int32_t* lens,
                                      void* out, hipStream_t stream) {
  if (!P || P->maps != 1) return BIFATTN_EINVAL;
  return attend(P, q, pages, ctx_table, tables, lens, nullptr, nullptr, 0.f, 1.f, out, stream);
}

bifattn_status_t bifattn_paged_decode_diff(bifattn_paged_plan_t P, const void* q, const bifattn_pages_t* pages,
                                           const int32_t* ctx_table, const int32_t* tables, const int32_t* lens,
                                           const float* lambda, const float* weight, float eps, float out_scale,
                                           void* out, hipStream_t stream) {
  if (!P || P->maps != 2 || !lambda || !(eps >= 0.f) || !std::isfinite(eps) || !std::isfinite(out_scale))
    return BIFATTN_EINVAL;
  if (!aligned(lambda, 4) || !aligned(weight, 16)) return BIFATTN_EALIGN;
  return attend(P, q, pages, ctx_table, tables, lens, lambda, weight, eps, out_scale, out, stream);
}

}  // extern "C"

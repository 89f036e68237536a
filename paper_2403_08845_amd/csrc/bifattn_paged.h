// Launch parameters shared by the host code and the HIP kernels of the paged
// caches (append, read-out, attention, differential attention).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "bifattn_internal.h"

namespace bifattn {

// Device-side status bit beside kStatusLens and kStatusScale: a page id
// outside the pool.
constexpr int kStatusPage = 4;

// Cache element types of a page pool (values of bifattn_kv_type_t).
enum PagedKv { kPagedBf16 = 0, kPagedFp8 = 1, kPagedMxfp4 = 4 };
constexpr int paged_row_bytes(int d, int kv) { return kv == kPagedBf16 ? 2 * d : kv == kPagedFp8 ? d : d / 2; }
// Elements that share one scale byte (MXFP4).
constexpr int kMxBlock = 32;

// The pool: rows of page `id`, group gam start at row (id*g + gam) << shift.
struct PagePool {
  uint8_t* K;          // [num_pages][g][page] rows
  uint8_t* V;
  uint8_t* K_exp;      // MXFP4: [num_pages][g][page][d/32] scale bytes, else null
  uint8_t* V_exp;
  const float* k_scale;  // [g], or null for 1 (never with MXFP4)
  const float* v_scale;
  int num_pages;
  int g;
  int shift;           // log2 of the rows of a page
};

struct PagedAttnParams {
  const uint16_t* q;          // [b][hn][d], hn = heads x tokens
  PagePool pool;
  const int32_t* ctx_table;   // page ids of the context
  const int32_t* tables;      // [b][table_pages]
  const int32_t* lens;        // [b], null without own rows
  float* ctx_acc;             // [g][S_c][M][d]
  float2* ctx_ml;             // [g][S_c][M]
  float* dec_acc;             // [b][g][S_d][4 waves][R][d]
  float2* dec_ml;             // [b][g][S_d][4 waves][R]
  int* status;
  int b, hn, g;
  int pn;                     // query rows of a (sample, group) unit in each map: heads x tokens
  int maps;                   // 1, or 2 (differential: map u uses half u of q and k)
  int R;                      // maps * pn: rows of a unit, row u*pn + jp
  int Mh, M;                  // b*pn rows of a group in each map; M = maps*Mh, row u*Mh + i*pn + jp
  int ntok;
  int m_c, m_d_max, table_pages;
  int ctx_keys, S_c;          // many-row path: keys of a context work-group; context splits
  int ctx_row_blocks;         // row blocks of all maps (many-row path)
  int ctx_wide;               // waves of a many-row work-group (8 or 4)
  int dec_keys, S_d;
  int n_ctx_blocks, n_ctx_small_blocks, n_dec_blocks;
  float scale_log2;           // |scale| * log2(e)
  uint32_t q_sign;            // 0x80008000 when scale < 0
};

struct PagedCombineParams {
  const float* ctx_acc;
  const float2* ctx_ml;
  const float* dec_acc;
  const float2* dec_ml;
  const int32_t* lens;
  const float* k_scale;
  const float* v_scale;
  const float* lambda;   // [h]: weight of the second map (maps = 2)
  const float* weight;   // [d] norm weight, or null: heads are not normalised
  float eps, out_scale;
  uint16_t* out;         // bf16 [b][hn][d]
  int* status;
  int b, hn, g, pn, maps, R, Mh, M, ntok;
  int m_d_max;
  int S_c, S_d;          // context splits, decode partials (4 per chunk)
};

// Small steps: both parts and the end of the row in one kernel.
struct PagedWholeParams {
  PagedAttnParams A;
  PagedCombineParams C;
};

struct PagedAppendParams {
  PagePool pool;
  const int32_t* table;     // [samples][table_pages]
  const int32_t* lens;      // [samples] first row to write
  const int32_t* counts;    // [samples] new rows, or null for n
  int32_t* lens_out;        // [samples]; may be lens or counts
  int in_place;             // it is one of them
  int* tickets;             // [samples], zero between calls: work-groups that have read lens and counts
  int* status;
  const uint16_t* q;        // null: no queries
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;          // [samples][h][n][d]
  const float* freqs;       // [rot/2] radians per position
  int64_t qs[3], ks[3], vs[3];  // elements between samples, heads, tokens
  int h, g, n, d, maps;
  int rot;                  // rotated elements of each of the maps parts of a row, a multiple of 16
  int neighbours;           // pairs (2j, 2j+1), else (j, j + rot/2)
  int table_pages, max_rows;
  int position0;            // position of row 0
  int samples;
  int tokens_per_block, token_blocks, heads_per_block, head_blocks;
};

struct PagedGatherParams {
  PagePool pool;
  const int32_t* table;
  const int32_t* first;     // [samples], or null for 0
  const int32_t* lens;
  uint16_t* k_out;          // bf16 [samples][g][rows][d]
  uint16_t* v_out;
  int* status;
  int d, samples, rows, table_pages, max_rows;
};

// Streaming launch: n_ctx_small_blocks few-row context work-groups (ctx_tiles
// query tiles, 0 without context), then n_dec_blocks decode ones (dec_tiles).
hipError_t launch_paged_stream(const PagedAttnParams& P, int d, int kv, int ctx_tiles, int dec_tiles,
                               hipStream_t stream);
// Many-row launch: n_ctx_blocks context work-groups, then n_dec_blocks decode
// ones (dec_tiles at most 2).
hipError_t launch_paged_wide(const PagedAttnParams& P, int d, int kv, int dec_tiles, hipStream_t stream);
// Small steps: one work-group per (sample, group), `tiles` (1 or 2) query tiles.
hipError_t launch_paged_whole(const PagedWholeParams& W, int d, int kv, int tiles, hipStream_t stream,
                              hipEvent_t stop);
hipError_t launch_paged_combine(const PagedCombineParams& C, int d, hipStream_t stream, hipEvent_t stop);
hipError_t launch_paged_append(const PagedAppendParams& A, int kv, hipStream_t stream, hipEvent_t stop);
hipError_t launch_paged_gather(const PagedGatherParams& G, int kv, hipStream_t stream, hipEvent_t stop);

}  // namespace bifattn

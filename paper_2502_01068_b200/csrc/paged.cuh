// Parameter blocks and launchers of the paged cache: appending rows (paged_append.cu) and attention (paged_attn.cu).
#pragma once

#include "common.cuh"
#include "paged_index.h"

namespace fastkv {

struct PagedView {
  int batch, max_pages, n_pages, page_log2, n_kv_heads;
  uint8_t* k_pages;           // [n_pages][n_kv_heads][page][d]
  uint8_t* v_pages;
  float* k_scales;            // [n_pages][n_kv_heads], 8-bit pages only
  float* v_scales;
  const int* block_table;     // [batch][max_pages]
};

struct AppendParams {
  PagedView c;
  int total, max_new, uniform, n_q_heads, rot_dim, adjacent, total_src;
  const int* lens;            // entries before the call
  int* new_lens;              // entries after it, may be null
  const int* cu_new;          // may be null (uniform)
  const int* cu_src;          // gathered rows: source offsets of the sequences, may be null (one sequence)
  const int* idx;             // gathered rows: [n_kv_heads][total], or null
  const int* pos;
  const float* inv_freq;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* q_out;
  long long q_tok, q_head, k_tok, k_head, v_tok, v_head;   // strides, elements
  WorkspaceHeader* hdr;
  long long wait_limit;       // cycles a wait polls before it gives up
  int skip_copy;              // test hook: this fill of the page role's slots is not started (-1: none)
  // work split, filled in by the launcher
  int page_blocks, heads_per_unit, row_heads, row_slices;  // row role, behind the page role's blocks
  int pages_per_seq, job_slices, jobs_per_slice;           // page role (8-bit pages)
  int small_log2;             // small role: lane groups of a (page, head)
};

// Whether the call reads k and v through tensor maps: (column, head, row) with boxes of a page's rows of one head, unswizzled.
bool paged_append_uses_maps(const AppendParams& p, bool e4m3);
cudaError_t launch_paged_append(AppendParams& p, const CUtensorMap (&maps)[2], int head_dim, bool e4m3, cudaStream_t stream);

constexpr int kPagedCtas = 2 * 148;      // attention CTAs that are resident at once: the most pieces of one (sequence, KV head)

struct PagedAttnParams {
  PagedView c;
  int n_q_heads, group, q_len, rows;     // rows = group * q_len query rows per (sequence, KV head)
  int row_tiles, tile_rows;   // tiles the rows are cut into, and rows of a tile (8 or 16)
  int splits;                 // static launches: CTAs that share a (sequence, KV head, row tile)
  int balanced, ctas;         // balanced launches: CTAs that share all of them
  long long wait_limit;       // cycles a wait polls before it gives up
  int skip_copy;              // test hook: the first pair of warps gets no copies for this chunk of a segment (-1: none)
  int joint, v_first;         // K and V are planes of one tensor map; the V pool lies at the lower address
  float scale_log2;           // softmax scale times log2(e)
  const int* lens;
  const uint16_t* q;          // [B][q_len][Hq][d]
  float* out;                 // [B][q_len][Hq][d]
  float* lse;                 // [B][q_len][Hq], may be null
  float2* part_ml;            // [pieces][tile_rows]: (max, sum)
  float* part_o;              // [pieces][tile_rows][d]
  WorkspaceHeader* hdr;
};

struct PagedAttnPlan {
  int row_tiles_of_8, row_tiles, splits, balanced, ctas;
};
PagedAttnPlan plan_paged_attn(int batch, int n_kv_heads, int rows, bool e4m3, int max_len, long long total_len);
size_t paged_attn_partials_offset(const PagedAttnPlan& plan, int batch, int n_kv_heads);
size_t paged_attn_workspace_bytes(const PagedAttnPlan& plan, int batch, int n_kv_heads, int head_dim);
// Entries of a page that one TMA box brings: a chunk's 32 of 8-bit pages when the page has them, else 16.
inline int paged_box_rows(bool e4m3, int page_size) { return e4m3 && page_size >= 32 ? 32 : 16; }
// tmap_k: with p.joint both pools, (column, row of the page, page x head, pool); else the K pool alone and tmap_v the V pool
cudaError_t launch_paged_attn(const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, PagedAttnParams& p, const PagedAttnPlan& plan,
                              int head_dim, bool e4m3, cudaStream_t stream, int* launches);

}  // namespace fastkv

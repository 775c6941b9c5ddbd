// Key-value cache in pages: launchers of page_table.hip, page_select.hip and paged_attention.hip, and what their hosts share.
#pragma once
#include "../../include/cerberus.h"
#include "common.h"

namespace cerb {

int set_error(int code, const char* fmt, ...);   // text of cerberus_last_error; returns code

// most: a sequence grows by at most that many rows
hipError_t launch_page_plan(const cerberus_page_table& pt, const int* new_rows, int most, int batch, int max_rows, int* row_start,
                            int* first_pos, int* slot, hipStream_t s);

struct PageStoreArgs {
  cerberus_pages pg;
  const void *k, *v;
  long long k_row, k_head, v_row, v_head;   // strides in elements
  const int* slot;
  int n_rows, page_shift;
  int* status;
};
hipError_t launch_page_store(const PageStoreArgs& a, hipStream_t s);

// bounds of the pages that a step's rows (slot [batch], one each) have filled, in all layers that keep any
hipError_t launch_page_bounds(const cerberus_pages* layers, int n_layers, const int* slot, int batch, hipStream_t s);

struct PageSelectArgs {
  cerberus_pages pg;
  const int *table, *lens;                  // [batch][max_blocks], [batch] rows
  int max_blocks, page_shift;
  const void* q;
  size_t q_lo_off;                          // bf16: if set, the queries' lo plane follows so many elements later
  long long q_row;
  int batch, n_heads, n_select;
  int* blocks;
  unsigned long long* keys;                 // workspace [batch][n_kv_heads][max_blocks]
};
size_t page_select_bytes(int batch, int n_kv_heads, int max_blocks);
hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t s);

struct PagedAttnArgs {
  cerberus_pages pg;
  const int *table, *lens;                  // [batch][max_blocks], [batch] rows to attend to
  int max_blocks, page_shift;
  const void* q;
  size_t q_lo_off;                          // as above
  long long q_row;
  void* out;
  size_t out_lo_off;                        // bf16: if set, the output's lo plane goes there
  long long out_row;
  int batch, n_heads;
  float scale;
  const int* blocks;                        // [batch][n_kv_heads][n_select], null: all blocks
  int n_select;
  // bf16: if set, what the cache's rounding left of the newest row (lens[b] - 1) of every sequence: [batch] rows of
  // n_kv_heads * head_dim, so many elements apart
  const void *own_k_lo, *own_v_lo;
  long long own_row;
  float* part;                              // workspace
  int* status;
};
int paged_attention_items(int batch, long long most, int unit, int per_head);   // pieces that a launch has workgroups for (unit 0: nothing is cut)
size_t paged_attention_bytes(int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s);

// What lies where in the workspace of the calls over pages
struct PagedWorkspace {
  float* part;                              // of the attention
  unsigned long long* keys;                 // of the choice of blocks
  // of the step over pages
  int *row_start, *first_pos, *slot, *lens; // [batch + 1], [batch], [batch], [batch]
  int* blocks;                              // [batch][n_kv_heads][n_select]
  size_t bytes;
};
PagedWorkspace paged_workspace(const cerberus_pages& pg, const cerberus_page_table& pt, int batch, int n_heads, int n_select, void* base);

// Inclusive sum over the 64 lanes of a wave in order, all of them active.  Shifts within rows of 16 lanes, then the rows' last lanes handed on:
// six adds without a trip through LDS (a scan by shuffles is ten times as long, and these kernels begin with it).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);    // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
  return v;
}
// the same for sums past 32 bits, of terms in 0 .. 2^40
__device__ __forceinline__ long long wave_scan(long long v) {
  const int lo = wave_scan((int)(v & 0xfffff)), hi = wave_scan((int)(v >> 20));
  return ((long long)hi << 20) + lo;
}

// argument checks of the public entry points, also those of the step over pages
int check_pages(const cerberus_pages* pg);
int check_page_table(const cerberus_page_table* pt, int batch);
int check_same_pages(const cerberus_pages* pg, const cerberus_page_table* pt);
inline int page_shift_of(int page_size) { int s = 0; while ((1 << s) < page_size) ++s; return s; }

}  // namespace cerb

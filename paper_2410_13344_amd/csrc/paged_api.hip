// Entry points of the cache in pages: argument checks and launches.  (The step over pages is with the other steps.)
#include "paged.h"

#include <cmath>
#include <limits.h>

using namespace cerb;

#define HIP_TRY(expr)                                                                                   \
  do {                                                                                                  \
    hipError_t e_ = (expr);                                                                             \
    if (e_ != hipSuccess) return set_error(CERBERUS_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_));   \
  } while (0)
#define TRY(expr)                       \
  do {                                  \
    int rc_ = (expr);                   \
    if (rc_ != CERBERUS_OK) return rc_; \
  } while (0)

namespace cerb {

namespace {
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
int elem_of(int dtype) { return dtype == CERBERUS_F32 ? 4 : 2; }
int check_page_size(int page_size) {
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)))
    return set_error(CERBERUS_ERR_SHAPE, "page_size must be a power of two in 16..256");
  return CERBERUS_OK;
}
}  // namespace

int check_pages(const cerberus_pages* pg) {
  if (!pg) return set_error(CERBERUS_ERR_ARG, "null pages");
  if (pg->dtype != CERBERUS_F32 && pg->dtype != CERBERUS_BF16) return set_error(CERBERUS_ERR_ARG, "dtype must be 0 (fp32) or 1 (bf16)");
  if (pg->head_dim != 64 && pg->head_dim != 128) return set_error(CERBERUS_ERR_SHAPE, "head_dim must be 64 or 128");
  TRY(check_page_size(pg->page_size));
  if (pg->n_pages < 1 || (long long)pg->n_pages * pg->page_size > INT_MAX) return set_error(CERBERUS_ERR_SHAPE, "n_pages out of 1..(2^31 - 1) / page_size");
  if (pg->n_kv_heads < 1 || pg->n_kv_heads > 1024) return set_error(CERBERUS_ERR_SHAPE, "n_kv_heads out of 1..1024");
  if (!pg->k || !pg->v) return set_error(CERBERUS_ERR_ARG, "null page pool");
  if (!aligned16(pg->k) || !aligned16(pg->v) || !aligned16(pg->bounds)) return set_error(CERBERUS_ERR_ARG, "page pools must be 16-byte aligned");
  return CERBERUS_OK;
}

int check_page_table(const cerberus_page_table* pt, int batch) {
  if (!pt) return set_error(CERBERUS_ERR_ARG, "null page table");
  if (!pt->block_table || !pt->kv_len || !pt->free_pages || !pt->n_free || !pt->status) return set_error(CERBERUS_ERR_ARG, "null pointer in cerberus_page_table");
  TRY(check_page_size(pt->page_size));
  if (pt->n_pages < 1 || (long long)pt->n_pages * pt->page_size > INT_MAX) return set_error(CERBERUS_ERR_SHAPE, "n_pages out of 1..(2^31 - 1) / page_size");
  if (pt->max_blocks < 1 || (long long)pt->max_blocks * pt->page_size > INT_MAX) return set_error(CERBERUS_ERR_SHAPE, "max_blocks out of 1..(2^31 - 1) / page_size");
  if (pt->max_seqs < 1 || pt->max_seqs > CERBERUS_MAX_SEQS) return set_error(CERBERUS_ERR_SHAPE, "max_seqs out of 1..%d", CERBERUS_MAX_SEQS);
  if (batch < 1 || batch > pt->max_seqs) return set_error(CERBERUS_ERR_ARG, "batch %d out of 1..%d", batch, pt->max_seqs);
  return CERBERUS_OK;
}

int check_same_pages(const cerberus_pages* pg, const cerberus_page_table* pt) {
  if (pg->page_size != pt->page_size || pg->n_pages != pt->n_pages) return set_error(CERBERUS_ERR_SHAPE, "pages and page table differ in page_size or n_pages");
  return CERBERUS_OK;
}

PagedWorkspace paged_workspace(const cerberus_pages& pg, const cerberus_page_table& pt, int batch, int n_heads, int n_select, void* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    unsigned char* p = reinterpret_cast<unsigned char*>(base) + off;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const size_t row = (size_t)batch * pg.n_kv_heads;
  PagedWorkspace w{};
  w.part = reinterpret_cast<float*>(take(paged_attention_bytes(n_heads, pg.n_kv_heads, pg.head_dim)));
  w.keys = reinterpret_cast<unsigned long long*>(take(n_select ? page_select_bytes(batch, pg.n_kv_heads, pt.max_blocks) : 0));
  w.row_start = reinterpret_cast<int*>(take((size_t)(batch + 1) * 4));
  w.first_pos = reinterpret_cast<int*>(take((size_t)batch * 4));
  w.slot = reinterpret_cast<int*>(take((size_t)batch * 4));
  w.lens = reinterpret_cast<int*>(take((size_t)batch * 4));
  w.blocks = reinterpret_cast<int*>(take(row * n_select * 4));
  w.bytes = off;
  return w;
}

}  // namespace cerb

namespace {

int check_heads(const cerberus_pages* pg, int n_heads) {
  if (n_heads < 1 || n_heads > 65535 || n_heads % pg->n_kv_heads) return set_error(CERBERUS_ERR_SHAPE, "n_heads must be a multiple of n_kv_heads, up to 65535");
  return CERBERUS_OK;
}

int check_rows(const cerberus_pages* pg, const void* p, int64_t row_stride, const char* what) {
  if (!p) return set_error(CERBERUS_ERR_ARG, "null %s", what);
  if (!aligned16(p) || (row_stride * elem_of(pg->dtype)) % 16) return set_error(CERBERUS_ERR_ARG, "%s and its strides must be multiples of 16 bytes", what);
  return CERBERUS_OK;
}

int check_workspace(const cerberus_pages* pg, const cerberus_page_table* pt, int batch, int n_heads, int n_select, const void* ws, size_t bytes) {
  const size_t need = cerberus_paged_workspace_bytes(pg, pt, batch, n_heads, n_select);
  if (need == 0) return set_error(CERBERUS_ERR_ARG, "n_select out of 0..max_blocks");
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) return set_error(CERBERUS_ERR_ARG, "workspace must be 256-byte aligned");
  if (bytes < need) return set_error(CERBERUS_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", bytes, need);
  return CERBERUS_OK;
}

}  // namespace

extern "C" {

int cerberus_page_plan(const cerberus_page_table* pt, const int32_t* new_rows, int32_t batch, int32_t max_rows, int32_t* row_start,
                       int32_t* first_pos, int32_t* slot, void* stream) {
  TRY(check_page_table(pt, batch));
  if (!new_rows || !row_start || !first_pos) return set_error(CERBERUS_ERR_ARG, "null argument");
  if (max_rows < 0 || (max_rows > 0 && !slot)) return set_error(CERBERUS_ERR_ARG, "max_rows < 0 or null slot");
  HIP_TRY(launch_page_plan(*pt, new_rows, INT_MAX, batch, max_rows, row_start, first_pos, slot, reinterpret_cast<hipStream_t>(stream)));
  return CERBERUS_OK;
}

int cerberus_page_store(const cerberus_pages* pg, const void* k, int64_t k_row_stride, int64_t k_head_stride, const void* v,
                        int64_t v_row_stride, int64_t v_head_stride, const int32_t* slot, int32_t n_rows, int32_t* status, void* stream) {
  TRY(check_pages(pg));
  if (n_rows < 0) return set_error(CERBERUS_ERR_ARG, "n_rows < 0");
  if (n_rows == 0) return CERBERUS_OK;
  if (!slot) return set_error(CERBERUS_ERR_ARG, "null slot");
  TRY(check_rows(pg, k, k_row_stride, "k"));
  TRY(check_rows(pg, v, v_row_stride, "v"));
  if ((k_head_stride * elem_of(pg->dtype)) % 16 || (v_head_stride * elem_of(pg->dtype)) % 16)
    return set_error(CERBERUS_ERR_ARG, "head strides must be multiples of 16 bytes");
  const PageStoreArgs a{*pg, k, v, k_row_stride, k_head_stride, v_row_stride, v_head_stride, slot, n_rows, page_shift_of(pg->page_size), status};
  HIP_TRY(launch_page_store(a, reinterpret_cast<hipStream_t>(stream)));
  return CERBERUS_OK;
}

size_t cerberus_paged_workspace_bytes(const cerberus_pages* pg, const cerberus_page_table* pt, int32_t batch, int32_t n_heads, int32_t n_select) {
  if (check_pages(pg) || check_page_table(pt, batch) || check_same_pages(pg, pt) || check_heads(pg, n_heads)) return 0;
  if (n_select < 0 || n_select > pt->max_blocks) { set_error(CERBERUS_ERR_ARG, "n_select out of 0..max_blocks"); return 0; }
  return paged_workspace(*pg, *pt, batch, n_heads, n_select, nullptr).bytes;
}

int cerberus_page_select(const cerberus_pages* pg, const cerberus_page_table* pt, const void* q, int64_t q_row_stride, int32_t batch,
                         int32_t n_heads, int32_t n_select, int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
  TRY(check_pages(pg));
  TRY(check_page_table(pt, batch));
  TRY(check_same_pages(pg, pt));
  TRY(check_heads(pg, n_heads));
  if (!pg->bounds) return set_error(CERBERUS_ERR_ARG, "cerberus_page_select needs the pages' bounds");
  if (n_select < 1 || !blocks) return set_error(CERBERUS_ERR_ARG, "n_select < 1 or null blocks");
  TRY(check_rows(pg, q, q_row_stride, "q"));
  TRY(check_workspace(pg, pt, batch, n_heads, n_select, workspace, workspace_bytes));
  const PagedWorkspace w = paged_workspace(*pg, *pt, batch, n_heads, n_select, workspace);
  PageSelectArgs a{};
  a.pg = *pg; a.table = pt->block_table; a.lens = pt->kv_len; a.max_blocks = pt->max_blocks; a.page_shift = page_shift_of(pg->page_size);
  a.q = q; a.q_row = q_row_stride; a.batch = batch; a.n_heads = n_heads; a.n_select = n_select; a.blocks = blocks; a.keys = w.keys;
  HIP_TRY(launch_page_select(a, reinterpret_cast<hipStream_t>(stream)));
  return CERBERUS_OK;
}

int cerberus_paged_attention(const cerberus_pages* pg, const cerberus_page_table* pt, const void* q, int64_t q_row_stride, void* out,
                             int64_t out_row_stride, int32_t batch, int32_t n_heads, float scale, const int32_t* blocks, int32_t n_select,
                             void* workspace, size_t workspace_bytes, void* stream) {
  TRY(check_pages(pg));
  TRY(check_page_table(pt, batch));
  TRY(check_same_pages(pg, pt));
  TRY(check_heads(pg, n_heads));
  if (blocks ? n_select < 1 : n_select != 0) return set_error(CERBERUS_ERR_ARG, "blocks and n_select go together");
  // (the kernel's scores are in powers of two: with a factor that is infinite there, scores of zero would be NaN)
  if (!std::isfinite(scale * 1.44269504088896340736f)) return set_error(CERBERUS_ERR_ARG, "scale must be finite, and scale / ln 2 too");
  TRY(check_rows(pg, q, q_row_stride, "q"));
  TRY(check_rows(pg, out, out_row_stride, "out"));
  TRY(check_workspace(pg, pt, batch, n_heads, n_select, workspace, workspace_bytes));
  const PagedWorkspace w = paged_workspace(*pg, *pt, batch, n_heads, n_select, workspace);
  PagedAttnArgs a{};
  a.pg = *pg; a.table = pt->block_table; a.lens = pt->kv_len; a.max_blocks = pt->max_blocks; a.page_shift = page_shift_of(pg->page_size);
  a.q = q; a.q_row = q_row_stride; a.out = out; a.out_row = out_row_stride; a.batch = batch; a.n_heads = n_heads; a.scale = scale;
  a.blocks = blocks; a.n_select = n_select; a.part = w.part; a.status = pt->status;
  HIP_TRY(launch_paged_attention(a, pg->dtype, reinterpret_cast<hipStream_t>(stream)));
  return CERBERUS_OK;
}

}  // extern "C"

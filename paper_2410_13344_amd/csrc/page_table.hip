// Pages of a key-value cache: which rows go where (k_page_plan, k_page_slots) and putting them there (k_page_store).
#include "paged.h"

#include <limits.h>

#include <algorithm>

namespace cerb {

namespace {

constexpr int kPlanThreads = 1024;   // a thread per sequence
static_assert(kPlanThreads == CERBERUS_MAX_SEQS, "k_page_plan has a thread per sequence");

// inclusive sum over the workgroup's threads in order; sh holds an entry per wave
__device__ __forceinline__ long long scan_sum(long long v, long long* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const long long o = __shfl_up(v, off, 64);
    if (lane >= off) v += o;
  }
  __syncthreads();                       // an earlier scan's entries have been read
  if (lane == 63) sh[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += sh[w];
  return v;
}

// first of n ascending sums that is above i (n where none is)
__device__ __forceinline__ int owner_of(const long long* ends, int n, long long i) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (ends[mid] > i) hi = mid; else lo = mid + 1;
  }
  return lo;
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Plan of a batch: lengths, block tables and free pages (see cerberus_page_plan), and the slots of up to
// kSlotsInPlan rows.  All of it follows from three running sums over the sequences, in their order: pages that come back,
// rows, pages that are needed.  Sequence b is granted its pages if it fits and needs none or the running sum of needs up
// to it is no more than the free pages; needs only grow along the sum, so the granted ones that need pages come before all
// refused ones that do, and their places on the stack of free pages are that same sum.  Pages and rows are dealt to
// threads one by one, whoever owns them (a search in the sums), not sequence by sequence: a prompt of thousands
// of blocks next to sequences that need none would otherwise be one thread's loop.
// One workgroup; its time is the chain of loads and barriers.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(kPlanThreads) void k_page_plan(const cerberus_page_table pt, const int* new_rows, int most, int batch,
                                                            int max_rows, int* row_start, int* first_pos, int* slot, int with_slots) {
  __shared__ long long sh[kPlanThreads / 64];
  __shared__ long long back_end[kPlanThreads], row_end[kPlanThreads], need_end[kPlanThreads];
  __shared__ int old_len[kPlanThreads], s_first[kPlanThreads];
  __shared__ long long s_grant;
  const int t = threadIdx.x, ps = pt.page_size;
  const long long cap = (long long)pt.max_blocks * ps;
  int L = 0, n = 0;
  if (t < batch) { L = pt.kv_len[t]; n = min(new_rows ? new_rows[t] : 1, most); }
  const int nf0 = min(max(*pt.n_free, 0), pt.n_pages);
  const bool sane = L >= 0 && L <= cap, ends = n < 0;
  const int held = sane ? (int)(((long long)L + ps - 1) / ps) : 0;
  const int rows = max(n, 0);

  const long long be = scan_sum(ends ? held : 0, sh), re = scan_sum(rows, sh);
  back_end[t] = be;
  row_end[t] = re;
  old_len[t] = L;
  if (t == 0) s_grant = 0;
  const bool fits = t < batch && !ends && sane && (long long)L + rows <= cap && re <= max_rows;
  const int total = fits ? (int)(((long long)L + rows + ps - 1) / ps) : held;
  const int need = fits ? total - held : 0;
  const long long ne = scan_sum(need, sh);
  need_end[t] = ne;
  __syncthreads();
  const long long returned = back_end[kPlanThreads - 1];
  const int nf1 = (int)min((long long)pt.n_pages, nf0 + returned);
  const bool granted = fits && (need == 0 || ne <= nf1);
  s_first[t] = granted ? L : -1;
  if (granted && need > 0) atomicMax(&s_grant, ne);

  // pages of the sequences that end, on top of the free ones in order of the sequences
  for (long long i = t; i < returned; i += kPlanThreads) {
    const int b = owner_of(back_end, batch, i);
    const long long j = i - (b ? back_end[b - 1] : 0);
    if (nf0 + i < pt.n_pages) pt.free_pages[nf0 + i] = pt.block_table[(size_t)b * pt.max_blocks + j];
  }
  __syncthreads();                         // (also: those pages are written before they are taken below)
  const long long grant = s_grant;
  for (long long i = t; i < grant; i += kPlanThreads) {
    const int b = owner_of(need_end, batch, i);
    const int l = old_len[b];
    const long long j = i - (b ? need_end[b - 1] : 0) + ((long long)l + ps - 1) / ps;
    pt.block_table[(size_t)b * pt.max_blocks + j] = pt.free_pages[nf1 - 1 - i];
  }
  if (t < batch) {
    if (ends || (granted && rows)) pt.kv_len[t] = ends ? 0 : L + rows;
    first_pos[t] = granted ? L : -1;
    row_start[t + 1] = (int)min(re, (long long)INT_MAX);
    if (!ends && !granted) atomicOr(pt.status, (int)CERBERUS_DEV_KV_OVERFLOW);
  }
  if (t == 0) {
    row_start[0] = 0;
    *pt.n_free = nf1 - (int)grant;
  }
  if (!with_slots) return;
  __syncthreads();                         // the tables are whole
  for (int i = t; i < max_rows; i += kPlanThreads) {
    const int b = owner_of(row_end, batch, i);
    int v = -1;
    if (b < batch && s_first[b] >= 0) {
      const int pos = s_first[b] + (int)(i - (b ? row_end[b - 1] : 0));
      v = pt.block_table[(size_t)b * pt.max_blocks + pos / ps] * ps + pos % ps;
    }
    slot[i] = v;
  }
}

// Slots of many rows, from what the plan left: a thread per row.
__global__ __launch_bounds__(256) void k_page_slots(const cerberus_page_table pt, int batch, int max_rows, const int* __restrict__ row_start,
                                                    const int* __restrict__ first_pos, int* __restrict__ slot) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= max_rows) return;
  int lo = 0, hi = batch;                  // first sequence whose rows end above i
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (row_start[mid + 1] > i) hi = mid; else lo = mid + 1;
  }
  int v = -1;
  if (lo < batch && first_pos[lo] >= 0) {
    const int pos = first_pos[lo] + i - row_start[lo];
    v = pt.block_table[(size_t)lo * pt.max_blocks + pos / pt.page_size] * pt.page_size + pos % pt.page_size;
  }
  slot[i] = v;
}

constexpr int kSlotsInPlan = 4096;

hipError_t launch_page_plan(const cerberus_page_table& pt, const int* new_rows, int most, int batch, int max_rows, int* row_start,
                            int* first_pos, int* slot, hipStream_t s) {
  const int with = max_rows <= kSlotsInPlan;
  hipLaunchKernelGGL(k_page_plan, dim3(1), dim3(kPlanThreads), 0, s, pt, new_rows, most, batch, max_rows, row_start, first_pos, slot, with);
  if (!with)
    hipLaunchKernelGGL(k_page_slots, dim3((max_rows + 255) / 256), dim3(256), 0, s, pt, batch, max_rows, row_start, first_pos, slot);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Store of rows, and bounds of the pages they go to.  Rows that follow each other into one page are a run; the workgroup
// that has a run's first row among its `chunk` rows takes the whole run for one key head: copies its K and V rows, folds
// its keys and those that the page held before into the lowest and highest coordinate, and writes these once.  Nothing is
// accumulated over calls, so a page that another sequence had before needs no clearing, and the order of workgroups does
// not matter.  A row is dh * sizeof(T) / 16 lanes of 16 bytes; the workgroup's groups of so many lanes take rows in turn.
// ---------------------------------------------------------------------------------------------
namespace {
template <typename T> struct Vec16;   // 16 bytes as numbers
template <> struct Vec16<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Vec16<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 put(const float (&f)[8]) {   // (values that are bf16 already: no rounding)
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(f[2 * i]) >> 16) | (__float_as_uint(f[2 * i + 1]) & 0xffff0000u);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
// the lower / higher of two, NaN if either is
__device__ __forceinline__ float lower(float a, float b) { return (a < b || a != a) ? a : b; }
__device__ __forceinline__ float higher(float a, float b) { return (a > b || a != a) ? a : b; }
}  // namespace

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_store(const PageStoreArgs a, int chunk) {
  constexpr int N = Vec16<T>::N, LPR = DH / N, ROWS = 256 / LPR;   // lanes per row, rows side by side
  __shared__ float sh[2][4][DH];
  const int h = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int sub = threadIdx.x / LPR, piece = threadIdx.x % LPR;
  const int ps = a.pg.page_size, r_end = (int)min((long long)a.n_rows, (blockIdx.x + 1ll) * chunk);
  const long long slots = (long long)a.pg.n_pages * ps;
  const T* k = reinterpret_cast<const T*>(a.k) + h * a.k_head + piece * N;
  const T* v = reinterpret_cast<const T*>(a.v) + h * a.v_head + piece * N;
  T* kp = reinterpret_cast<T*>(a.pg.k) + piece * N;
  T* vp = reinterpret_cast<T*>(a.pg.v) + piece * N;

  for (int r = blockIdx.x * chunk; r < r_end;) {
    const int s0 = a.slot[r];
    if (s0 < 0 || s0 >= slots) {                                   // (uniform over the workgroup, like all below)
      if (s0 >= 0 && h == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, (int)CERBERUS_DEV_BAD_PAGE);
      ++r;
      continue;
    }
    const int off0 = s0 & (ps - 1);
    // rows from here on that follow each other in this page
    int len = 1;
    const int most = min(ps - off0, a.n_rows - r);
    for (int i = 1; i < most; i += 64) {
      const bool next = i + lane < most && a.slot[r + i + lane] == s0 + i + lane;
      const unsigned long long m = __ballot(next);
      if (m != ~0ull) { len += __ffsll((long long)~m) - 1; break; }
      len += 64;
    }
    len = min(len, most);
    if (off0 != 0 && r > 0 && r == (int)blockIdx.x * chunk && a.slot[r - 1] == s0 - 1) {   // the run began in the chunk before
      r += len;
      continue;
    }
    const size_t row0 = ((size_t)(s0 >> a.page_shift) * a.pg.n_kv_heads + h) * ps;     // the page's rows of this head
    float lo[N], hi[N];
#pragma unroll
    for (int e = 0; e < N; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
    auto fold = [&](const uint4& u) {
      float f[N];
      Vec16<T>::get(u, f);
#pragma unroll
      for (int e = 0; e < N; ++e) { lo[e] = lower(f[e], lo[e]); hi[e] = higher(f[e], hi[e]); }
    };
    for (int i = sub; i < len; i += ROWS) {
      const uint4 ku = *reinterpret_cast<const uint4*>(k + (long long)(r + i) * a.k_row);
      const uint4 vu = *reinterpret_cast<const uint4*>(v + (long long)(r + i) * a.v_row);
      *reinterpret_cast<uint4*>(kp + (row0 + off0 + i) * DH) = ku;
      *reinterpret_cast<uint4*>(vp + (row0 + off0 + i) * DH) = vu;
      fold(ku);
    }
    if (a.pg.bounds) {
      for (int i = sub; i < off0; i += ROWS) fold(*reinterpret_cast<const uint4*>(kp + (row0 + i) * DH));
#pragma unroll
      for (int off = LPR; off < 64; off <<= 1)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          lo[e] = lower(__shfl_xor(lo[e], off, 64), lo[e]);
          hi[e] = higher(__shfl_xor(hi[e], off, 64), hi[e]);
        }
      __syncthreads();                                             // an earlier run's entries have been read
      if (lane < LPR) {
#pragma unroll
        for (int e = 0; e < N; ++e) { sh[0][wave][piece * N + e] = lo[e]; sh[1][wave][piece * N + e] = hi[e]; }
      }
      __syncthreads();
      if (threadIdx.x < 2 * LPR) {
        const int side = threadIdx.x / LPR;
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          f[e] = sh[side][0][piece * N + e];
#pragma unroll
          for (int w = 1; w < 4; ++w) f[e] = side ? higher(sh[1][w][piece * N + e], f[e]) : lower(sh[0][w][piece * N + e], f[e]);
        }
        T* b = reinterpret_cast<T*>(a.pg.bounds) + ((((size_t)(s0 >> a.page_shift) * a.pg.n_kv_heads + h) * 2 + side) * DH) + piece * N;
        *reinterpret_cast<uint4*>(b) = Vec16<T>::put(f);
      }
    }
    r += len;
  }
}

constexpr int kStoreWorkgroups = 2048;

hipError_t launch_page_store(const PageStoreArgs& a, hipStream_t s) {
  // Workgroups for the whole card before any takes several runs: a row each while there are few (a decoding step's rows are
  // runs of one), up to about a page of rows for prompts, whose runs are pages; never more than 2^20 along the rows.
  const long long work = (long long)a.n_rows * a.pg.n_kv_heads;
  int chunk = (int)std::min<long long>(std::max<long long>(1, work / kStoreWorkgroups), a.pg.page_size);
  chunk = std::max(chunk, (a.n_rows - 1) / (1 << 20) + 1);
  dim3 grid((a.n_rows + chunk - 1) / chunk, a.pg.n_kv_heads);
  const bool wide = a.pg.head_dim == 128;
  if (a.pg.dtype == CERBERUS_F32) {
    if (wide) hipLaunchKernelGGL((k_page_store<float, 128>), grid, dim3(256), 0, s, a, chunk);
    else hipLaunchKernelGGL((k_page_store<float, 64>), grid, dim3(256), 0, s, a, chunk);
  } else {
    if (wide) hipLaunchKernelGGL((k_page_store<bf16_t, 128>), grid, dim3(256), 0, s, a, chunk);
    else hipLaunchKernelGGL((k_page_store<bf16_t, 64>), grid, dim3(256), 0, s, a, chunk);
  }
  return hipGetLastError();
}

}  // namespace cerb

// Pages of a key-value cache: which rows go where (k_page_plan, k_page_slots) and putting them there (k_page_store).
#include "paged.h"

#include <limits.h>

#include <algorithm>

namespace cerb {

namespace {

constexpr int kPlanThreads = 1024;   // a thread per sequence
static_assert(kPlanThreads == CERBERUS_MAX_SEQS, "k_page_plan has a thread per sequence");

// inclusive sum over the workgroup's threads in order; sh holds an entry per wave and belongs to this sum alone
__device__ __forceinline__ long long scan_sum(long long v, long long* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) sh[wave] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) v += w < wave ? sh[w] : 0;
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
// Plan of a batch: lengths, block tables, free pages and slots (see cerberus_page_plan).  All of it follows from three running
// sums over the sequences, in their order: pages that come back, rows, pages that are needed.  Sequence b is granted
// its pages if it fits and needs none or the running sum of needs up to it is no more than the free pages; needs only grow
// along the sum, so the granted ones that need pages come before all refused ones that do, and their places on the
// stack of free pages are that same sum.  Pages and rows are dealt to threads one by one, whoever owns them (a search in
// the sums), not sequence by sequence: a prompt of thousands of blocks next to sequences that need none would otherwise be one thread's loop.
// What is on place p of the stack is known without waiting for the pages that come back to be written there: from place nf0 on
// it is a block of a sequence that ends.  So moving pages and forming slots only read what was there before the call
// (free pages below nf0, blocks held, tables of sequences that end) and write other places.
// A step's few rows take one workgroup and one launch (ALL; 4 us, a chain of loads and barriers); with a prompt's rows
// many workgroups form the sums each for itself and share the pages and rows, and k_page_commit then writes what they read.
// 256 requests with 73600 pages and rows to move and form: 7 us + 2 for the commit; one workgroup and a launch for the slots took 21.
// ---------------------------------------------------------------------------------------------
template <bool ALL>
__global__ __launch_bounds__(kPlanThreads) void k_page_plan(const cerberus_page_table pt, const int* new_rows, int most, int batch,
                                                            int max_rows, int* row_start, int* first_pos, int* slot) {
  __shared__ long long sh[3][kPlanThreads / 64];
  __shared__ long long back_end[kPlanThreads], row_end[kPlanThreads], need_end[kPlanThreads];
  __shared__ int old_len[kPlanThreads], s_first[kPlanThreads];
  __shared__ long long s_grant;
  const int t = threadIdx.x, ps = pt.page_size, shift = 31 - __clz(ps);    // (a power of two)
  const long long cap = (long long)pt.max_blocks * ps;
  int L = 0, n = 0;
  if (t < batch) { L = pt.kv_len[t]; n = min(new_rows ? new_rows[t] : 1, most); }
  const int nf0 = min(max(*pt.n_free, 0), pt.n_pages);
  const bool sane = L >= 0 && L <= cap, ends = n < 0;
  const int held = sane ? (int)(((long long)L + ps - 1) >> shift) : 0;
  const int rows = max(n, 0);
  if (t == 0) s_grant = 0;

  const long long be = scan_sum(ends ? held : 0, sh[0]), re = scan_sum(rows, sh[1]);
  back_end[t] = be;
  row_end[t] = re;
  old_len[t] = L;
  const bool fits = t < batch && !ends && sane && (long long)L + rows <= cap && re <= max_rows;
  const int total = fits ? (int)(((long long)L + rows + ps - 1) >> shift) : held;
  const int need = fits ? total - held : 0;
  const long long ne = scan_sum(need, sh[2]);
  need_end[t] = ne;
  __syncthreads();
  const long long returned = back_end[kPlanThreads - 1];
  const int nf1 = (int)min((long long)pt.n_pages, nf0 + returned);
  const bool granted = fits && (need == 0 || ne <= nf1);
  s_first[t] = granted ? L : -1;
  if (granted && need > 0) atomicMax(&s_grant, ne);
  __syncthreads();
  const long long grant = s_grant;

  // what is on place p of the stack of free pages once the pages that come back are on it
  auto on_stack = [&](long long p) {
    if (p < nf0) return pt.free_pages[p];
    const int b = owner_of(back_end, batch, p - nf0);
    return pt.block_table[(size_t)b * pt.max_blocks + (p - nf0 - (b ? back_end[b - 1] : 0))];
  };
  // One list of all that is to be moved or formed, so that a thread's few turns are one after the other in any of the three kinds.
  const long long n_back = nf1 - nf0, n_all = n_back + grant + max_rows, step = (long long)gridDim.x * kPlanThreads;
  for (long long item = (long long)blockIdx.x * kPlanThreads + t; item < n_all; item += step) {
    if (item < n_back) {                       // a page that comes back (one that is taken again at once keeps its place behind the list's end)
      pt.free_pages[nf0 + item] = on_stack(nf0 + item);
    } else if (item < n_back + grant) {        // a page for a block
      const long long i = item - n_back;
      const int b = owner_of(need_end, batch, i);
      const long long j = i - (b ? need_end[b - 1] : 0) + (((long long)old_len[b] + ps - 1) >> shift);
      pt.block_table[(size_t)b * pt.max_blocks + j] = on_stack(nf1 - 1 - i);
    } else {                                   // a row's slot
      const long long i = item - n_back - grant;
      const int b = owner_of(row_end, batch, i);
      int v = -1;
      if (b < batch && s_first[b] >= 0) {
        const int pos = s_first[b] + (int)(i - (b ? row_end[b - 1] : 0)), blk = pos >> shift;
        const int have = (int)(((long long)old_len[b] + ps - 1) >> shift);
        const int page = blk < have ? pt.block_table[(size_t)b * pt.max_blocks + blk] : on_stack(nf1 - 1 - ((b ? need_end[b - 1] : 0) + blk - have));
        // (A page number that no pool has is not made a slot: in 32 bits its rows can be those of another sequence's page.)
        if (page >= 0 && page < pt.n_pages) v = page * ps + (pos & (ps - 1));
        else atomicOr(pt.status, (int)CERBERUS_DEV_BAD_PAGE);
      }
      slot[i] = v;
    }
  }
  if (blockIdx.x != 0) return;
  if (t < batch) {
    first_pos[t] = granted ? L : -1;
    row_start[t + 1] = (int)min(re, (long long)INT_MAX);
    if (!ends && !granted) atomicOr(pt.status, (int)CERBERUS_DEV_KV_OVERFLOW);
    if (ALL && (ends || (granted && rows))) pt.kv_len[t] = ends ? 0 : L + rows;   // (everybody has read it)
  }
  if (t == 0) {
    row_start[0] = 0;
    if (ALL) *pt.n_free = nf1 - (int)grant;
  }
}

// Lengths and free pages after a plan of many workgroups.
__global__ __launch_bounds__(kPlanThreads) void k_page_commit(const cerberus_page_table pt, const int* __restrict__ new_rows, int most, int batch,
                                                              const int* __restrict__ first_pos) {
  __shared__ long long sh[2][kPlanThreads / 64];
  const int t = threadIdx.x, ps = pt.page_size, shift = 31 - __clz(ps);    // (a power of two)
  const long long cap = (long long)pt.max_blocks * ps;
  const int nf0 = min(max(*pt.n_free, 0), pt.n_pages);
  long long back = 0, taken = 0;
  if (t < batch) {
    const int L = pt.kv_len[t], n = min(new_rows ? new_rows[t] : 1, most);
    if (n < 0) {
      back = L >= 0 && L <= cap ? ((long long)L + ps - 1) >> shift : 0;
      pt.kv_len[t] = 0;
    } else if (n > 0 && first_pos[t] >= 0) {
      taken = (((long long)L + n + ps - 1) >> shift) - (((long long)L + ps - 1) >> shift);
      pt.kv_len[t] = L + n;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) { back += __shfl_xor(back, off, 64); taken += __shfl_xor(taken, off, 64); }
  if ((t & 63) == 0) { sh[0][t >> 6] = back; sh[1][t >> 6] = taken; }
  __syncthreads();
  if (t != 0) return;
  back = taken = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) { back += sh[0][w]; taken += sh[1][w]; }
  *pt.n_free = (int)(min((long long)pt.n_pages, nf0 + back) - taken);
}

// us, one workgroup / many, for plans of 16, 1024, 2048, 4096 and 8192 rows: of one prompt 3.5 / 6.6, 4.3 / 6.6, 4.7 / 6.9, 5.7 / 6.9, 8.0 / 6.9; of 256
// sequences 6.3 / 8.8, 8.1 / 9.8, 9.0 / 10.0, 10.8 / 10.1, 15.0 / 10.1.  (What comes back from sequences that end is not in the rule: 1024 of 512 pages each
// take one workgroup 0.53 ms.)
constexpr int kRowsOfOne = 2048, kPlanWorkgroups = 128;

hipError_t launch_page_plan(const cerberus_page_table& pt, const int* new_rows, int most, int batch, int max_rows, int* row_start,
                            int* first_pos, int* slot, hipStream_t s) {
  if (max_rows <= kRowsOfOne) {
    hipLaunchKernelGGL(k_page_plan<true>, dim3(1), dim3(kPlanThreads), 0, s, pt, new_rows, most, batch, max_rows, row_start, first_pos, slot);
  } else {
    hipLaunchKernelGGL(k_page_plan<false>, dim3(kPlanWorkgroups), dim3(kPlanThreads), 0, s, pt, new_rows, most, batch, max_rows, row_start, first_pos, slot);
    hipLaunchKernelGGL(k_page_commit, dim3(1), dim3(kPlanThreads), 0, s, pt, new_rows, most, batch, first_pos);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Store of rows, and bounds of the pages they go to.  Rows that follow each other into one page are a run; the workgroup
// that has a run's first row among its `chunk` rows takes the whole run for one key head: copies its K and V rows, folds
// its keys and those that the page held before into the lowest and highest coordinate, and writes these once.  Nothing is
// accumulated over calls, so a page that another sequence had before needs no clearing, and the order of workgroups does
// not matter.  Heads vary fastest over the workgroups, so that neighbours read what lies together in the rows; pages are written
// past the caches, which they would only pass through before they are read again (14154 rows of 8 heads: 35 us
// with plain stores and rows fastest, 28 with these stores, 26 with both; 23 is a copy of the same bytes).  A row is
// dh * sizeof(T) / 16 lanes of 16 bytes; the workgroup's groups of so many lanes take rows in turn.  A decoding step's 16 rows of 32
// heads take 6 us: slots, rows of the page so far, the fold and the stores, one after the other.
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

// Lowest and highest coordinates of a page's keys, by a workgroup of 256: a lane folds pieces (16 bytes, always of the same columns)
// of the rows it sees, then the lanes and the four waves join.
template <typename T, int DH>
struct PageFold {
  static constexpr int N = Vec16<T>::N, LPR = DH / N;                // lanes per row
  float lo[N], hi[N];
  __device__ __forceinline__ PageFold() {
#pragma unroll
    for (int e = 0; e < N; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  }
  __device__ __forceinline__ void add(const uint4& u) {
    float f[N];
    Vec16<T>::get(u, f);
#pragma unroll
    for (int e = 0; e < N; ++e) { lo[e] = lower(f[e], lo[e]); hi[e] = higher(f[e], hi[e]); }
  }
  // to the page's two rows of bounds; sh may still be read by others when this begins
  __device__ __forceinline__ void write(T* bounds, float (&sh)[2][4][DH]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = threadIdx.x % LPR;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        lo[e] = lower(__shfl_xor(lo[e], off, 64), lo[e]);
        hi[e] = higher(__shfl_xor(hi[e], off, 64), hi[e]);
      }
    __syncthreads();
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
      *reinterpret_cast<uint4*>(bounds + side * DH + piece * N) = Vec16<T>::put(f);
    }
  }
};

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_store(const PageStoreArgs a, int chunk) {
  constexpr int N = Vec16<T>::N, LPR = DH / N, ROWS = 256 / LPR;   // lanes per row, rows side by side
  __shared__ float sh[2][4][DH];
  const int h = blockIdx.x, lane = threadIdx.x & 63;
  const int sub = threadIdx.x / LPR, piece = threadIdx.x % LPR;
  const int ps = a.pg.page_size, r_end = (int)min((long long)a.n_rows, (blockIdx.y + 1ll) * chunk);
  const long long slots = (long long)a.pg.n_pages * ps;
  const T* k = reinterpret_cast<const T*>(a.k) + h * a.k_head + piece * N;
  const T* v = reinterpret_cast<const T*>(a.v) + h * a.v_head + piece * N;
  T* kp = reinterpret_cast<T*>(a.pg.k) + piece * N;
  T* vp = reinterpret_cast<T*>(a.pg.v) + piece * N;

  const int begin = blockIdx.y * chunk;
  for (int r = begin; r < r_end;) {
    // the slots from here on, one lane each, that of the row before the chunk, and the first row itself (whatever its slot)
    const int ahead = r + lane < a.n_rows ? a.slot[r + lane] : -1;
    const int before = r == begin && r > 0 ? a.slot[r - 1] : -1;
    uint4 k0 = make_uint4(0, 0, 0, 0), v0 = k0;
    if (sub == 0) {
      k0 = *reinterpret_cast<const uint4*>(k + (long long)r * a.k_row);
      v0 = *reinterpret_cast<const uint4*>(v + (long long)r * a.v_row);
    }
    const int s0 = __builtin_amdgcn_readfirstlane(ahead);
    if (s0 < 0 || s0 >= slots) {                                   // (uniform over the workgroup, like all below)
      if (s0 >= 0 && h == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, (int)CERBERUS_DEV_BAD_PAGE);
      ++r;
      continue;
    }
    const int off0 = s0 & (ps - 1);
    // rows from here on that follow each other in this page
    const int most = min(ps - off0, a.n_rows - r);
    unsigned long long gap = ~__ballot(ahead == s0 + lane);
    int len = gap ? __ffsll((long long)gap) - 1 : 64;
    while (gap == 0 && len < most) {
      gap = ~__ballot(len + lane < most && a.slot[r + len + lane] == s0 + len + lane);
      len += gap ? __ffsll((long long)gap) - 1 : 64;
    }
    len = min(len, most);
    if (off0 != 0 && before == s0 - 1) {                           // the run began in the chunk before
      r += len;
      continue;
    }
    const size_t row0 = ((size_t)(s0 >> a.page_shift) * a.pg.n_kv_heads + h) * ps;     // the page's rows of this head
    PageFold<T, DH> fold;
    for (int i = sub; i < len; i += ROWS) {
      uint4 ku = k0, vu = v0;
      if (i > 0) {
        ku = *reinterpret_cast<const uint4*>(k + (long long)(r + i) * a.k_row);
        vu = *reinterpret_cast<const uint4*>(v + (long long)(r + i) * a.v_row);
      }
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, ku), reinterpret_cast<u32x4_t*>(kp + (row0 + off0 + i) * DH));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, vu), reinterpret_cast<u32x4_t*>(vp + (row0 + off0 + i) * DH));
      fold.add(ku);
    }
    if (a.pg.bounds) {
      for (int i = sub; i < off0; i += ROWS) fold.add(*reinterpret_cast<const uint4*>(kp + (row0 + i) * DH));
      fold.write(reinterpret_cast<T*>(a.pg.bounds) + ((size_t)(s0 >> a.page_shift) * a.pg.n_kv_heads + h) * 2 * DH, sh);
    }
    r += len;
  }
}

constexpr int kStoreWorkgroups = 2048;

hipError_t launch_page_store(const PageStoreArgs& a, hipStream_t s) {
  // Workgroups for the whole card before any takes several runs: a row each while there are few (a decoding step's rows are
  // runs of one), up to about a page of rows for prompts, whose runs are pages; never more than a grid has along the rows.
  const long long work = (long long)a.n_rows * a.pg.n_kv_heads;
  int chunk = (int)std::min<long long>(std::max<long long>(1, work / kStoreWorkgroups), a.pg.page_size);
  chunk = std::max(chunk, (a.n_rows - 1) / 65535 + 1);
  dim3 grid(a.pg.n_kv_heads, (a.n_rows - 1) / chunk + 1);
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

// ---------------------------------------------------------------------------------------------
// Bounds after a decoding step, whose rows the projections have written into the pages themselves.  A page that is not full is its sequence's
// newest, which every choice of blocks takes whatever it scores; so its bounds are formed once, when its last row is there, in one launch
// for all layers at the end of the step.  16 sequences fill a page every page_size / 16 steps; else the launch finds nothing to do.
// ---------------------------------------------------------------------------------------------
namespace {
constexpr int kBoundsLayers = 64;    // of a launch
struct PageBoundsArgs {
  const void* k[kBoundsLayers];
  void* bounds[kBoundsLayers];
  const int* slot;
  int n_kv_heads, page_shift;
};
}  // namespace

template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_bounds(const PageBoundsArgs a) {
  constexpr int N = Vec16<T>::N, LPR = DH / N, ROWS = 256 / LPR;
  __shared__ float sh[2][4][DH];
  const int h = blockIdx.x, l = blockIdx.z, s = a.slot[blockIdx.y], ps = 1 << a.page_shift;
  if (s < 0 || (s & (ps - 1)) != ps - 1 || !a.bounds[l]) return;
  const size_t head = (size_t)(s >> a.page_shift) * a.n_kv_heads + h;
  const T* rows = reinterpret_cast<const T*>(a.k[l]) + head * ps * DH + (threadIdx.x % LPR) * N;
  PageFold<T, DH> fold;
  for (int i = threadIdx.x / LPR; i < ps; i += ROWS) fold.add(*reinterpret_cast<const uint4*>(rows + (size_t)i * DH));
  fold.write(reinterpret_cast<T*>(a.bounds[l]) + head * 2 * DH, sh);
}

hipError_t launch_page_bounds(const cerberus_pages* layers, int n_layers, const int* slot, int batch, hipStream_t s) {
  for (int l0 = 0; l0 < n_layers; l0 += kBoundsLayers) {
    const int n = std::min(kBoundsLayers, n_layers - l0);
    PageBoundsArgs a{};
    bool any = false;
    for (int l = 0; l < n; ++l) {
      a.k[l] = layers[l0 + l].k;
      a.bounds[l] = layers[l0 + l].bounds;
      any = any || a.bounds[l];
    }
    if (!any) continue;
    a.slot = slot;
    a.n_kv_heads = layers->n_kv_heads;
    a.page_shift = page_shift_of(layers->page_size);
    const dim3 grid(layers->n_kv_heads, batch, n);
    const bool wide = layers->head_dim == 128;
    if (layers->dtype == CERBERUS_F32) {
      if (wide) hipLaunchKernelGGL((k_page_bounds<float, 128>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((k_page_bounds<float, 64>), grid, dim3(256), 0, s, a);
    } else {
      if (wide) hipLaunchKernelGGL((k_page_bounds<bf16_t, 128>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((k_page_bounds<bf16_t, 64>), grid, dim3(256), 0, s, a);
    }
  }
  return hipGetLastError();
}

}  // namespace cerb

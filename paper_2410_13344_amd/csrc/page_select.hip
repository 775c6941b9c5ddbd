// Choice of the blocks that a query attends to, by a bound on its scores.
#include "paged.h"

namespace cerb {

namespace {

// Order of a score as an unsigned number: higher score, higher number; NaN counts as +inf, both zeros alike.  The two
// highest numbers are left for the newest and the first block.
__device__ __forceinline__ unsigned long long order_of(double s) {
  if (s != s) s = INFINITY;
  const long long b = __double_as_longlong(s + 0.0);
  return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | (1ull << 63);
}
constexpr unsigned long long kNewest = ~0ull, kFirst = ~0ull - 1;

template <typename T> struct Piece;      // 16 bytes of bounds as numbers, those a mask leaves out as zero
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const uint4& u, int e, uint32_t keep) { return __uint_as_float((&u.x)[e] & keep); }
};
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const uint4& u, int e, uint32_t keep) {
    const uint32_t w = (&u.x)[e / 2];
    return __uint_as_float((e & 1 ? w & 0xffff0000u : w << 16) & keep);
  }
};

}  // namespace

// ---------------------------------------------------------------------------------------------
// Scores.  With Q the sum of a key head's queries, the block's score is the sum over d of Q_d times the higher bound where Q_d >= 0 and the
// lower one elsewhere.  Two blocks next to the border of the choice change places with the last bits of a
// sum, so products and sums are in 64 bits, where the products of 16- or 24-bit numbers are exact.  A wave takes 64
// blocks of one key head.  A block's bounds (both sides, 2 DH numbers in one piece of memory) are 16 bytes for each of LPB
// lanes; a lane's side and columns are the same for every block, so it holds its queries' sums, zero where the other
// side counts, and a mask that takes the bound out as well (an infinite bound that does not count is not a NaN).  Eight loads are in flight; their
// sums over the lanes are folded together, eight values over 2, 4, 8 lanes, then one.
// Bound by the bytes of the bounds.
// ---------------------------------------------------------------------------------------------
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_scores(const PageSelectArgs a) {
  constexpr int N = Piece<T>::N, LPB = 2 * DH / N, BPL = 64 / LPB;     // lanes per block, blocks per load of the wave
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, ps = a.pg.page_size, nkv = a.pg.n_kv_heads;
  const int h = blockIdx.y, b = blockIdx.z, group = a.n_heads / nkv;
  const int L = min(max(a.lens[b], 0), a.max_blocks << a.page_shift), held = (int)(((long long)L + ps - 1) >> a.page_shift);
  if (held <= a.n_select) return;                                       // all are chosen
  const int sub = lane % LPB, side = sub / (LPB / 2), d0 = sub % (LPB / 2) * N;
  double q[N];
  uint32_t keep[N];
#pragma unroll
  for (int e = 0; e < N; ++e) q[e] = 0.0;
  for (int i = 0; i < group; ++i) {
    const T* qp = reinterpret_cast<const T*>(a.q) + b * a.q_row + (h * group + i) * DH + d0;
    const uint4 u = *reinterpret_cast<const uint4*>(qp);
#pragma unroll
    for (int e = 0; e < N; ++e) q[e] += (double)Piece<T>::get(u, e, ~0u);
    if (a.q_lo_off) {
      const uint4 w = *reinterpret_cast<const uint4*>(qp + a.q_lo_off);
#pragma unroll
      for (int e = 0; e < N; ++e) q[e] += (double)Piece<T>::get(w, e, ~0u);
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const bool counts = (q[e] >= 0.0) == (side == 1);
    keep[e] = counts ? ~0u : 0u;
    q[e] = counts ? q[e] : 0.0;
  }
  const T* bounds = reinterpret_cast<const T*>(a.pg.bounds) + (size_t)h * 2 * DH + sub * N;
  unsigned long long* keys = a.keys + ((size_t)b * nkv + h) * a.max_blocks;
  for (int j0 = (blockIdx.x * 4 + wave) * 64; j0 < held; j0 += gridDim.x * 256) {
    int page = -1;
    if (j0 + lane < held) page = a.table[(size_t)b * a.max_blocks + j0 + lane];
    if (page >= a.pg.n_pages) page = -1;
    for (int i0 = 0; i0 < 64 / BPL && j0 + i0 * BPL < held; i0 += 8) {
      double s[8];
      uint4 u[8];
      int pg[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        pg[i] = __shfl(page, (i0 + i) * BPL + lane / LPB, 64);          // (i0 + i < 64 / BPL: 8 divides it)
        u[i] = *reinterpret_cast<const uint4*>(bounds + (size_t)max(pg[i], 0) * nkv * 2 * DH);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i] = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) s[i] = fma(q[e], (double)Piece<T>::get(u[i], e, keep[e]), s[i]);
        if (pg[i] < 0) s[i] = 0.0;
      }
      // fold: lanes whose bit is set go on with the upper half of the values
#pragma unroll
      for (int n = 4, bit = LPB / 2; n >= 1; n >>= 1, bit >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const bool up = lane & bit;
          const double give = up ? s[i] : s[i + n], have = up ? s[i + n] : s[i];
          s[i] = have + __shfl_xor(give, bit, 64);
        }
#pragma unroll
      for (int bit = LPB / 16; bit >= 1; bit >>= 1) s[0] += __shfl_xor(s[0], bit, 64);
      if (sub % (LPB / 8) == 0) {
        const int j = j0 + (i0 + sub / (LPB / 8)) * BPL + lane / LPB;   // which of the eight: the lane's top three bits below LPB
        if (j < held) keys[j] = j == held - 1 ? kNewest : j == 0 ? kFirst : order_of(s[0]);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// The n_select highest of a list, in order of their places: a workgroup per (sequence, key head).  The lowest number that n_select or
// fewer reach is found bit by bit from the first bit in which the numbers differ; a count is a ballot per wave and
// one barrier, and the search ends as soon as exactly n_select reach it, for scores without ties after
// about log2 of the blocks' number of bits.  Ties that are left go to the lowest places.  A thread keeps its first kKept
// numbers in registers; longer lists are read again for every count.
// ---------------------------------------------------------------------------------------------
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_page_pick(const PageSelectArgs a) {
  constexpr int kKept = 8, WAVES = THREADS / 64;
  const int h = blockIdx.x, b = blockIdx.y, ps = a.pg.page_size, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int L = min(max(a.lens[b], 0), a.max_blocks << a.page_shift), held = (int)(((long long)L + ps - 1) >> a.page_shift);
  const int want = a.n_select;
  const size_t row = (size_t)b * a.pg.n_kv_heads + h;
  const unsigned long long* keys = a.keys + row * a.max_blocks;
  int* out = a.blocks + row * want;
  if (held <= want) {
    for (int j = threadIdx.x; j < want; j += THREADS) out[j] = j < held ? j : -1;
    return;
  }
  __shared__ unsigned long long s_or[WAVES], s_and[WAVES];
  __shared__ int s_n[2][WAVES], s_eq[2][WAVES];
  const int rounds = (held + THREADS - 1) / THREADS;
  unsigned long long kept[kKept];
#pragma unroll
  for (int i = 0; i < kKept; ++i) {
    const int j = i * THREADS + threadIdx.x;
    kept[i] = j < held ? keys[j] : 0;                                    // (no block's number is 0)
  }
  auto number = [&](int i) { const int j = i * THREADS + threadIdx.x; return j < held ? keys[j] : 0ull; };   // round i >= kKept
  // bits in which the numbers differ
  unsigned long long any = 0, all = ~0ull;
  auto fold = [&](unsigned long long v) { any |= v; all &= v ? v : ~0ull; };
#pragma unroll
  for (int i = 0; i < kKept; ++i) fold(kept[i]);
  for (int i = kKept; i < rounds; ++i) fold(number(i));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) { any |= __shfl_xor(any, off, 64); all &= __shfl_xor(all, off, 64); }
  if (lane == 0) { s_or[wave] = any; s_and[wave] = all; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { any |= s_or[w]; all &= s_and[w]; }
  int flip = 0;
  auto count = [&](unsigned long long least) {                           // numbers that reach `least`, over the workgroup
    int n = 0;
#pragma unroll
    for (int i = 0; i < kKept; ++i) n += __popcll(__ballot(kept[i] >= least));
    for (int i = kKept; i < rounds; ++i) n += __popcll(__ballot(number(i) >= least));
    if (lane == 0) s_n[flip][wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) n += s_n[flip][w];
    flip ^= 1;                                                           // (the next count writes the other entries: one barrier is enough)
    return n;
  };
  const int top = any == all ? -1 : 63 - __clzll((long long)(any ^ all));
  unsigned long long least = top < 0 ? all : top == 63 ? 0 : all >> (top + 1) << (top + 1);
  int n = held;                                                          // reach `least`
  for (int bit = top; bit >= 0 && n > want; --bit) {
    const int c = count(least | 1ull << bit);
    if (c >= want) { least |= 1ull << bit; n = c; }
  }
  // n > want: `least` itself is there several times, only the first of those go along
  const int ties = n > want ? want - (least == ~0ull ? 0 : count(least + 1)) : held;
  __syncthreads();
  int base = 0, base_eq = 0;
  for (int i = 0; i < rounds; ++i) {
    unsigned long long v = 0;
#pragma unroll
    for (int r = 0; r < kKept; ++r) v = i == r ? kept[r] : v;
    if (i >= kKept) v = number(i);
    const unsigned long long below = (1ull << lane) - 1, eq = __ballot(v == least);
    int place_eq = base_eq + __popcll(eq & below);
    if (lane == 0) s_eq[i & 1][wave] = __popcll(eq);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      place_eq += w < wave ? s_eq[i & 1][w] : 0;
      base_eq += s_eq[i & 1][w];
    }
    const bool take = v > least || (v == least && place_eq < ties);
    const unsigned long long m = __ballot(take);
    int place = base + __popcll(m & below);
    if (lane == 0) s_n[i & 1][wave] = __popcll(m);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      place += w < wave ? s_n[i & 1][w] : 0;
      base += s_n[i & 1][w];
    }
    if (take) out[place] = i * THREADS + threadIdx.x;
  }
}

size_t page_select_bytes(int batch, int n_kv_heads, int max_blocks) { return (size_t)batch * n_kv_heads * max_blocks * 8; }

hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t s) {
  dim3 grid(a.max_blocks < 1 << 20 ? (a.max_blocks + 255) / 256 : 1 << 12, a.pg.n_kv_heads, a.batch);
  const bool wide = a.pg.head_dim == 128;
  if (a.pg.dtype == CERBERUS_F32) {
    if (wide) hipLaunchKernelGGL((k_page_scores<float, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_scores<float, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((k_page_scores<bf16_t, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_scores<bf16_t, 64>), grid, dim3(256), 0, s, a);
  }
  if (a.max_blocks <= 2048) hipLaunchKernelGGL(k_page_pick<256>, dim3(a.pg.n_kv_heads, a.batch), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_page_pick<1024>, dim3(a.pg.n_kv_heads, a.batch), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace cerb

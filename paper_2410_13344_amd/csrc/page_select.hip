// Choice of the blocks that a query attends to, by a bound on its scores.
#include "paged.h"

#include <algorithm>

namespace cerb {

namespace {

constexpr unsigned long long kOutside = 1;   // number of a block whose page the pool does not have: below that of every score

// Order of a score as an unsigned number: higher score, higher number, none below 2; NaN counts as +inf, both zeros alike.
__device__ __forceinline__ unsigned long long order_of(double s) {
  if (s != s) s = INFINITY;
  const long long b = __double_as_longlong(s + 0.0);
  return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | (1ull << 63);
}

template <typename T> struct Piece;      // 16 bytes as numbers
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ float get(const uint4& u, int e) { return __uint_as_float((&u.x)[e]); }
};
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ float get(const uint4& u, int e) {
    const uint32_t w = (&u.x)[e / 2];
    return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
  }
};

}  // namespace

// ---------------------------------------------------------------------------------------------
// Scores.  With Q the sum of a key head's queries, the block's score is the sum over d of Q_d times the higher bound where Q_d >= 0
// and the lower one elsewhere.  Two blocks next to the border of the choice change places with the last bits of a sum, so
// products and sums are in 64 bits, where the products of 16- or 24-bit numbers are exact.  A wave takes 16, 32 or 64 blocks of one
// key head at a time.  Each of LPB lanes per block loads 16 bytes of both sides, the same columns for every block; a mask
// from its queries' signs takes one side's bits before anything is computed (an infinite bound that does not count is
// not a NaN).  Eight blocks per lane are in flight; their sums over the lanes are folded together, eight values over 2, 4, 8 lanes,
// then one.
// ---------------------------------------------------------------------------------------------
template <typename T, int DH>
struct Scores {
  static constexpr int N = Piece<T>::N, LPB = DH / N, BPL = 64 / LPB, AT_ONCE = 8 * BPL;   // lanes per block, blocks side by side
  double q[N];
  uint32_t high[4];          // bits of the 16 bytes that come from the higher bounds
  const T* bounds;
  size_t page_stride;
  int sub, held, n_pages;

  __device__ __forceinline__ void init(const PageSelectArgs& a, int b, int h, int held_) {
    const int lane = threadIdx.x & 63, nkv = a.pg.n_kv_heads, group = a.n_heads / nkv;
    sub = lane % LPB;
    held = held_;
    n_pages = a.pg.n_pages;
    page_stride = (size_t)nkv * 2 * DH;
    bounds = reinterpret_cast<const T*>(a.pg.bounds) + (size_t)h * 2 * DH + sub * N;
    const T* qp = reinterpret_cast<const T*>(a.q) + b * a.q_row + (size_t)h * group * DH + sub * N;
#pragma unroll
    for (int e = 0; e < N; ++e) q[e] = 0.0;
    for (int i0 = 0; i0 < group; i0 += 4) {                               // four loads in flight
      uint4 u[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = *reinterpret_cast<const uint4*>(qp + (size_t)min(i0 + i, group - 1) * DH);
        if (a.q_lo_off) w[i] = *reinterpret_cast<const uint4*>(qp + a.q_lo_off + (size_t)min(i0 + i, group - 1) * DH);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i0 + i < group) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            q[e] += (double)Piece<T>::get(u[i], e);
            if (a.q_lo_off) q[e] += (double)Piece<T>::get(w[i], e);
          }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) high[i] = 0;
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (q[e] >= 0.0) high[e * 4 / N] |= N == 4 ? ~0u : e & 1 ? 0xffff0000u : 0x0000ffffu;
  }

  // blocks j0 .. j0 + AT_ONCE - 1, `page` that of block j0 + lane: put(j, number) for each that is held
  template <typename Put>
  __device__ __forceinline__ void run(int j0, int page, Put put) const {
    const int lane = threadIdx.x & 63;
    double s[8];
    uint4 lo[8], hi[8];
    page = page < n_pages ? page : -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pg = max(__shfl(page, i * BPL + lane / LPB, 64), 0);       // (page 0 where there is none: what it gives is not used)
      const T* p = bounds + (size_t)pg * page_stride;
      lo[i] = *reinterpret_cast<const uint4*>(p);
      hi[i] = *reinterpret_cast<const uint4*>(p + DH);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint4 x;
      x.x = (hi[i].x & high[0]) | (lo[i].x & ~high[0]);
      x.y = (hi[i].y & high[1]) | (lo[i].y & ~high[1]);
      x.z = (hi[i].z & high[2]) | (lo[i].z & ~high[2]);
      x.w = (hi[i].w & high[3]) | (lo[i].w & ~high[3]);
      s[i] = 0.0;
#pragma unroll
      for (int e = 0; e < N; ++e) s[i] = fma(q[e], (double)Piece<T>::get(x, e), s[i]);
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
    const int at = sub / (LPB / 8) * BPL + lane / LPB, j = j0 + at;       // which of the eight: the top three bits of sub
    const bool outside = __shfl(page, at, 64) < 0;
    if (sub % (LPB / 8) == 0 && j < held)
      put(j, j == 0 || j == held - 1 ? 0 : outside ? kOutside : order_of(s[0]));   // (those two go by their places)
  }
};

__device__ __forceinline__ int blocks_held(const PageSelectArgs& a, int b) {
  const int L = min(max(a.lens[b], 0), a.max_blocks << a.page_shift);
  return (int)(((long long)L + a.pg.page_size - 1) >> a.page_shift);
}

// ---------------------------------------------------------------------------------------------
// The choice of `want` of `held` > want blocks, in ascending order, by WAVES waves that all come here: the newest one, then the first, then
// those with the highest numbers; number(i) is that of block i * WAVES * 64 + thread, 0 for those two and behind the end.
// The highest number that enough blocks reach is found bit by bit from the first bit in which the numbers differ; a count is
// a ballot per wave and, with several waves, one barrier, and the search ends as soon as the count is right: for scores without
// ties after about as many bits as the number of blocks has, and a few.  Ties that are left go to the lowest places.
// A thread keeps its first KEPT numbers in registers; those of longer lists are read again for every count.
// ---------------------------------------------------------------------------------------------
template <int WAVES, int KEPT, typename Number>
__device__ __forceinline__ void pick(int held, int n_select, Number number, int* out) {
  constexpr int THREADS = WAVES * 64;
  __shared__ unsigned long long s_or[WAVES], s_and[WAVES];
  __shared__ int s_n[2][WAVES], s_eq[2][WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rounds = (held + THREADS - 1) / THREADS;
  unsigned long long kept[KEPT];
#pragma unroll
  for (int i = 0; i < KEPT; ++i) kept[i] = number(i);
  // bits in which the numbers differ
  unsigned long long any = 0, all = ~0ull;
  auto fold = [&](unsigned long long v) { any |= v; all &= v ? v : ~0ull; };
#pragma unroll
  for (int i = 0; i < KEPT; ++i) fold(kept[i]);
  for (int i = KEPT; i < rounds; ++i) fold(number(i));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) { any |= __shfl_xor(any, off, 64); all &= __shfl_xor(all, off, 64); }
  if constexpr (WAVES > 1) {
    if (lane == 0) { s_or[wave] = any; s_and[wave] = all; }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { any |= s_or[w]; all &= s_and[w]; }
  }
  int flip = 0;
  auto count = [&](unsigned long long least) {                           // numbers that reach `least`
    int n = 0;
#pragma unroll
    for (int i = 0; i < KEPT; ++i) n += __popcll(__ballot(kept[i] >= least));
    for (int i = KEPT; i < rounds; ++i) n += __popcll(__ballot(number(i) >= least));
    if constexpr (WAVES > 1) {
      if (lane == 0) s_n[flip][wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) n += s_n[flip][w];
      flip ^= 1;                                                         // (the next count writes the other entries: one barrier is enough)
    }
    return n;
  };
  const int want = max(n_select - 2, 0);                                 // (held > n_select: without the two there are more than want)
  const int top = any == all ? -1 : 63 - __clzll((long long)(any ^ all));
  unsigned long long least = top < 0 ? all : top == 63 ? 0 : all >> (top + 1) << (top + 1);
  int n = held - 2;                                                      // reach `least`
  if (want == 0) { least = ~0ull; n = 0; }                               // (no number is that high)
  for (int bit = top; bit >= 0 && n > want; --bit) {
    const int c = count(least | 1ull << bit);
    if (c >= want) { least |= 1ull << bit; n = c; }
  }
  // n > want: `least` itself is there several times, only the first of those go along
  const int ties = n > want ? want - count(least + 1) : held;
  if constexpr (WAVES > 1) __syncthreads();
  const unsigned long long below = (1ull << lane) - 1;
  int base = 0, base_eq = 0;
  auto give = [&](int i, unsigned long long v) {
    const unsigned long long eq = __ballot(v == least);
    int place_eq = base_eq + __popcll(eq & below);
    if constexpr (WAVES > 1) {
      if (lane == 0) s_eq[i & 1][wave] = __popcll(eq);
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        place_eq += w < wave ? s_eq[i & 1][w] : 0;
        base_eq += s_eq[i & 1][w];
      }
    } else {
      base_eq += __popcll(eq);
    }
    const int j = i * THREADS + threadIdx.x;
    const bool take = v > least || (v == least && place_eq < ties) || j == held - 1 || (j == 0 && n_select > 1);
    const unsigned long long m = __ballot(take);
    int place = base + __popcll(m & below);
    if constexpr (WAVES > 1) {
      if (lane == 0) s_n[i & 1][wave] = __popcll(m);
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        place += w < wave ? s_n[i & 1][w] : 0;
        base += s_n[i & 1][w];
      }
    } else {
      base += __popcll(m);
    }
    if (take) out[place] = j;
  };
#pragma unroll
  for (int i = 0; i < KEPT; ++i)
    if (i < rounds) give(i, kept[i]);
  for (int i = KEPT; i < rounds; ++i) give(i, number(i));
}

// (512 threads: 13.2 us for 128 lists of 512 blocks, 7.8 for 256 of up to 208; 1024: 16.3 and 9.4, 256: 14.7 and 8.4)
constexpr int kOneLaunch = 1024, kChooseThreads = 512, kChooseWaves = kChooseThreads / 64;

// Up to kOneLaunch blocks: a workgroup per (sequence, key head) scores them all into LDS, one of its waves picks.  12.8 us for 32 of
// 512 blocks of 16 sequences x 8 key heads (33 MB of bounds; without the pick 9.8, without the scores 4.8), of which 2.4 are
// the launch, and a scan of 128 lists keeps half the compute units busy.  us of 8 blocks chosen, this launch / the two below: 128 lists of 64 blocks
// 6.8 / 22, of 512 13.9 / 28, of 1024 24 / 32; 512 lists of 1024 51 / 72; only few long lists lose (8 of 1024: 20.6 / 17.8).
template <typename T, int DH>
__global__ __launch_bounds__(kChooseThreads) void k_page_choose(const PageSelectArgs a) {
  __shared__ unsigned long long keys[kOneLaunch];
  const int h = blockIdx.x, b = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, want = a.n_select;
  const int held = blocks_held(a, b);
  int* out = a.blocks + ((size_t)b * a.pg.n_kv_heads + h) * want;
  if (held <= want) {
    for (int j = threadIdx.x; j < want; j += kChooseThreads) out[j] = j < held ? j : -1;
    return;
  }
  using S = Scores<T, DH>;
  if (wave * S::AT_ONCE < held) {
    const int* table = a.table + (size_t)b * a.max_blocks;
    int page = wave * S::AT_ONCE + lane < held ? table[wave * S::AT_ONCE + lane] : -1;
    S s;
    s.init(a, b, h, held);
    for (int j0 = wave * S::AT_ONCE; j0 < held; j0 += kChooseWaves * S::AT_ONCE) {
      s.run(j0, page, [&](int j, unsigned long long v) { keys[j] = v; });
      page = j0 + kChooseWaves * S::AT_ONCE + lane < held ? table[j0 + kChooseWaves * S::AT_ONCE + lane] : -1;
    }
  }
  __syncthreads();
  if (wave != 0) return;
  auto number = [&](int i) { return i * 64 + lane < held ? keys[i * 64 + lane] : 0ull; };
  if (held <= 256) pick<1, 4>(held, want, number, out);
  else if (held <= 512) pick<1, 8>(held, want, number, out);
  else pick<1, 16>(held, want, number, out);
}

// More blocks: the scores by as many workgroups as they need, then a workgroup per (sequence, key head) picks.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_scores(const PageSelectArgs a) {
  const int h = blockIdx.y, b = blockIdx.z, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int held = blocks_held(a, b);
  using S = Scores<T, DH>;
  int j0 = (blockIdx.x * 4 + wave) * S::AT_ONCE;
  if (held <= a.n_select || j0 >= held) return;
  unsigned long long* keys = a.keys + ((size_t)b * a.pg.n_kv_heads + h) * a.max_blocks;
  const int* table = a.table + (size_t)b * a.max_blocks;
  int page = j0 + lane < held ? table[j0 + lane] : -1;
  S s;
  s.init(a, b, h, held);
  for (const int step = gridDim.x * 4 * S::AT_ONCE; j0 < held; j0 += step) {
    s.run(j0, page, [&](int j, unsigned long long v) { keys[j] = v; });
    page = j0 + step + lane < held ? table[j0 + step + lane] : -1;
  }
}

__global__ __launch_bounds__(1024) void k_page_pick(const PageSelectArgs a) {
  const int h = blockIdx.x, b = blockIdx.y, want = a.n_select, held = blocks_held(a, b);
  const size_t row = (size_t)b * a.pg.n_kv_heads + h;
  const unsigned long long* keys = a.keys + row * a.max_blocks;
  int* out = a.blocks + row * want;
  if (held <= want) {
    for (int j = threadIdx.x; j < want; j += 1024) out[j] = j < held ? j : -1;
    return;
  }
  pick<16, 8>(held, want, [&](int i) { const int j = i * 1024 + threadIdx.x; return j < held ? keys[j] : 0ull; }, out);
}

size_t page_select_bytes(int batch, int n_kv_heads, int max_blocks) {
  return max_blocks <= kOneLaunch ? 0 : (size_t)batch * n_kv_heads * max_blocks * 8;
}

namespace {
template <typename T, int DH>
void launch(const PageSelectArgs& a, hipStream_t s) {
  if (a.max_blocks <= kOneLaunch) {
    hipLaunchKernelGGL((k_page_choose<T, DH>), dim3(a.pg.n_kv_heads, a.batch), dim3(kChooseThreads), 0, s, a);
    return;
  }
  // (A wide table's sequences may be short: no more workgroups than keep the memory busy if every list is long.  64 sequences of 32 blocks with
  // room for 8192 took 64 us with a workgroup for every part of the table.)
  const int once = 4 * Scores<T, DH>::AT_ONCE, lists = a.pg.n_kv_heads * a.batch;
  const int along = (int)std::min<long long>(((long long)a.max_blocks + once - 1) / once, std::max(1, 2048 / lists));
  hipLaunchKernelGGL((k_page_scores<T, DH>), dim3(along, a.pg.n_kv_heads, a.batch), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_page_pick, dim3(a.pg.n_kv_heads, a.batch), dim3(1024), 0, s, a);
}
}  // namespace

hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t s) {
  const bool wide = a.pg.head_dim == 128;
  if (a.pg.dtype == CERBERUS_F32) {
    if (wide) launch<float, 128>(a, s);
    else launch<float, 64>(a, s);
  } else {
    if (wide) launch<bf16_t, 128>(a, s);
    else launch<bf16_t, 64>(a, s);
  }
  return hipGetLastError();
}

}  // namespace cerb

// Attention of one new token per sequence over a key-value cache in pages: out = softmax(scale q K^T) V.
#include "paged.h"

#include <limits.h>

#include <algorithm>

namespace cerb {

namespace {

typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

// How the rows of a batch are cut.  Sequence b has rows_of(b) rows to look at (with chosen blocks: the rows of all places of
// its list); they are cut into pieces of `piece` rows, a multiple of what a workgroup takes at a time, and every (piece, key
// head, 16 of its query heads) is a workgroup.  A sequence of one piece is written out by its workgroup, the pieces of
// others are joined by k_paged_join.  Every wave finds its place in that list by itself, from the lengths on the device.
struct Cut {
  int piece;        // rows
  int b;            // sequence of the asked item, -1: behind the end
  int j, pieces;    // which of its pieces, how many
  int slot0;        // partial results of the cut sequences before it
};

__device__ __forceinline__ int rows_of(const PagedAttnArgs& a, int b) {
  const int L = min(max(a.lens[b], 0), a.max_blocks << a.page_shift);
  return a.blocks && L > 0 ? a.n_select << a.page_shift : L;
}

// Rows of a piece if there are `total` and per_head pieces are wanted, which makes eight workgroups for every compute unit, where two run
// at a time: many pieces even out sequences of all lengths, but a piece's beginning and end show in its time.
// So pieces are not cut below 1024 rows for the last half of them, nor below 512 for the third quarter.  us with per_head pieces for
// 512 / 1024 / 2048 workgroups without those two limits: 64 sequences of up to 16384 rows x 8 key heads 204 / 192 / 184, one of 131072 91 / 90 / 96,
// 16 of 257..2049 rows x 32 heads 66 / 63 / 62, lists of 2048 rows for 16 x 8 key heads 31 / 35 / 37.
template <typename I>
__device__ __forceinline__ I piece_rows(I total, I per_head) {
  const I half = (per_head + 1) / 2, quarter = (per_head + 3) / 4;
  const I a = (total + per_head - 1) / per_head, b = (total + half - 1) / half, c = (total + quarter - 1) / quarter;
  const I b1 = b < 1024 ? b : 1024, c1 = c < 512 ? c : 512;
  return a > b1 ? (a > c1 ? a : c1) : (b1 > c1 ? b1 : c1);
}

// unit: pieces are a multiple of so many rows; 0: nothing is cut.  item: which one to find, or (of_seq) the first one of that sequence.
// Lane l looks after sequences l, l + 64, .. (K of them at most); pieces are counted lane by lane.
template <int K>
__device__ __forceinline__ Cut find_cut_of(const PagedAttnArgs& a, int item, bool of_seq, int unit, int per_head) {
  const int lane = threadIdx.x & 63, k = K == 1 ? 1 : (a.batch + 63) >> 6;
  int rows[K];                                                      // (all loads in flight before the first sum)
#pragma unroll
  for (int i = 0; i < K; ++i) rows[i] = i < k && i * 64 + lane < a.batch ? rows_of(a, i * 64 + lane) : 0;
  long long total = 0;
#pragma unroll
  for (int i = 0; i < K; ++i) total += rows[i];
  {
    const int lo = __builtin_amdgcn_readlane(wave_scan((int)(total & 0xfffff)), 63), hi = __builtin_amdgcn_readlane(wave_scan((int)(total >> 20)), 63);
    total = ((long long)hi << 20) + lo;
  }
  Cut c;
  const long long want = total < 1 << 30 ? piece_rows<unsigned>((unsigned)total, per_head) : piece_rows<long long>(total, per_head);   // (64-bit division is slow)
  c.piece = (int)min((max(want, 1ll) + unit - 1) / unit * unit, (long long)INT_MAX);   // (at INT_MAX nothing is cut)
  const unsigned piece = c.piece;
  int n = 0, cuts = 0;
#pragma unroll
  for (int i = 0; i < K; ++i)
    if (i < k) {                                                    // rows[i] becomes the sequence's pieces
      rows[i] = i * 64 + lane < a.batch ? max(1, (int)(((unsigned)rows[i] + piece - 1u) / piece)) : 0;
      n += rows[i];
      cuts += rows[i] > 1 ? rows[i] : 0;
    }
  const int both = wave_scan(n | cuts << 16), n_end = both & 0xffff, cut_end = both >> 16;   // (items: a piece per sequence and kTarget, cut ones: 2 kTarget at most)
  const unsigned long long mine = __ballot(of_seq ? item % 64 == lane : item >= n_end - n && item < n_end);
  c.b = -1;
  c.j = c.pieces = c.slot0 = 0;
  if (mine == 0) return c;
  const int owner = __ffsll((long long)mine) - 1;
  int at = __builtin_amdgcn_readlane(n_end - n, owner), slot = __builtin_amdgcn_readlane(cut_end - cuts, owner);
#pragma unroll
  for (int i = 0; i < K; ++i)
    if (i < k) {
      const int b = i * 64 + owner, p = __builtin_amdgcn_readlane(rows[i], owner);
      if (c.b < 0 && (of_seq ? b == item : item < at + p)) { c.b = b; c.j = of_seq ? 0 : item - at; c.pieces = p; c.slot0 = slot; }
      at += p;
      slot += p > 1 ? p : 0;
    }
  return c;
}
__device__ __forceinline__ Cut find_cut(const PagedAttnArgs& a, int item, bool of_seq, int unit, int per_head) {
  if (unit == 0) return Cut{INT_MAX, item, 0, 1, 0};
  return a.batch <= 64 ? find_cut_of<1>(a, item, of_seq, unit, per_head) : find_cut_of<CERBERUS_MAX_SEQS / 64>(a, item, of_seq, unit, per_head);
}

template <typename T> struct Tile;      // 16-key tiles a wave takes at a time
template <> struct Tile<bf16_t> { static constexpr int U = 2; };
template <> struct Tile<float> { static constexpr int U = 1; };
template <typename T> constexpr int kUnit = 4 * 16 * Tile<T>::U;   // rows that the four waves of a workgroup take at a time

// What a wave holds of its tiles: K in the order of the first product's fragments, V rows as they lie.
template <typename T, int DH> struct Stage;
template <int DH> struct Stage<bf16_t, DH> {
  uint4 k[2][DH / 32];                  // [tile][k-step]: key lane % 16, columns ks * 32 + (lane / 16) * 8 ..
  uint32_t v[8][DH / 32];               // [tile * 4 + i]: key 4 * (lane / 16) + i, columns (lane % 16) * DH / 16 ..
  int rows[2];                          // rows of every tile that count
  int place;                            // own row's place in the wave's tiles, -1: not here (a step over pages)
};
template <int DH> struct Stage<float, DH> {
  float4 k[1][DH / 16];                 // key lane % 16, columns s * 16 + (lane / 16) * 4 ..
  float4 v[4][DH / 64];                 // key 4 * (lane / 16) + i, columns r * 64 + (lane % 16) * 4 ..
  int rows[1];
  int place;
};

}  // namespace

// ---------------------------------------------------------------------------------------------
// A workgroup takes a piece of one sequence's rows for one key head and up to 16 of the query heads that share it; its four
// waves take tiles of the piece in turn, each with a running softmax of its own, joined at the end.  The work is bound by
// the bytes of K and V, each used once, so everything goes from memory straight into registers in the order that the
// matrix instructions want; there is no barrier in the loop, and a wave has the next tiles' loads in flight while it works.
//   S^T = K Q^T   A = 16 keys, B = up to 16 queries (the columns of missing ones are thrown away: with one query per key
//                 head the instructions are 15/16 idle and still not what takes the time)
//                 -> lane: query lane % 16, keys 4 * (lane / 16) + i
//   O^T = V^T P^T B = P^T straight from the S^T registers.  bf16: contraction slot 8 g + 4 u + i of the 32-key product is
//                 key 4 g + i of tile u, so a lane's own scores are its fragment; A = V^T: lane (n, g) has loaded whole pieces
//                 of the eight V rows of those slots, columns n * DH / 16 + j, and the fragment of product j is column j of that
//                 8 x DH/16 square, turned around within the lane by byte permutes.  Product j gives columns j, j + DH / 16, ..
//                 fp32: product (r, c, i) contracts keys 4 g + i over g and gives columns 64 r + 4 n + c.
// A lane's outputs all belong to its query, so the running maximum's factor is the lane's own.
// bf16: probabilities go into the second product as two bf16 planes (p to 2^-17): the matrix units have time.
// Two waves per SIMD with 256 registers each: 16 KB of K and V in work and 16 KB in flight per wave, 128 KB in flight per compute unit.
// Measured (bf16, 128 columns, this kernel alone, least and average of 421 launches): 131072 rows x 8 key heads 81-84 us, 6.4-6.7 TB/s with the matrix
// units busy 6 % of the time; 64 sequences of up to 16384 rows x 8 key heads 176-184, 6.0-6.2; 16 of 257..2049 x 32 heads 55-58,
// 5.6-5.8; 1025 rows x 32 heads 5.6-7.2, which is the chain of length, table and rows.  A copy of 1 GiB runs at 5.1 TB/s.
// STEP: a decoding step's queries and outputs are two bf16 planes, and the newest row has a second plane next to the cache.
// ---------------------------------------------------------------------------------------------
// ONCE: K and V are read once in the launch (up to 16 queries per key head): loaded with the streaming hint.  A model's layers hold more
// than the caches do, so nothing of them is there again in the next step.  131072 rows x 8 key heads: 103 -> 91 us, 64 sequences of
// up to 16384: 206 -> 192; only caches that fit the last-level cache whole lose (134 MB read again and again: 28 -> 32).
template <typename T, int DH, bool STEP, bool ONCE>
__global__ __launch_bounds__(256, 2) void k_paged_attn(const PagedAttnArgs a, int unit, int per_head, int tiles, int items) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int U = Tile<T>::U, DV = DH / 16, KS = BF ? DH / 32 : DH / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lq = lane & 15, g = lane >> 4;
  const int nkv = a.pg.n_kv_heads, group = a.n_heads / nkv;
  // Workgroups in order of pieces, key heads, tiles of 16 queries; consecutive ones go to the 8 XCDs in turn, so the tiles of
  // one (piece, key head), which read the same rows, are 8 apart and meet in one L2.
  // (Pieces are at most one per sequence and kTarget, heads at most 65535: below 2^31.)
  const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, of8 = id / 8, pair = of8 / tiles * 8 + id % 8;
  const int item = pair / nkv, hk = pair % nkv, h0 = of8 % tiles * 16;   // piece, key head, first of its queries
  if (item >= items) return;
  const Cut cut = find_cut(a, item, false, unit, per_head);
  if (cut.b < 0) return;                                            // (uniform over the workgroup)
  const int b = __builtin_amdgcn_readfirstlane(cut.b), ps = a.pg.page_size;
  const int L = min(max(a.lens[b], 0), a.max_blocks << a.page_shift), held = (int)(((long long)L + ps - 1) >> a.page_shift);
  const int begin = __builtin_amdgcn_readfirstlane(cut.j * cut.piece);
  const int end = (int)min((long long)begin + cut.piece, (long long)rows_of(a, b)), first = wave * 16 * U;
  const int n_it = end - begin > first ? (end - begin - first - 1) / kUnit<T> + 1 : 0;   // rounds of this wave

  const int h = hk * group + min(h0 + lq, group - 1);
  const T* qrow = reinterpret_cast<const T*>(a.q) + b * a.q_row + h * DH;
  uint4 qf[KS], ql[STEP ? KS : 1];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    qf[s] = *reinterpret_cast<const uint4*>(qrow + (BF ? s * 32 + g * 8 : s * 16 + g * 4));
    if constexpr (STEP) ql[s] = *reinterpret_cast<const uint4*>(qrow + a.q_lo_off + s * 32 + g * 8);
  }

  // Pages of the next 64 tiles, one lane each: tile e of the wave is tile e % U of its round e / U.
  int my_page = -1, my_rows = 0, my_off = 0, my_place = -1;
  auto look_up = [&](int it) {
    const long long row = begin + (long long)(it + lane / U) * kUnit<T> + first + (lane % U) * 16;
    my_page = -1;
    my_rows = 0;
    my_off = (int)row & (ps - 1);
    my_place = -1;
    if (row < end) {
      int blk = (int)(row >> a.page_shift);
      if (a.blocks) blk = a.blocks[((size_t)b * nkv + hk) * a.n_select + blk];
      if (blk >= 0 && blk < held) {
        const int page = a.table[(size_t)b * a.max_blocks + blk], pos = (blk << a.page_shift) + my_off;
        if (page >= 0 && page < a.pg.n_pages) {
          my_page = page;
          my_rows = min(max(L - pos, 0), 16);
          if (STEP && L - 1 >= pos && L - 1 < pos + 16) my_place = L - 1 - pos;
        } else {
          atomicOr(a.status, (int)CERBERUS_DEV_BAD_PAGE);
        }
      }
    }
  };
  const T* pool_k = reinterpret_cast<const T*>(a.pg.k);
  const T* pool_v = reinterpret_cast<const T*>(a.pg.v);
  auto load = [&](Stage<T, DH>& st, int it) {
    constexpr int kRounds = 64 / U;
    if (it % kRounds == 0) look_up(it);
    st.place = -1;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = it % kRounds * U + u;
      const int page = max(__builtin_amdgcn_readlane(my_page, e), 0), rows = __builtin_amdgcn_readlane(my_rows, e);   // (no rows: page 0, unused)
      const size_t row0 = ((size_t)page * nkv + hk) * ps + __builtin_amdgcn_readlane(my_off, e);
      const int last = max(rows - 1, 0);                            // rows that do not count are re-reads of the last one
      st.rows[u] = rows;
      if constexpr (STEP) {
        const int place = __builtin_amdgcn_readlane(my_place, e);
        if (place >= 0) st.place = u * 16 + place;
      }
      const T* kr = pool_k + (row0 + min(lq, last)) * DH;
      if constexpr (BF) {
#pragma unroll
        for (int s = 0; s < KS; ++s) st.k[u][s] = ld_w<ONCE>(reinterpret_cast<const uint4*>(kr + s * 32 + g * 8));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T* vr = pool_v + (row0 + min(4 * g + i, last)) * DH + lq * DV;
          if constexpr (DV == 8) {
            const uint4 w = ld_w<ONCE>(reinterpret_cast<const uint4*>(vr));
            st.v[u * 4 + i][0] = w.x; st.v[u * 4 + i][1] = w.y; st.v[u * 4 + i][2] = w.z; st.v[u * 4 + i][3] = w.w;
          } else {
            const u32x2_t* p = reinterpret_cast<const u32x2_t*>(vr);
            const u32x2_t w = ONCE ? __builtin_nontemporal_load(p) : *p;
            st.v[u * 4 + i][0] = w[0]; st.v[u * 4 + i][1] = w[1];
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) st.k[u][s] = __builtin_bit_cast(float4, ld_w<ONCE>(reinterpret_cast<const uint4*>(kr + s * 16 + g * 4)));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int r = 0; r < DH / 64; ++r)
            st.v[i][r] = __builtin_bit_cast(float4, ld_w<ONCE>(reinterpret_cast<const uint4*>(pool_v + (row0 + min(4 * g + i, last)) * DH + r * 64 + lq * 4)));
      }
    }
  };

  constexpr int NA = BF ? DV : DH / 16;
  f32x4_t acc[NA];
#pragma unroll
  for (int j = 0; j < NA; ++j) acc[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                                     // l: of the lane's own keys
  const float scale2 = a.scale * 1.44269504088896340736f;           // scores in powers of two

  // bf16: the second product over the wave's 32 keys, V in vv
  auto values = [&](const uint32_t (&vv)[8][DH / 32 > 0 ? DH / 32 : 1], const uint4& ph, const uint4& pl) {
#pragma unroll
    for (int j = 0; j < DV; ++j) {
      uint4 f;
      const unsigned sel = j & 1 ? 0x07060302u : 0x05040100u;
      f.x = __builtin_amdgcn_perm(vv[1][j / 2], vv[0][j / 2], sel);
      f.y = __builtin_amdgcn_perm(vv[3][j / 2], vv[2][j / 2], sel);
      f.z = __builtin_amdgcn_perm(vv[5][j / 2], vv[4][j / 2], sel);
      f.w = __builtin_amdgcn_perm(vv[7][j / 2], vv[6][j / 2], sel);
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, ph), acc[j], 0, 0, 0);
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, pl), acc[j], 0, 0, 0);
    }
  };

  auto work = [&](Stage<T, DH>& st) {
    f32x4_t s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if constexpr (BF) {
          s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, st.k[u][k]), __builtin_bit_cast(bf16x8_t, qf[k]), s[u], 0, 0, 0);
          if constexpr (STEP)
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, st.k[u][k]), __builtin_bit_cast(bf16x8_t, ql[k]), s[u], 0, 0, 0);
        } else {
          const float4 x = st.k[u][k], y = __builtin_bit_cast(float4, qf[k]);
          s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, y.x, s[u], 0, 0, 0);
          s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, y.y, s[u], 0, 0, 0);
          s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, y.z, s[u], 0, 0, 0);
          s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, y.w, s[u], 0, 0, 0);
        }
      }
    }
    if constexpr (STEP) {
      if (st.place >= 0) {                                          // what the cache's rounding left of the newest key
        const T* kl = reinterpret_cast<const T*>(a.own_k_lo) + b * a.own_row + hk * DH;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            uint4 f = make_uint4(0, 0, 0, 0);
            if (st.place == u * 16 + lq) f = *reinterpret_cast<const uint4*>(kl + k * 32 + g * 8);
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, qf[k]), s[u], 0, 0, 0);
          }
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[u][i] *= scale2;
      if (st.rows[u] < 16) {                                        // (uniform over the wave)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool off = 4 * g + i >= st.rows[u];
          if (off) s[u][i] = -INFINITY;
          if constexpr (BF) {
#pragma unroll
            for (int w = 0; w < DH / 32; ++w) st.v[u * 4 + i][w] = off ? 0u : st.v[u * 4 + i][w];
          } else {
#pragma unroll
            for (int r = 0; r < DH / 64; ++r) if (off) st.v[i][r] = make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[u][i]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.f : mn;
    const float fac = __builtin_amdgcn_exp2f(m - base);             // first tiles: 2^-inf = 0
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[u][i] = __builtin_amdgcn_exp2f(s[u][i] - base);
        sum += s[u][i];
      }
    if (__ballot(fac != 1.f)) {
      l *= fac;
#pragma unroll
      for (int j = 0; j < NA; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] *= fac;
    }
    l += sum;
    if constexpr (BF) {
      union { bf16_t e[8]; uint4 w; } ph, pl;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ph.e[u * 4 + i] = f32_to_bf16(s[u][i]);
          pl.e[u * 4 + i] = f32_to_bf16(s[u][i] - bf16_to_f32(ph.e[u * 4 + i]));
        }
      values(st.v, ph.w, pl.w);
      if constexpr (STEP) {
        if (st.place >= 0) {
          const T* vl = reinterpret_cast<const T*>(a.own_v_lo) + b * a.own_row + hk * DH + lq * DV;
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = 0; w < DH / 32; ++w)
              st.v[e][w] = st.place == (e / 4) * 16 + 4 * g + e % 4 ? *reinterpret_cast<const uint32_t*>(vl + 2 * w) : 0u;
          values(st.v, ph.w, pl.w);
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < DH / 64; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 x = st.v[i][r];
          acc[r * 4 + 0] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, s[0][i], acc[r * 4 + 0], 0, 0, 0);
          acc[r * 4 + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, s[0][i], acc[r * 4 + 1], 0, 0, 0);
          acc[r * 4 + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, s[0][i], acc[r * 4 + 2], 0, 0, 0);
          acc[r * 4 + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, s[0][i], acc[r * 4 + 3], 0, 0, 0);
        }
    }
  };

  Stage<T, DH> s0, s1;
  if (n_it > 0) load(s0, 0);
  for (int it = 0; it < n_it; it += 2) {
    if (it + 1 < n_it) load(s1, it + 1);
    work(s0);
    if (it + 1 < n_it) {
      if (it + 2 < n_it) load(s0, it + 2);
      work(s1);
    }
  }

  // the four waves' sums: to the highest maximum, then added
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __shared__ float sm[4][16], sl[4][16];
  __shared__ __attribute__((aligned(16))) float so[4][16][DH + 4];
  if (g == 0) { sm[wave][lq] = m; sl[wave][lq] = l; }
  const bool live = h0 + lq < group;
  if (live) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NA; ++j) {
        const int d = BF ? DV * (4 * g + i) + j : (j / 4) * 64 + 4 * (4 * g + i) + j % 4;
        so[wave][lq][d] = acc[j][i];
      }
  }
  __syncthreads();
  const int n_live = min(16, group - h0);
  for (int t = threadIdx.x; t < n_live * (DH / 4); t += 256) {
    const int q = t / (DH / 4), d = t % (DH / 4) * 4;
    float M = sm[0][q];
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, sm[w][q]);
    float den = 0.f, num[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = sm[w][q] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][q] - M);
      const float4 o = *reinterpret_cast<const float4*>(&so[w][q][d]);
      den += f * sl[w][q];
      num[0] += f * o.x; num[1] += f * o.y; num[2] += f * o.z; num[3] += f * o.w;
    }
    const int head = hk * group + h0 + q;
    if (cut.pieces > 1) {
      const size_t at = (size_t)(cut.slot0 + cut.j) * a.n_heads + head;
      *reinterpret_cast<float4*>(a.part + at * DH + d) = make_float4(num[0], num[1], num[2], num[3]);
      if (d == 0) {
        float* ml = a.part + (size_t)2 * per_head * a.n_heads * DH + at * 2;
        ml[0] = M;
        ml[1] = den;
      }
    } else {
      const float inv = den == 0.f ? 0.f : 1.f / den;               // nothing to look at: zeros
      const float o[4] = {num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
      T* out = reinterpret_cast<T*>(a.out) + b * a.out_row + head * DH + d;
      if constexpr (STEP) {
        st_a4(out, a.out_lo_off, o);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) st_f(out + e, o[e]);
      }
    }
  }
}

// Joins the pieces of a sequence: a workgroup takes `heads` (a power of two) heads, groups of DH / 4 lanes take pieces in turn,
// four at a time.  3.4 to 4.5 us, the chain of lengths, partial results and LDS; a head per workgroup 6.2 for 64 sequences x 32 heads.
template <typename T, int DH, bool STEP>
__global__ __launch_bounds__(256) void k_paged_join(const PagedAttnArgs a, int unit, int per_head, int heads) {
  constexpr int LPP = DH / 4, GROUPS = 256 / LPP;
  const int b = blockIdx.y, t = threadIdx.x / LPP, d = threadIdx.x % LPP * 4;
  const Cut cut = find_cut(a, b, true, unit, per_head);
  if (cut.pieces <= 1) return;                                      // written out already
  const int per = GROUPS / heads, h = min((int)blockIdx.x * heads + t / per, a.n_heads - 1), first = t % per;
  const float* ml = a.part + (size_t)2 * per_head * a.n_heads * DH;
  float M = -INFINITY, den = 0.f, num[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = first; j0 < cut.pieces; j0 += 4 * per) {
    float2 x[4];
    float4 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const size_t at = (size_t)(cut.slot0 + min(j0 + i * per, cut.pieces - 1)) * a.n_heads + h;
      x[i] = *reinterpret_cast<const float2*>(ml + at * 2);
      o[i] = *reinterpret_cast<const float4*>(a.part + at * DH + d);
    }
    float mn = M;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (j0 + i * per >= cut.pieces) { x[i] = make_float2(-INFINITY, 0.f); o[i] = make_float4(0.f, 0.f, 0.f, 0.f); }
      mn = fmaxf(mn, x[i].x);
    }
    const float base = mn == -INFINITY ? 0.f : mn, f0 = __builtin_amdgcn_exp2f(M - base);
    M = mn;
    den *= f0; num[0] *= f0; num[1] *= f0; num[2] *= f0; num[3] *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = __builtin_amdgcn_exp2f(x[i].x - base);
      den += x[i].y * f;
      num[0] += o[i].x * f; num[1] += o[i].y * f; num[2] += o[i].z * f; num[3] += o[i].w * f;
    }
  }
  __shared__ float sm[GROUPS], sd[GROUPS];
  __shared__ __attribute__((aligned(16))) float so[GROUPS][DH];
  *reinterpret_cast<float4*>(&so[t][d]) = make_float4(num[0], num[1], num[2], num[3]);
  if (d == 0) { sm[t] = M; sd[t] = den; }
  __syncthreads();
  if (first != 0 || (int)blockIdx.x * heads + t / per >= a.n_heads) return;
  for (int i = 1; i < per; ++i) M = fmaxf(M, sm[t + i]);
  den = num[0] = num[1] = num[2] = num[3] = 0.f;
  for (int i = 0; i < per; ++i) {
    const float f = sm[t + i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[t + i] - M);
    const float4 o = *reinterpret_cast<const float4*>(&so[t + i][d]);
    den += f * sd[t + i];
    num[0] += f * o.x; num[1] += f * o.y; num[2] += f * o.z; num[3] += f * o.w;
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  const float o[4] = {num[0] * inv, num[1] * inv, num[2] * inv, num[3] * inv};
  T* out = reinterpret_cast<T*>(a.out) + b * a.out_row + h * DH + d;
  if constexpr (STEP) {
    st_a4(out, a.out_lo_off, o);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) st_f(out + e, o[e]);
  }
}

// Pieces of a batch at most, its sequences being no longer than `most` rows: one for each and one for every piece_rows(total) rows, and
// each of the three limits of piece_rows bounds the number of those for any total.
int paged_attention_items(int batch, long long most, int unit, int per_head) {
  if (unit == 0) return batch;
  const long long rows = batch * most, half = (per_head + 1) / 2, quarter = (per_head + 3) / 4;
  const long long cuts = std::min<long long>({per_head, std::max(half, (rows + 1023) / 1024), std::max(quarter, (rows + 511) / 512)});
  return (int)std::min(batch + cuts, batch * ((most - 1) / unit + 1));
}

namespace {

constexpr int kTarget = 2048;     // workgroups a launch aims for at most
constexpr int kTurns = 4;         // turns of a workgroup that take less time than a join
// Lists of chosen blocks from which on none is cut: a workgroup for every compute unit.  us, whole / cut and joined, for 128, 192, 256, 320, 512, 640 and 1024
// lists of 2048 rows: 38 / 29, 39 / 39, 43 / 50, 70 / 64, 82 / 86, 114 / 111, 161 / 171; of 8192 rows: 142 / 91, 139 / 129, 162 / 171, 273 / 220, 320 / 329,
// 456 / 462, 644 / 656.  Just above a whole number of rounds (257..383 and 513..639 lists) long lists would still be better cut.
constexpr int kLists = 256;

int head_tiles(int n_heads, int n_kv_heads) { return (n_heads / n_kv_heads + 15) / 16; }
// pieces that a launch aims for per (key head, 16 queries)
int per_head_of(int n_heads, int n_kv_heads) { return std::max(1, kTarget / (n_kv_heads * head_tiles(n_heads, n_kv_heads))); }

template <typename T, int DH, bool STEP>
void launch(const PagedAttnArgs& a, hipStream_t s) {
  const int tiles = head_tiles(a.n_heads, a.pg.n_kv_heads), per_head = per_head_of(a.n_heads, a.pg.n_kv_heads);
  // Joining pieces is a launch of its own, 5 to 8 us with what goes before it, and a workgroup by itself takes about 1.4 us a turn.  So
  // nothing is cut where all that the table or the list has room for is a few turns, twice as many where every compute unit has
  // its two workgroups anyway (us, 32 heads, cut / whole: 256 rows 10.3 / 7.7, 500 10.4 / 10.6, 1000 11.1 / 18.0; 16 sequences of 1000 50.1 / 45.4),
  // and lists, which are of one length, are not where they are enough workgroups to keep the memory busy.
  const long long most = (long long)(a.blocks ? a.n_select : a.max_blocks) << a.page_shift, pairs = (long long)a.batch * a.pg.n_kv_heads * tiles;
  const bool cuts = most > kTurns * kUnit<T> * (pairs >= 512 ? 2 : 1) && !(a.blocks && pairs >= kLists);
  const int unit = cuts ? kUnit<T> : 0;
  const int items = paged_attention_items(a.batch, most, unit, per_head);
  const long long all = ((long long)items * a.pg.n_kv_heads + 7) / 8 * 8 * tiles, row = std::max(8ll * tiles, (1ll << 18) / (8 * tiles) * (8 * tiles));
  const dim3 grid((unsigned)std::min(all, row), (unsigned)((all - 1) / row + 1));
  if (STEP || tiles == 1) hipLaunchKernelGGL((k_paged_attn<T, DH, STEP, true>), grid, dim3(256), 0, s, a, unit, per_head, tiles, items);   // (a step's heads share no keys)
  else hipLaunchKernelGGL((k_paged_attn<T, DH, STEP, STEP>), grid, dim3(256), 0, s, a, unit, per_head, tiles, items);
  if (cuts) {
    // A head per workgroup where that is at most four for every compute unit (few sequences have many pieces each), else up to
    // four heads: most sequences of a large batch have nothing to join, and their workgroups only find that out.
    const int heads = a.batch * a.n_heads <= 1024 ? 1 : 4;
    hipLaunchKernelGGL((k_paged_join<T, DH, STEP>), dim3((a.n_heads + heads - 1) / heads, a.batch), dim3(256), 0, s, a, unit, per_head, heads);
  }
}

}  // namespace

// partial results: cut sequences have at most 2 per_head pieces (see find_cut: a cut one has more than `piece` rows)
size_t paged_attention_bytes(int n_heads, int n_kv_heads, int head_dim) {
  return (size_t)2 * per_head_of(n_heads, n_kv_heads) * n_heads * (head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s) {
  const bool wide = a.pg.head_dim == 128;
  if (dtype == CERBERUS_F32) {
    if (wide) launch<float, 128, false>(a, s);
    else launch<float, 64, false>(a, s);
  } else if (a.own_k_lo) {
    if (wide) launch<bf16_t, 128, true>(a, s);
    else launch<bf16_t, 64, true>(a, s);
  } else {
    if (wide) launch<bf16_t, 128, false>(a, s);
    else launch<bf16_t, 64, false>(a, s);
  }
  return hipGetLastError();
}

}  // namespace cerb

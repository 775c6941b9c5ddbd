// Attention of one new token per sequence over a key-value cache in pages.
#include "paged.h"

namespace cerb {

// A workgroup per (sequence, head): DH / 4 lanes hold one key's row, four elements each, every key slot with a running
// softmax of its own, merged at the end.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_paged_attn(const PagedAttnArgs a) {
  constexpr int LPK = DH / 4, SLOTS = 256 / LPK;
  const int b = blockIdx.x, h = blockIdx.y, hk = h / (a.n_heads / a.pg.n_kv_heads);
  const int slot = threadIdx.x / LPK, e0 = (threadIdx.x % LPK) * 4;
  const int ps = a.pg.page_size, L = min(max(a.lens[b], 0), a.max_blocks * ps), held = (L + ps - 1) / ps;
  const T* q = reinterpret_cast<const T*>(a.q) + b * a.q_row + h * DH + e0;
  float qv[4], o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    qv[e] = ld_f(q + e);
    if (a.q_lo_off) qv[e] += ld_f(q + a.q_lo_off + e);
    qv[e] *= a.scale;
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  const int nk = a.blocks ? a.n_select * ps : L;
  for (int p0 = 0; p0 < nk; p0 += SLOTS) {
    const int p = p0 + slot;
    int blk = min(p, nk - 1) / ps;
    const int off = p & (ps - 1);
    bool vis = p < nk;
    if (a.blocks) blk = a.blocks[((size_t)b * a.pg.n_kv_heads + hk) * a.n_select + blk];
    vis = vis && blk >= 0 && blk < held && (long long)blk * ps + off < L;
    const int page = vis ? a.table[(size_t)b * a.max_blocks + blk] : 0;
    if (page < 0 || page >= a.pg.n_pages) { vis = false; atomicOr(a.status, (int)CERBERUS_DEV_BAD_PAGE); }
    float kv[4] = {0.f, 0.f, 0.f, 0.f}, vv[4] = {0.f, 0.f, 0.f, 0.f};
    if (vis) {
      const size_t row = ((size_t)page * a.pg.n_kv_heads + hk) * ps + off;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        kv[e] = ld_f(reinterpret_cast<const T*>(a.pg.k) + row * DH + e0 + e);
        vv[e] = ld_f(reinterpret_cast<const T*>(a.pg.v) + row * DH + e0 + e);
      }
      if (a.own_k_lo && blk * ps + off == L - 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kv[e] += ld_f(reinterpret_cast<const T*>(a.own_k_lo) + b * a.own_row + hk * DH + e0 + e);
          vv[e] += ld_f(reinterpret_cast<const T*>(a.own_v_lo) + b * a.own_row + hk * DH + e0 + e);
        }
      }
    }
    float s = (qv[0] * kv[0] + qv[1] * kv[1]) + (qv[2] * kv[2] + qv[3] * kv[3]);
#pragma unroll
    for (int off2 = LPK / 2; off2 > 0; off2 >>= 1) s += __shfl_xor(s, off2, 64);
    if (vis && s != -INFINITY) {
      const float mn = fmaxf(m, s), corr = expf(m - mn), pw = expf(s - mn);
      l = l * corr + pw;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] * corr + pw * vv[e];
      m = mn;
    }
  }
  __shared__ float sm[SLOTS], sl[SLOTS], so[SLOTS][DH];
#pragma unroll
  for (int e = 0; e < 4; ++e) so[slot][e0 + e] = o[e];
  if (e0 == 0) { sm[slot] = m; sl[slot] = l; }
  __syncthreads();
  const int t = threadIdx.x;
  if (t >= DH) return;
  float M = -INFINITY, num = 0.f, den = 0.f;
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) M = fmaxf(M, sm[j]);
#pragma unroll
  for (int j = 0; j < SLOTS; ++j) {
    if (sl[j] == 0.f) continue;
    const float w = expf(sm[j] - M);
    den += w * sl[j];
    num += w * so[j][t];
  }
  const float r = den == 0.f ? 0.f : num / den;
  T* out = reinterpret_cast<T*>(a.out) + b * a.out_row + h * DH + t;
  if (a.out_lo_off) st_a(out, a.out_lo_off, r);
  else st_f(out, r);
}

size_t paged_attention_bytes(int, int, int, int, int, int, int) { return 256; }

hipError_t launch_paged_attention(const PagedAttnArgs& a, int dtype, hipStream_t s) {
  dim3 grid(a.batch, a.n_heads);
  const bool wide = a.pg.head_dim == 128;
  if (dtype == CERBERUS_F32) {
    if (wide) hipLaunchKernelGGL((k_paged_attn<float, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_paged_attn<float, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((k_paged_attn<bf16_t, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_paged_attn<bf16_t, 64>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace cerb

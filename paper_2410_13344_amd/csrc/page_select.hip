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
}  // namespace

// A wave per (block, key head): the score's products and sums in double, because two blocks next to the border of the choice
// change places with the last bits.
template <typename T, int DH>
__global__ __launch_bounds__(256) void k_page_scores(const PageSelectArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int j = blockIdx.x * 4 + wave, h = blockIdx.y, b = blockIdx.z, ps = a.pg.page_size, group = a.n_heads / a.pg.n_kv_heads;
  const int L = min(max(a.lens[b], 0), a.max_blocks * ps), held = (L + ps - 1) / ps;
  if (j >= held) return;
  const int page = a.table[(size_t)b * a.max_blocks + j];
  double s = 0.0;
  if (page >= 0 && page < a.pg.n_pages) {
    const T* bounds = reinterpret_cast<const T*>(a.pg.bounds) + ((size_t)page * a.pg.n_kv_heads + h) * 2 * DH;
    for (int d = lane; d < DH; d += 64) {
      double q = 0.0;
      for (int g = 0; g < group; ++g) {
        const T* qp = reinterpret_cast<const T*>(a.q) + b * a.q_row + (h * group + g) * DH + d;
        q += (double)ld_f(qp);
        if (a.q_lo_off) q += (double)ld_f(qp + a.q_lo_off);
      }
      s += q * (double)ld_f(bounds + (q >= 0.0 ? DH : 0) + d);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
  }
  if (lane == 0)
    a.keys[((size_t)b * a.pg.n_kv_heads + h) * a.max_blocks + j] = j == held - 1 ? kNewest : j == 0 ? kFirst : order_of(s);
}

// A workgroup per (sequence, key head): a block is chosen if fewer than n_select come before it.
__global__ __launch_bounds__(256) void k_page_pick(const PageSelectArgs a) {
  const int h = blockIdx.x, b = blockIdx.y, ps = a.pg.page_size;
  const int L = min(max(a.lens[b], 0), a.max_blocks * ps), held = (L + ps - 1) / ps;
  const size_t row = (size_t)b * a.pg.n_kv_heads + h;
  const unsigned long long* keys = a.keys + row * a.max_blocks;
  int* out = a.blocks + row * a.n_select;
  __shared__ int n_out, wsum[4];
  if (threadIdx.x == 0) n_out = 0;
  for (int j0 = 0; j0 < held; j0 += 256) {
    const int j = j0 + threadIdx.x;
    bool take = false;
    if (j < held) {
      const unsigned long long mine = keys[j];
      int before = 0;
      for (int i = 0; i < held; ++i) before += keys[i] > mine || (keys[i] == mine && i < j);
      take = before < a.n_select;
    }
    const unsigned long long m = __ballot(take);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    if (lane == 0) wsum[wave] = __popcll(m);
    __syncthreads();
    int at = n_out + __popcll(m & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) at += wsum[w];
    if (take) out[at] = j;
    __syncthreads();
    if (threadIdx.x == 0) n_out += wsum[0] + wsum[1] + wsum[2] + wsum[3];
    __syncthreads();
  }
  __syncthreads();
  for (int i = n_out + threadIdx.x; i < a.n_select; i += 256) out[i] = -1;
}

size_t page_select_bytes(int batch, int n_kv_heads, int max_blocks) { return (size_t)batch * n_kv_heads * max_blocks * 8; }

hipError_t launch_page_select(const PageSelectArgs& a, hipStream_t s) {
  dim3 grid((a.max_blocks + 3) / 4, a.pg.n_kv_heads, a.batch);
  const bool wide = a.pg.head_dim == 128;
  if (a.pg.dtype == CERBERUS_F32) {
    if (wide) hipLaunchKernelGGL((k_page_scores<float, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_scores<float, 64>), grid, dim3(256), 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((k_page_scores<bf16_t, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_page_scores<bf16_t, 64>), grid, dim3(256), 0, s, a);
  }
  hipLaunchKernelGGL(k_page_pick, dim3(a.pg.n_kv_heads, a.batch), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace cerb

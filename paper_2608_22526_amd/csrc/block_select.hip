// The blocks that each query attends to: scores against the mean keys and the
// top_k of them (see rs3_block_select).
#include "block.h"

namespace rs3 {

// One thread per (row, block): the score in fp64.
template <class T>
__global__ __launch_bounds__(256) void k_block_score(BlockSelectArgs p) {
  const int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (it >= p.rows * p.n_blk) return;
  const int64_t row = it / p.n_blk, oi = row / p.H_kv;
  const int b = (int)(it - row * p.n_blk), g = (int)(row - oi * p.H_kv), G = p.H / p.H_kv;
  const int64_t o = oi / p.n_q, i = oi - o * p.n_q;
  const T* q = (const T*)p.Q + o * p.qo + i * p.qs + (int64_t)g * G * p.d_h;
  const T* k = (const T*)p.Kmean + ((o * p.H_kv + g) * p.n_blk + b) * p.d_h;
  double s = 0.0;
  for (int h = 0; h < G; ++h)
    for (int d = 0; d < p.d_h; ++d) s += (double)to_f32<T>(q[h * p.d_h + d]) * (double)to_f32<T>(k[d]);
  p.score[it] = s;
}

// Order of the scores as unsigned integers; a NaN counts as -inf.
__device__ __forceinline__ uint64_t order_key(double s) {
  if (s != s) s = -INFINITY;
  const uint64_t u = (uint64_t)__double_as_longlong(s == 0.0 ? 0.0 : s);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// One wave per row: the largest key that at least `want` free blocks reach is
// found bit by bit; blocks above it are kept, and of those at it the lowest.
__global__ __launch_bounds__(64) void k_block_pick(BlockSelectArgs p) {
  const int64_t row = blockIdx.x, oi = row / p.H_kv;
  const int lane = threadIdx.x;
  const int v = visible_keys(p.n_vis, oi, p.n_kv);
  const int nb = (v + p.block - 1) / p.block, want_all = min(p.top_k, nb);
  const int last0 = max(nb - p.n_last, 0);   // forced: below n_first, or from last0
  const int f_lo = min(p.n_first, last0), forced = f_lo + (nb - last0);
  const int want = want_all - forced;        // free blocks [f_lo, last0) to keep
  const double* sc = p.score + row * p.n_blk;
  uint64_t at = 0;
  if (want > 0)
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t t = at | (1ull << bit);
      int n = 0;
      for (int b = f_lo + lane; b < last0; b += 64) n += order_key(sc[b]) >= t;
      for (int m = 1; m < 64; m <<= 1) n += __shfl_xor(n, m, 64);
      if (n >= want) at = t;
    }
  int above = 0;
  if (want > 0) {
    for (int b = f_lo + lane; b < last0; b += 64) above += order_key(sc[b]) > at;
    for (int m = 1; m < 64; m <<= 1) above += __shfl_xor(above, m, 64);
  }
  int ties = want - above, out = 0;   // blocks at the key still to keep
  int32_t* idx = p.idx + row * p.top_k;
  const uint64_t below = (1ull << lane) - 1;
  for (int b0 = 0; b0 < nb; b0 += 64) {
    const int b = b0 + lane;
    const bool on = b < nb, is_forced = on && (b < f_lo || b >= last0), free = on && !is_forced && want > 0;
    const uint64_t key = free ? order_key(sc[b]) : 0;
    const uint64_t eq = __ballot(free && key == at);
    const bool keep = is_forced || (free && (key > at || (key == at && (int)__popcll(eq & below) < ties)));
    ties -= (int)__popcll(eq);
    const uint64_t kept = __ballot(keep);
    if (keep) idx[out + __popcll(kept & below)] = b;
    out += (int)__popcll(kept);
  }
  for (int t = out + lane; t < p.top_k; t += 64) idx[t] = -1;
  if (lane == 0) p.count[row] = out;
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_select(const BlockSelectArgs& a, int dtype, hipStream_t st) {
  if (a.n_blk > 0) {
    const int64_t items = a.rows * a.n_blk;
    const dim3 grid((unsigned)((items + 255) / 256));
    if (dtype == RS3_BF16) RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, k_block_score<bf16_t>, grid, dim3(256), 0, st, a);
    else RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, k_block_score<float>, grid, dim3(256), 0, st, a);
  }
  RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, k_block_pick, dim3((unsigned)a.rows), dim3(64), 0, st, a);
  return hipGetLastError();
}

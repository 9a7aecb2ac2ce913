// Softmax attention of each query over the keys of its listed blocks.
#include "block.h"

namespace rs3 {

// One wave per (query, head): 64 keys at a time, a key per lane for the
// logits, then a channel per lane for the values, with a running maximum and
// sum.  Keys that the query does not see are not read.
template <class T>
__global__ __launch_bounds__(64) void k_block_attend(BlockAttendArgs p) {
  __shared__ float sq[256], sw[64];
  const int64_t oi = blockIdx.x;
  const int h = blockIdx.y, g = h / p.G, lane = threadIdx.x;
  const int64_t o = oi / p.n_q, i = oi - o * p.n_q;
  const T* q = (const T*)p.Q + o * p.qo + i * p.qs + (int64_t)h * p.d_h;
  for (int d = lane; d < p.d_h; d += 64) sq[d] = to_f32<T>(q[d]) * p.qscale;
  __syncthreads();
  const int v = visible_keys(p.n_vis, oi, p.n_kv);
  const int64_t row = oi * p.H_kv + g;
  const int cnt = min(max(p.count[row], 0), p.top_k);
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int t = 0; t < cnt; ++t) {
    const int b = p.idx[row * p.top_k + t];
    if (b < 0 || b >= p.n_blk || (t > 0 && b <= p.idx[row * p.top_k + t - 1])) continue;
    const int64_t j0 = (int64_t)b * p.block;
    const int keys = (int)min((int64_t)p.block, v - j0);
    for (int k0 = 0; k0 < keys; k0 += 64) {
      float s = -INFINITY;
      if (k0 + lane < keys) {
        const T* k = (const T*)p.K + o * p.ko + (j0 + k0 + lane) * p.ks + (int64_t)g * p.d_h;
        s = 0.f;
        for (int d = 0; d < p.d_h; ++d) s += sq[d] * to_f32<T>(k[d]);
      }
      float mx = s;
      for (int w = 1; w < 64; w <<= 1) mx = fmaxf(mx, __shfl_xor(mx, w, 64));
      const float mn = fmaxf(m, mx);
      if (mn == -INFINITY) continue;
      const float alpha = exp2f(m - mn), w = s == -INFINITY ? 0.f : exp2f(s - mn);
      m = mn;
      float sum = w;
      for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
      l = l * alpha + sum;
      __syncthreads();
      sw[lane] = w;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] *= alpha;
      const int n = min(64, keys - k0);
      for (int k = 0; k < n; ++k) {
        const T* vp = (const T*)p.V + o * p.vo + (j0 + k0 + k) * p.vs + (int64_t)g * p.d_h;
        const float wk = sw[k];
        if (wk == 0.f) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (lane + 64 * e < p.d_h) acc[e] += wk * to_f32<T>(vp[lane + 64 * e]);
      }
    }
  }
  T* out = (T*)p.O + o * p.oo + i * p.os + (int64_t)h * p.d_h;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + 64 * e < p.d_h) out[lane + 64 * e] = from_f32<T>(l == 0.f ? 0.f : acc[e] / l);
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_attend(const BlockAttendArgs& a, int dtype, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.n_obj * a.n_q), a.H);
  if (dtype == RS3_BF16) RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, k_block_attend<bf16_t>, grid, dim3(64), 0, st, a);
  else RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, k_block_attend<float>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

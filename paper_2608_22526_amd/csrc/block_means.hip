// Mean keys of the blocks (the scores' side of the block-sparse attention).
#include "block.h"

namespace rs3 {

// grid (blocks, H_kv, n_obj), block 256: d_h/EPL lanes read a key row in
// 16-byte chunks, the groups of lanes take the block's rows in turn, and the
// groups' fp64 sums meet in LDS.  bf16 keys add up exactly in fp64 unless a
// channel's values span more than 2^45 / block, so that the rounded mean does not
// depend on the order.  Bound by the read of the keys: 65536 keys of 8 heads of 128
// in bf16, 136 MB in 26.8 us (5.1 TB/s); the newest blocks of 64 caches in 4 us, a
// launch and a round trip.
template <class T>
__global__ __launch_bounds__(256) void k_block_means(BlockMeansArgs p) {
  constexpr int EPL = 16 / sizeof(T);
  __shared__ double part[256 * EPL];
  const int o = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int len = p.kv_len ? min(max(p.kv_len[o], 0), p.n_kv) : p.n_kv;
  int b = blockIdx.x;
  if (p.n_new > 0) {
    b += max(len - p.n_new, 0) / p.block;
    if ((int64_t)b * p.block >= len) return;
  }
  const int cpr = p.d_h / EPL, groups = 256 / cpr, c = tid % cpr, g = tid / cpr;
  const int64_t j0 = (int64_t)b * p.block;
  const int keys = (int)min((int64_t)p.block, max((int64_t)len - j0, (int64_t)0));
  const T* kp = (const T*)p.K + o * p.ko + (int64_t)h * p.d_h + c * EPL;
  double s[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) s[e] = 0.0;
  for (int r = g; r < keys; r += groups) {
    const u32x4 v = gload((const u32x4*)(kp + (j0 + r) * p.ks));
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      if constexpr (sizeof(T) == 2)
        s[e] += (double)(e & 1 ? __uint_as_float(v[e / 2] & 0xffff0000u) : __uint_as_float(v[e / 2] << 16));
      else
        s[e] += (double)__uint_as_float(v[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < EPL; ++e) part[e * 256 + tid] = s[e];
  __syncthreads();
  for (int d = tid; d < p.d_h; d += 256) {
    double t = 0.0;
    for (int i = 0; i < groups; ++i) t += part[(d % EPL) * 256 + i * cpr + d / EPL];
    ((T*)p.Kmean)[(((int64_t)o * p.H_kv + h) * p.n_blk + b) * p.d_h + d] =
        from_f64<T>(keys > 0 ? t / keys : 0.0);
  }
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_means(const BlockMeansArgs& a, int n_obj, int dtype, hipStream_t st) {
  int nb = a.n_blk;
  if (a.n_new > 0) {   // the blocks that n_new consecutive keys can touch
    const int64_t touch = ((int64_t)a.n_new + a.block - 2) / a.block + 1;
    nb = (int)std::min<int64_t>(nb, touch);
  }
  const dim3 grid(nb, a.H_kv, n_obj);
  if (dtype == RS3_BF16) RS3_LAUNCH(RS3_K_BLOCK_MEANS, st, k_block_means<bf16_t>, grid, dim3(256), 0, st, a);
  else RS3_LAUNCH(RS3_K_BLOCK_MEANS, st, k_block_means<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

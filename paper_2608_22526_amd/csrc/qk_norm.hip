// RMS norm of each head of queries and keys and the rotation of its first
// channels by the token's position, in one pass over the data.
#include "block.h"

namespace rs3 {

// One group of LPH lanes per (row, head), each lane holding 16 bytes of the
// head: the sum of squares is a reduction over the group, adjacent pairs lie
// in one lane and the pairs of the halves in two lanes d_rot/2 channels apart.
template <class T, int LPH>
__global__ __launch_bounds__(256) void k_qk_norm(QkNormArgs p) {
  constexpr int EPL = 16 / sizeof(T), GPW = 256 / LPH;
  const int heads = p.heads[0] + p.heads[1];
  const int64_t item = (int64_t)blockIdx.x * GPW + threadIdx.x / LPH;
  const int64_t row = item / heads;
  if (row >= p.n) return;
  int h = (int)(item - row * heads);
  const int side = h >= p.heads[0];
  if (side) h -= p.heads[0];
  const int ps = p.pos ? p.pos[row] : (int)row;
  if (ps < 0 || (p.d_rot && ps >= p.n_pos)) return;
  const int c = threadIdx.x % LPH, c0 = c * EPL;
  const bool on = c0 < p.d_h;
  float x[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) x[e] = 0.f;
  if (on) {
    const T* xp = (const T*)p.X[side] + row * p.xs[side] + (int64_t)h * p.d_h + c0;
    const u32x4 v = gload((const u32x4*)xp);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      if constexpr (sizeof(T) == 2)
        x[e] = e & 1 ? __uint_as_float(v[e / 2] & 0xffff0000u) : __uint_as_float(v[e / 2] << 16);
      else
        x[e] = __uint_as_float(v[e]);
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) ss += x[e] * x[e];
#pragma unroll
  for (int m = 1; m < LPH; m <<= 1) ss += __shfl_xor(ss, m, 64);
  const float inv = 1.f / sqrtf(ss * p.inv_d + p.eps);
  const float* gain = p.gain[side];
#pragma unroll
  for (int e = 0; e < EPL; ++e) x[e] *= on && gain ? inv * gain[c0 + e] : inv;
  if (p.d_rot) {
    const float* tab = p.table + (int64_t)ps * p.d_rot;
    const bool turn = c0 < p.d_rot;
    if (p.halves) {
      const int hl = p.d_rot / 2 / EPL;            // lanes of a half
      const bool lo = c < hl;
      const int lane = threadIdx.x & 63, other = turn ? (lo ? lane + hl : lane - hl) : lane;
      const int q0 = (lo ? c : c - hl) * EPL;      // the lane's first pair
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float y = __shfl(x[e], other, 64);
        if (turn) {
          const float cs = tab[2 * (q0 + e)], sn = tab[2 * (q0 + e) + 1];
          x[e] = lo ? x[e] * cs - y * sn : y * sn + x[e] * cs;
        }
      }
    } else if (turn) {
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        const float cs = tab[c0 + e], sn = tab[c0 + e + 1], a = x[e], b = x[e + 1];
        x[e] = a * cs - b * sn;
        x[e + 1] = a * sn + b * cs;
      }
    }
  }
  if (!on) return;
  u32x4 w;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(x[e]);
  }
  gstore((u32x4*)((T*)p.Y[side] + row * p.ys[side] + (int64_t)h * p.d_h + c0), w);
}

template <class T>
hipError_t launch(const QkNormArgs& a, hipStream_t st) {
  const int lanes = a.d_h / (16 / (int)sizeof(T));
  const int64_t items = (int64_t)a.n * (a.heads[0] + a.heads[1]);
#define RS3_NORM(LPH)                                                                                   \
  RS3_LAUNCH(RS3_K_QK_NORM, st, (k_qk_norm<T, LPH>), dim3((unsigned)((items + 256 / LPH - 1) / (256 / LPH))), \
             dim3(256), 0, st, a)
  if (lanes <= 2) RS3_NORM(2);
  else if (lanes <= 4) RS3_NORM(4);
  else if (lanes <= 8) RS3_NORM(8);
  else if (lanes <= 16) RS3_NORM(16);
  else if (lanes <= 32) RS3_NORM(32);
  else RS3_NORM(64);
#undef RS3_NORM
  return hipGetLastError();
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_qk_norm(const QkNormArgs& a, int dtype, hipStream_t st) {
  return dtype == RS3_BF16 ? launch<bf16_t>(a, st) : launch<float>(a, st);
}

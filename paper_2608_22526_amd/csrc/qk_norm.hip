// RMS norm of each head of queries and keys and the rotation of its first
// channels by the token's position, in one pass over the data.
#include "block.h"

namespace rs3 {

// Sum over groups of N lanes (a power of two), the same bits in every lane.
template <int N>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (N == 64) return wave_sum(v);
  if constexpr (N >= 2) v += dppf<0xB1>(v);
  if constexpr (N >= 4) v += dppf<0x4E>(v);
  if constexpr (N >= 8) v += dppf<0x141>(v);
  if constexpr (N >= 16) v += dppf<0x140>(v);
  if constexpr (N >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// A group of LPH lanes per row and HC of its heads, each lane holding 16 bytes of
// every one: the heads are in flight together and share the row's factors, which
// are as many bytes as four bf16 heads.  The sum of squares is a reduction over
// the group; adjacent pairs lie in one lane, the pairs of the halves in two lanes
// d_rot/2 channels apart.  Bound by the read and write of the tensors: 16384 rows
// of 32 + 8 heads of 128 in bf16, a tenth of them padding, 344 MB in 61 us (5.6 TB/s);
// 16384 rows of 8 + 8 heads of 32, 36 MB in 9.
template <class T, int LPH, int HC>
__global__ __launch_bounds__(256) void k_qk_norm(QkNormArgs p) {
  constexpr int EPL = 16 / sizeof(T), GPW = 256 / LPH;
  const int64_t item = (int64_t)blockIdx.x * GPW + threadIdx.x / LPH;
  const int per_row = p.chunks[0] + p.chunks[1];
  const int64_t row = item / per_row;
  if (row >= p.n) return;
  int ch = (int)(item - row * per_row);
  const int side = ch >= p.chunks[0];
  if (side) ch -= p.chunks[0];
  const int h0 = ch * HC, heads = p.heads[side];
  const int c = threadIdx.x % LPH, c0 = c * EPL;
  const bool on = c0 < p.d_h;
  const int cl = on ? c0 : 0;   // lanes past the head read its start
  const T* xp = (const T*)p.X[side] + row * p.xs[side] + cl;
  u32x4 v[HC];
#pragma unroll
  for (int h = 0; h < HC; ++h) v[h] = gload((const u32x4*)(xp + (int64_t)min(h0 + h, heads - 1) * p.d_h));
  const int ps = p.pos ? gload(p.pos + row) : (int)row;
  float gain[EPL];
  if (p.gain[side]) {
#pragma unroll
    for (int e = 0; e < EPL; e += 4) {
      const f32x4 w = gload((const f32x4*)(p.gain[side] + cl + e));
#pragma unroll
      for (int k = 0; k < 4; ++k) gain[e + k] = w[k];
    }
  } else {
#pragma unroll
    for (int e = 0; e < EPL; ++e) gain[e] = 1.f;
  }
  if (ps < 0 || (p.d_rot && ps >= p.n_pos)) return;
  // factors of the lane's channels (lanes that turn none read some and leave
  // their values as they are).  Halves: channel e times cs[e] plus its partner
  // times sn[e]; adjacent: pair e/2 has (cs[e/2], sn[e/2])
  float cs[EPL], sn[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) cs[e] = sn[e] = 0.f;
  const int hl = p.d_rot / 2 / EPL;   // lanes of a half
  const bool turn = c0 < p.d_rot;
  int other = threadIdx.x & 63;
  if (p.d_rot) {
    const bool lo = c < hl;
    const float* tab = p.table + (int64_t)ps * p.d_rot + (!turn ? 0 : p.halves ? 2 * EPL * (lo ? c : c - hl) : c0);
    if (p.halves) {
      if (turn) other += lo ? hl : -hl;
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        const f32x4 w = gload((const f32x4*)(tab + 2 * e));
        cs[e] = w[0];
        cs[e + 1] = w[2];
        sn[e] = lo ? -w[1] : w[1];
        sn[e + 1] = lo ? -w[3] : w[3];
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPL; e += 4) {
        const f32x4 w = gload((const f32x4*)(tab + e));
        cs[e / 2] = w[0];
        sn[e / 2] = w[1];
        cs[e / 2 + 1] = w[2];
        sn[e / 2 + 1] = w[3];
      }
    }
  }
  T* yp = (T*)p.Y[side] + row * p.ys[side] + cl;
#pragma unroll
  for (int h = 0; h < HC; ++h) {
    float x[EPL], ss = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      if constexpr (sizeof(T) == 2)
        x[e] = e & 1 ? __uint_as_float(v[h][e / 2] & 0xffff0000u) : __uint_as_float(v[h][e / 2] << 16);
      else
        x[e] = __uint_as_float(v[h][e]);
      ss = __builtin_fmaf(x[e], x[e], ss);
    }
    const float inv = 1.f / sqrtf(group_sum<LPH>(on ? ss : 0.f) * p.inv_d + p.eps);
#pragma unroll
    for (int e = 0; e < EPL; ++e) x[e] *= inv * gain[e];
    if (p.d_rot) {
      if (p.halves) {
        float y[EPL];
        if (LPH >= 16 && hl == 8) {   // eight lanes on within rows of 16
#pragma unroll
          for (int e = 0; e < EPL; ++e) y[e] = dppf<0x128>(x[e]);
        } else {
#pragma unroll
          for (int e = 0; e < EPL; ++e) y[e] = __shfl(x[e], other, 64);
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = turn ? __builtin_fmaf(x[e], cs[e], y[e] * sn[e]) : x[e];
      } else {
#pragma unroll
        for (int e = 0; e < EPL; e += 2) {
          const float a = x[e], b = x[e + 1];
          x[e] = turn ? a * cs[e / 2] - b * sn[e / 2] : a;
          x[e + 1] = turn ? a * sn[e / 2] + b * cs[e / 2] : b;
        }
      }
    }
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) w[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
      else w[e] = __float_as_uint(x[e]);
    }
    if (on && h0 + h < heads) gstore((u32x4*)(yp + (int64_t)(h0 + h) * p.d_h), w);
  }
}

template <class T, int LPH, int HC>
hipError_t launch(QkNormArgs a, hipStream_t st) {
  for (int i = 0; i < 2; ++i) a.chunks[i] = (a.heads[i] + HC - 1) / HC;
  const int64_t items = (int64_t)a.n * (a.chunks[0] + a.chunks[1]);
  RS3_LAUNCH(RS3_K_QK_NORM, st, (k_qk_norm<T, LPH, HC>), dim3((unsigned)((items + 256 / LPH - 1) / (256 / LPH))),
             dim3(256), 0, st, a);
  return hipGetLastError();
}

// Four heads per group where that leaves two waves for every SIMD, else one: a few
// rows are a matter of latency.  One and four heads in us, 32/8 heads of 128: 64
// rows 9.4/9.9, 1024 10.0/9.8, 2048 15.7/11.1, 4096 26/17.5, 16384 111/62 (two heads
// 71, eight 65).
template <class T, int LPH>
hipError_t launch_heads(const QkNormArgs& a, hipStream_t st) {
  const int64_t lanes = (int64_t)a.n * (a.heads[0] + a.heads[1]) * LPH;
  return lanes >= 4 * 2 * 64 * 1024 ? launch<T, LPH, 4>(a, st) : launch<T, LPH, 1>(a, st);
}

template <class T>
hipError_t launch_width(const QkNormArgs& a, hipStream_t st) {
  const int lanes = a.d_h / (16 / (int)sizeof(T));
  if (lanes <= 2) return launch_heads<T, 2>(a, st);
  if (lanes <= 4) return launch_heads<T, 4>(a, st);
  if (lanes <= 8) return launch_heads<T, 8>(a, st);
  if (lanes <= 16) return launch_heads<T, 16>(a, st);
  if (lanes <= 32) return launch_heads<T, 32>(a, st);
  return launch_heads<T, 64>(a, st);
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_qk_norm(const QkNormArgs& a, int dtype, hipStream_t st) {
  return dtype == RS3_BF16 ? launch_width<bf16_t>(a, st) : launch_width<float>(a, st);
}

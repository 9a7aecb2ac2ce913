// Block-sparse attention, a work-group per query and key head (or a part of
// its keys), and the merge of partial rows.
#include "block.h"

#include <type_traits>

namespace rs3 {

// Operand of 16 heads: the sum over the four lane groups that share a head,
// and the maximum (NaN is handed on).
__device__ __forceinline__ float sum4(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  return sum_with_partner(v);
}
__device__ __forceinline__ float max4(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
  return max_with_partner(v);
}

// LDS of k_block_row: two stages of KP keys and values per wave, or after the
// products every wave's sums of 16 heads.  KP is 32, the keys of one bf16 value
// product; long fp32 rows, whose products take eight times as long, go in pieces
// of 16 so that more waves (and their SIMDs) find room.
template <class T, int D>
struct RowLayout {
  static constexpr int CPR = D * (int)sizeof(T) / 16, KP = CPR >= 32 && sizeof(T) == 4 ? 16 : 32;
  static constexpr int VOFF = KP * CPR * 16, STAGE = 2 * VOFF, WAVE = 2 * STAGE;
  static constexpr int NW = 131072 / WAVE < 4 ? 131072 / WAVE : 4;
  static constexpr int XP = D + 4;   // floats of a head's sums
  static_assert(16 * XP * 4 + 16 * 8 <= WAVE, "the sums fit the stages");
};

// One work-group per (query, key head), 16 of its query heads and a split of
// its keys.  The valid blocks of the list go to LDS; the waves take their
// KP-key pieces in turn, each into stages of its own by direct-to-LDS loads one
// piece ahead, so that no barrier stands between the pieces.  The G query heads
// of the key head are the columns of 16x16 products: S^T = K Q^T, and the
// weights feed O^T += V^T P^T from their registers.  Keys past the last that
// the query sees read that one again; their weights and values are 0.  In bf16 the
// weights are rounded for the products (2^-8 of a weight, as O's own rounding), and
// their sum is of the rounded ones.  Bound by the read of the keys and values: one
// token of 32 streams, 32 heads of 128 to 8, 2048 of up to 16384 keys each, 269 MB in
// 50 us (5.4 TB/s), in fp32 538 MB in 95 (5.7).  Few waves (fp32 heads of 256: two, 8
// query heads to 2 key heads, 1024 keys of 32 streams) 135 MB in 39 us (3.5).
template <class T, int D, int NW>
__global__ __launch_bounds__(64 * NW) void k_block_row(BlockAttendArgs p, BlockPartArgs part, int HT) {
  using L = RowLayout<T, D>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int CPR = L::CPR, KP = L::KP, NKT = KP / 16, NDT = D / 16, NQ = BF ? D / 32 : D / 16;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  __shared__ int blist[256], bcount;
  const int tid = threadIdx.x, lane = tid & 63, l15 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t bid = folded_block();
  const int ht = (int)(bid % HT), s = (int)(bid / HT % part.S);
  const int64_t row = bid / HT / part.S, oi = row / p.H_kv;
  if (oi >= (int64_t)p.n_obj * p.n_q) return;
  const int hk = (int)(row - oi * p.H_kv);
  const int64_t o = oi / p.n_q, i = oi - o * p.n_q;
  const int v = visible_keys(p.n_vis, oi, p.n_kv);
  if (wave == 0) {
    const int cnt = min(gload(p.count + row), p.slots);
    const int32_t* list = p.idx + row * p.top_k;
    int n = 0;
    for (int t0 = 0; t0 < cnt; t0 += 64) {
      const int t = min(t0 + lane, cnt - 1);
      const int b = gload(list + t), prev = gload(list + max(t - 1, 0));
      const bool ok = t0 + lane < cnt && b >= 0 && b < p.n_blk && (t == 0 || b > prev) && (int64_t)b * p.block < v;
      const uint64_t m = __ballot(ok);
      if (ok) blist[n + (int)__popcll(m & ((1ull << lane) - 1))] = b;
      n += (int)__popcll(m);
    }
    if (lane == 0) bcount = n;
  }
  // the queries of this lane's head (column l15)
  const int hg = ht * 16 + l15;
  const bool head_on = hg < p.G;
  const T* qp = (const T*)p.Q + o * p.qo + i * p.qs + (int64_t)(hk * p.G + min(hg, p.G - 1)) * D;
  u32x4 q[NQ];
#pragma unroll
  for (int k = 0; k < NQ; ++k) q[k] = gload((const u32x4*)(qp + (BF ? 32 * k + 8 * g : 16 * k + 4 * g)));
#pragma unroll
  for (int k = 0; k < NQ; ++k) q[k] = head_on ? q[k] : u32x4{0, 0, 0, 0};
  __syncthreads();
  const int upb = p.block / KP, U = bcount * upb;   // pieces
  const int u1 = (int)((int64_t)U * (s + 1) / part.S);
  int u = (int)((int64_t)U * s / part.S) + wave;
  const T* Kg = (const T*)p.K + o * p.ko + (int64_t)hk * D;
  const T* Vg = (const T*)p.V + o * p.vo + (int64_t)hk * D;
  // value rows: in bf16 eight keys x 32 bytes per cycle, in fp32 four keys (4
  // apart) x 64 bytes
  auto fv = [](int r) { return BF ? Swz<CPR>::template v<2, 0>(r) : Swz<CPR>::template v<4, 2>(r); };
  uint8_t* mine = lds + wave * L::WAVE;
  auto first_key = [&](int x) { return (int64_t)blist[x / upb] * p.block + x % upb * KP; };
  // Direct-to-LDS loads: load k covers 64 chunks, rows k * RPL + r0 with r0 <
  // RPL, whose swizzles are those of r0 xor those of k * RPL.  Rows past the last
  // that the query sees read that one.
  constexpr int RPL = 64 / CPR;
  const int r0 = lane / CPR, x0 = lane % CPR;
  const int ksb = (int)p.ks * (int)sizeof(T), vsb = (int)p.vs * (int)sizeof(T);   // row strides below 2^24 bytes
  const int xk = 16 * (x0 ^ Swz<CPR>::k(r0)), xv = 16 * (x0 ^ fv(r0));
  auto issue = [&](int x, int slot) {
    const int64_t j0 = first_key(x);
    uint8_t* st = mine + slot * L::STAGE;
    const uint8_t* kb = (const uint8_t*)(Kg + j0 * p.ks);
    const uint8_t* vb = (const uint8_t*)(Vg + j0 * p.vs);
    if (j0 + KP <= v) {
      const int ro = r0 * ksb, wo = r0 * vsb;
#pragma unroll
      for (int k = 0; k < CPR * KP / 64; ++k)
        dma16(kb + (int64_t)k * RPL * ksb + (ro + (xk ^ 16 * Swz<CPR>::k(k * RPL))), st + k * 1024);
#pragma unroll
      for (int k = 0; k < CPR * KP / 64; ++k)
        dma16(vb + (int64_t)k * RPL * vsb + (wo + (xv ^ 16 * fv(k * RPL))), st + L::VOFF + k * 1024);
    } else {
      const int64_t last = v - 1 - j0;   // below 0 where the query sees none of these keys
#pragma unroll
      for (int k = 0; k < CPR * KP / 64; ++k) {
        const int64_t r = min((int64_t)(k * RPL + r0), last);
        dma16(kb + r * ksb + (xk ^ 16 * Swz<CPR>::k(k * RPL)), st + k * 1024);
      }
#pragma unroll
      for (int k = 0; k < CPR * KP / 64; ++k) {
        const int64_t r = min((int64_t)(k * RPL + r0), last);
        dma16(vb + r * vsb + (xv ^ 16 * fv(k * RPL)), st + L::VOFF + k * 1024);
      }
    }
  };
  f32x4 acc[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  if (u < u1) issue(u, 0);
  for (int slot = 0; u < u1; u += NW, slot ^= 1) {
    const int left = (int)min(v - first_key(u), (int64_t)KP);
    if (u + NW < u1) {
      issue(u + NW, slot ^ 1);
      wait_vmcnt<(CPR * KP / 32 < 63 ? CPR * KP / 32 : 62)>();
    } else {
      wait_vmcnt<0>();
    }
    asm volatile("" ::: "memory");   // the stage is read after the wait
    uint8_t* st = mine + slot * L::STAGE;
    if (left < KP) {   // values that the query does not see count as 0 (0 times an infinity is no number)
      for (int c = max(left, 0) * CPR + lane; c < KP * CPR; c += 64) *(u32x4*)(st + L::VOFF + c * 16) = u32x4{0, 0, 0, 0};
      __builtin_amdgcn_wave_barrier();
      asm volatile("" ::: "memory");   // a wave's LDS accesses take place in order
    }
    f32x4 sc[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) sc[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        const u32x4 a = *(const u32x4*)(st + ((16 * kt + l15) * CPR + ((4 * k + g) ^ Swz<CPR>::k(16 * kt + l15))) * 16);
        if constexpr (BF) {
          sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(q[k]), sc[kt], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(q[k][e]), sc[kt], 0, 0, 0);
        }
      }
    if (left < KP) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[kt][r] = 16 * kt + 4 * g + r < left ? sc[kt][r] : -INFINITY;
    }
    float mx = __builtin_elementwise_maximum(max3f(sc[0][0], sc[0][1], sc[0][2]), sc[0][3]);
#pragma unroll
    for (int kt = 1; kt < NKT; ++kt) mx = max3f(max3f(mx, sc[kt][0], sc[kt][1]), sc[kt][2], sc[kt][3]);
    const float mn = __builtin_elementwise_maximum(m, max4(mx) * p.qscale);
    const float sub = mn == -INFINITY ? 0.f : mn;
    const float alpha = __builtin_amdgcn_exp2f(m - sub);
    if (__any(mn > m)) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) acc[dt] *= alpha;
    }
    m = mn;
    l *= alpha;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 4; ++r) sc[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][r], p.qscale, -sub));
    if constexpr (BF) {
      u32x4 pk;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        pk[x] = pack_bf16x2(sc[x >> 1][2 * (x & 1)], sc[x >> 1][2 * (x & 1) + 1]);
        l = add_bf16x2(pk[x], l);
      }
      const int kr = 4 * g + (l15 >> 2), f = fv(kr);
      const uint8_t* vb = st + L::VOFF + kr * CPR * 16 + (lane & 1) * 8;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const uint8_t* va = vb + ((2 * dt + ((lane >> 1) & 1)) ^ f) * 16;
        const u32x2 lo = lds_tr4(va), hi = lds_tr4(va + 16 * CPR * 16);
        acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]}), as_bf16x8(pk),
                                                          acc[dt], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          l += sc[kt][r];
          const int kr = 16 * kt + 4 * g + r;
          const uint8_t* vb = st + L::VOFF + kr * CPR * 16 + (l15 & 3) * 4;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt)
            acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(*(const float*)(vb + ((4 * dt + (l15 >> 2)) ^ fv(kr)) * 16),
                                                           sc[kt][r], acc[dt], 0, 0, 0);
        }
    }
  }
  l = sum4(l);
  // the waves' sums meet in LDS, each in its own stages
  float* xo = (float*)mine;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) *(f32x4*)(xo + l15 * L::XP + 16 * dt + 4 * g) = acc[dt];
  if (g == 0) {
    xo[16 * L::XP + 2 * l15] = m;
    xo[16 * L::XP + 2 * l15 + 1] = l;
  }
  __syncthreads();
  const int heads = min(16, p.G - ht * 16);
  constexpr int CH = BF ? 8 : 4;   // channels of a thread
  for (int x = tid; x < heads * (D / CH); x += 64 * NW) {
    const int h = x / (D / CH), d0 = x % (D / CH) * CH;
    float mw[NW], lw[NW], M = -INFINITY, sum = 0.f, out[CH];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float* xw = (const float*)(lds + w * L::WAVE) + 16 * L::XP + 2 * h;
      mw[w] = xw[0];
      lw[w] = xw[1];
      M = __builtin_elementwise_maximum(M, mw[w]);
    }
#pragma unroll
    for (int e = 0; e < CH; ++e) out[e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      if (mw[w] == -INFINITY) continue;
      const float a = __builtin_amdgcn_exp2f(mw[w] - M);
      const float* xw = (const float*)(lds + w * L::WAVE) + h * L::XP + d0;
      sum += a * lw[w];
#pragma unroll
      for (int e = 0; e < CH; ++e) out[e] += a * xw[e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < CH; ++e) out[e] *= inv;
    const int hh = ht * 16 + h;
    if (part.S == 1) {
      T* dst = (T*)p.O + o * p.oo + i * p.os + (int64_t)(hk * p.G + hh) * D + d0;
      u32x4 w4;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF) w4[e] = pack_bf16x2(out[2 * e], out[2 * e + 1]);
        else w4[e] = __float_as_uint(out[e]);
      }
      gstore((u32x4*)dst, w4);
    } else {
      const int64_t prow = (row * part.S + s) * p.G + hh;
      float* dst = (float*)part.Opart + prow * D + d0;
#pragma unroll
      for (int e = 0; e < CH; e += 4) gstore((f32x4*)(dst + e), f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]});
      if (d0 == 0) *(float2*)(part.ML + 2 * prow) = make_float2(sum == 0.f ? -INFINITY : M, sum);
    }
  }
}

// One thread per (query, head, 16 bytes of O): log-sum-exp merge of the S
// partials, batches of 8 (the last of 4 or 1, where that holds the rest) in
// flight.  F16: values and pairs as k_block_tile leaves them, else fp32.  Bound by
// the read of the partials, 268 MB of f16 in 45 us (6 TB/s).
template <class T, bool F16>
__global__ __launch_bounds__(256) void k_block_merge(BlockAttendArgs p, BlockPartArgs w) {
  constexpr int CH = 16 / sizeof(T);
  const int cpr = p.d_h / CH;
  const int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x, r = it / cpr;
  const int d0 = (int)(it - r * cpr) * CH;
  const int64_t oq = r / p.H;
  const int h = (int)(r - oq * p.H), hk = h / p.G;
  const int64_t o = oq / w.nq, i = oq - o * w.nq;
  if (o >= p.n_obj) return;
  const int64_t row0 = (oq * p.H_kv + hk) * w.S * p.G + (h - hk * p.G);
  const int64_t ml0 = ((o * p.n_q + w.i0 + i) * p.H_kv + hk) * w.S * p.G + (h - hk * p.G);
  float M = -INFINITY, W = 0.f, acc[CH];
#pragma unroll
  for (int e = 0; e < CH; ++e) acc[e] = 0.f;
  auto batch = [&](auto nb, int s0) {
    constexpr int NB = decltype(nb)::value;
    float m[NB], l[NB];
    u32x4 v[NB][F16 ? 1 : CH / 4];
    float top = M;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int64_t at = (int64_t)min(s0 + k, w.S - 1) * p.G, row = row0 + at;
      const u32x2 ml = gload((const u32x2*)(w.ML + 2 * (ml0 + at)));
      m[k] = s0 + k < w.S ? __uint_as_float(ml[0]) : -INFINITY;
      l[k] = __uint_as_float(ml[1]);
#pragma unroll
      for (int x = 0; x < (F16 ? 1 : CH / 4); ++x)
        v[k][x] = F16 ? pload((const u32x4*)((const bf16_t*)w.Opart + row * p.d_h + d0))
                      : pload((const u32x4*)((const float*)w.Opart + row * p.d_h + d0) + x);
    }
#pragma unroll
    for (int k = 0; k < NB; ++k) top = fmaxf(top, m[k]);
    const float sub = top == -INFINITY ? 0.f : top, a = __builtin_amdgcn_exp2f(M - sub);
    W *= a;
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] *= a;
    M = top;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      if (m[k] == -INFINITY) continue;   // nothing was written there
      float wt = __builtin_amdgcn_exp2f(m[k] - sub) * (F16 ? part_sum(l[k]) : l[k]);
      W += wt;
      if constexpr (F16) {
        wt *= part_scale(l[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[2 * e] += wt * part_lo<true>(v[k][0][e]);
          acc[2 * e + 1] += wt * part_hi<true>(v[k][0][e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[e] += wt * __uint_as_float(v[k][e / 4][e % 4]);
      }
    }
  };
  int s0 = 0;
  for (; s0 + 4 < w.S; s0 += 8) batch(std::integral_constant<int, 8>{}, s0);
  if (s0 + 1 < w.S) batch(std::integral_constant<int, 4>{}, s0);
  else if (s0 < w.S) batch(std::integral_constant<int, 1>{}, s0);
  const float inv = W == 0.f ? 0.f : 1.f / W;
  u32x4 w4;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (sizeof(T) == 2) w4[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    else w4[e] = __float_as_uint(acc[e] * inv);
  }
  gstore((u32x4*)((T*)p.O + o * p.oo + (w.i0 + i) * p.os + (int64_t)h * p.d_h + d0), w4);
}

template <class T, int D>
hipError_t launch_row(const BlockAttendArgs& a, const BlockPartArgs& w, hipStream_t st) {
  const int HT = (a.G + 15) / 16;
  const int64_t n = (int64_t)a.n_obj * a.n_q * a.H_kv * w.S * HT;
  RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, (k_block_row<T, D, RowLayout<T, D>::NW>), folded(n), dim3(64 * RowLayout<T, D>::NW),
             (RowLayout<T, D>::NW * RowLayout<T, D>::WAVE), st, a, w, HT);
  return hipGetLastError();
}

template <class T>
hipError_t launch_row_width(const BlockAttendArgs& a, const BlockPartArgs& w, hipStream_t st) {
  switch (a.d_h) {
    case 32: return launch_row<T, 32>(a, w, st);
    case 64: return launch_row<T, 64>(a, w, st);
    case 128: return launch_row<T, 128>(a, w, st);
    default: return launch_row<T, 256>(a, w, st);
  }
}

template <class T, int D>
hipError_t allow() {
  return hipFuncSetAttribute((const void*)k_block_row<T, D, RowLayout<T, D>::NW>, hipFuncAttributeMaxDynamicSharedMemorySize,
                             RowLayout<T, D>::NW * RowLayout<T, D>::WAVE);
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_row(const BlockAttendArgs& a, const BlockPartArgs& w, int dtype, hipStream_t st) {
  return dtype == RS3_BF16 ? launch_row_width<bf16_t>(a, w, st) : launch_row_width<float>(a, w, st);
}

hipError_t rs3_launch_block_merge(const BlockAttendArgs& a, const BlockPartArgs& w, int dtype, bool f16,
                                  hipStream_t st) {
  const int64_t n = (int64_t)a.n_obj * w.nq * a.H * (a.d_h / (dtype == RS3_BF16 ? 8 : 4));
  const dim3 grid((unsigned)((n + 255) / 256));
  if (dtype == RS3_F32) RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, (k_block_merge<float, false>), grid, dim3(256), 0, st, a, w);
  else if (f16) RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, (k_block_merge<bf16_t, true>), grid, dim3(256), 0, st, a, w);
  else RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, (k_block_merge<bf16_t, false>), grid, dim3(256), 0, st, a, w);
  return hipGetLastError();
}

hipError_t rs3_block_setup() {
  const hipError_t es[] = {allow<bf16_t, 32>(), allow<bf16_t, 64>(), allow<bf16_t, 128>(), allow<bf16_t, 256>(),
                           allow<float, 32>(), allow<float, 64>(), allow<float, 128>(), allow<float, 256>(),
                           rs3_block_tile_setup(), rs3_block_select_setup()};
  for (hipError_t e : es)
    if (e != hipSuccess) return e;
  return hipSuccess;
}

// The blocks that each query attends to: scores against the mean keys and the
// top_k of them (see rs3_block_select).
//
// The lists go by scores in fp64, so that they do not depend on the order of a
// sum.  Two forms:
//
//  k_select_row  : a work-group per (query, key head), every score in fp64.  For
//      few queries, where the read of the mean keys is the bound and the fp64
//      units have time.
//  k_select_tile : up to 32 queries of a key head per work-group, scores on the
//      bf16 matrix cores with a bound on their error.  A row whose top_k-th score
//      stands clear of the next by twice the bound is done; otherwise the blocks
//      within that distance of it are scored again in fp64 (a few rows in a
//      hundred, two or three blocks each), and where there are many of them (equal
//      keys, zero queries, values that are no numbers) the whole row is.
#include "block.h"

namespace rs3 {

constexpr int NWS = 8;        // waves of a work-group
constexpr int VPL = 8;        // scores that a lane keeps in registers

// Order of the scores as unsigned integers; a NaN counts as -inf.  0 is no score.
__device__ __forceinline__ uint64_t key64(double s) {
  if (s != s) s = -INFINITY;
  const uint64_t u = (uint64_t)__double_as_longlong(s == 0.0 ? 0.0 : s);
  return u >> 63 ? ~u : u | (1ull << 63);
}
__device__ __forceinline__ double of_key64(uint64_t k) {
  return __longlong_as_double((long long)(k >> 63 ? k ^ (1ull << 63) : ~k));
}
__device__ __forceinline__ uint32_t key32(float s) {
  if (s != s) s = -INFINITY;
  const uint32_t u = __float_as_uint(s == 0.f ? 0.f : s);
  return u >> 31 ? ~u : u | (1u << 31);
}
__device__ __forceinline__ float of_key32(uint32_t k) { return __uint_as_float(k >> 31 ? k ^ (1u << 31) : ~k); }

// The blocks of one row: of those it sees [0, nb), [0, f_lo) and [last0, nb) are
// forced and `want` of the others are to be found.
struct RowRange {
  int nb, f_lo, last0, want;
};
__device__ __forceinline__ RowRange row_range(const BlockSelectArgs& p, int64_t oi) {
  RowRange r;
  r.nb = (visible_keys(p.n_vis, oi, p.n_kv) + p.block - 1) / p.block;
  r.last0 = max(r.nb - p.n_last, 0);
  r.f_lo = min(p.n_first, r.last0);
  r.want = min(p.top_k, r.nb) - (r.f_lo + r.nb - r.last0);
  return r;
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
  return v;
}

// The list of one row from its fp64 scores, by the whole work-group: the largest
// key that `want` scores reach, by halving (first of the values, which needs few
// steps for ordinary scores, then of the keys, which always ends), then the
// blocks above it and the lowest of those at it.  A wave owns a stretch of
// blocks.  sh: 3 * NWS words of LDS.
__device__ void pick_row(const double* sc, const RowRange& r, int top_k, int32_t* idx, int32_t* count, int* sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int seg = (r.nb + 64 * NWS - 1) / (64 * NWS), b0 = wave * seg * 64;
  const uint64_t below = (1ull << lane) - 1;
  auto key_at = [&](int j) -> uint64_t {
    const int b = b0 + 64 * j + lane;
    return b >= r.f_lo && b < r.last0 ? key64(sc[b]) : 0ull;
  };
  uint64_t kept[VPL];
#pragma unroll
  for (int j = 0; j < VPL; ++j) kept[j] = j < seg ? key_at(j) : 0ull;
  int turn = 0;
  auto reach = [&](uint64_t t) {   // scores at or above t, over the work-group
    int n = 0;
#pragma unroll
    for (int j = 0; j < VPL; ++j) n += (int)__popcll(__ballot(kept[j] >= t));
    for (int j = VPL; j < seg; ++j) n += (int)__popcll(__ballot(key_at(j) >= t));
    if (lane == 0) sh[turn * NWS + wave] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < NWS; ++w) n += sh[turn * NWS + w];
    turn ^= 1;
    return n;
  };
  uint64_t lo = 1, hi = ~0ull;   // `want` scores reach lo, fewer reach hi
  int above = 0;
  if (r.want > 0) {
    double span = 0.0;   // the largest finite magnitude, as a start
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const double x = kept[j] ? fabs(of_key64(kept[j])) : 0.0;
      span = x < INFINITY ? fmax(span, x) : span;
    }
    float top = (float)span;
    top = wave_max(top);
    if (lane == 0) sh[2 * NWS + wave] = __float_as_int(top);
    __syncthreads();
    top = 0.f;
#pragma unroll
    for (int w = 0; w < NWS; ++w) top = fmaxf(top, __int_as_float(sh[2 * NWS + w]));
    double vlo = -2.0 * top, vhi = 2.0 * top;
    bool found = false;
    for (int step = 0; step < 20 && top > 0.f && top < INFINITY; ++step) {
      const double v = 0.5 * (vlo + vhi);
      const uint64_t t = key64(v);
      if (!(t > lo && t < hi)) break;
      const int n = reach(t);
      if (n >= r.want) {
        lo = t;
        vlo = v;
      } else {
        hi = t;
        vhi = v;
      }
      if (n == r.want) {
        found = true;
        break;
      }
    }
    while (!found && hi - lo > 1) {
      const uint64_t t = lo + ((hi - lo) >> 1);
      const int n = reach(t);
      if (n >= r.want) lo = t;
      else hi = t;
      found = n == r.want;
    }
    above = reach(lo + 1);
  }
  // kept: forced, above lo, and the first want - above at lo
  int n_eq = 0, n_keep = 0;
  for (int j = 0; j < seg; ++j) {
    const int b = b0 + 64 * j + lane;
    const uint64_t k = r.want > 0 ? key_at(j) : 0ull;
    n_eq += (int)__popcll(__ballot(k == lo));
    n_keep += (int)__popcll(__ballot((b < r.nb && (b < r.f_lo || b >= r.last0)) || k > lo));
  }
  __syncthreads();
  if (lane == 0) {
    sh[wave] = n_eq;
    sh[NWS + wave] = n_keep;
  }
  __syncthreads();
  int ties = r.want - above, out = 0;   // ties left to this wave, entries before it
  for (int w = 0; w < wave; ++w) {
    out += sh[NWS + w] + min(max(ties, 0), sh[w]);
    ties -= sh[w];
  }
  for (int j = 0; j < seg; ++j) {
    const int b = b0 + 64 * j + lane;
    const uint64_t k = r.want > 0 ? key_at(j) : 0ull;
    const uint64_t eq = __ballot(k == lo);
    const bool keep = (b < r.nb && (b < r.f_lo || b >= r.last0)) || k > lo || (k == lo && (int)__popcll(eq & below) < ties);
    ties -= (int)__popcll(eq);
    const uint64_t m = __ballot(keep);
    if (keep) idx[out + (int)__popcll(m & below)] = b;
    out += (int)__popcll(m);
  }
  const int n_all = min(top_k, r.nb);
  for (int t = n_all + tid; t < top_k; t += 64 * NWS) idx[t] = -1;
  if (tid == 0) *count = n_all;
}

// Value e of a 16-byte chunk.
template <class T>
__device__ __forceinline__ float chunk_val(const u32x4& v, int e) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v[e % 4]);
  else return __uint_as_float(e & 1 ? v[e / 2 % 4] & 0xffff0000u : v[e / 2 % 4] << 16);
}

// fp64 scores of blocks [a, b) of one row by the whole work-group: D / EPL lanes a
// block, each with EPL channels of the query summed over its heads (products of
// finite values stay in the fp64 range; where a score is infinite or no number
// the products are added up head by head, whose infinities the sum could hide).
template <class T, int D>
__device__ void score_row(const BlockSelectArgs& p, const T* q, const T* km, int a, int b, double* sc) {
  constexpr int EPL = 16 / sizeof(T), LPB = D / EPL, BPP = 64 * NWS / LPB;
  const int c = threadIdx.x % LPB, G = p.H / p.H_kv;
  double qs[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) qs[e] = 0.0;
  for (int h = 0; h < G; ++h) {
    const u32x4 v = gload((const u32x4*)(q + h * D + c * EPL));
#pragma unroll
    for (int e = 0; e < EPL; ++e) qs[e] += (double)chunk_val<T>(v, e);
  }
  constexpr int U = 4;   // blocks of a lane in flight
  for (int b0 = a + threadIdx.x / LPB; b0 - (int)(threadIdx.x / LPB) < b; b0 += U * BPP) {
    u32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = gload((const u32x4*)(km + (int64_t)min(b0 + u * BPP, b - 1) * D + c * EPL));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double s = 0.0;
#pragma unroll
      for (int e = 0; e < EPL; ++e) s += qs[e] * (double)chunk_val<T>(v[u], e);
#pragma unroll
      for (int m = 1; m < LPB; m <<= 1) s += __shfl_xor(s, m, 64);
      if (__any(!(fabs(s) < INFINITY))) {
        double t = 0.0;
        for (int h = 0; h < G; ++h) {
          const u32x4 w = gload((const u32x4*)(q + h * D + c * EPL));
#pragma unroll
          for (int e = 0; e < EPL; ++e) t += (double)chunk_val<T>(w, e) * (double)chunk_val<T>(v[u], e);
        }
#pragma unroll
        for (int m = 1; m < LPB; m <<= 1) t += __shfl_xor(t, m, 64);
        s = fabs(s) < INFINITY ? s : t;
      }
      if (c == 0 && b0 + u * BPP < b) sc[b0 + u * BPP] = s;
    }
  }
}

template <class T>
__device__ __forceinline__ const T* query_of(const BlockSelectArgs& p, int64_t oi, int g, int D) {
  const int64_t o = oi / p.n_q, i = oi - o * p.n_q;
  return (const T*)p.Q + o * p.qo + i * p.qs + (int64_t)g * (p.H / p.H_kv) * D;
}
template <class T>
__device__ __forceinline__ const T* means_of(const BlockSelectArgs& p, int64_t oi, int g, int D) {
  return (const T*)p.Kmean + ((oi / p.n_q) * p.H_kv + g) * p.n_blk * D;
}

// One (query, key head) per work-group with its scores in LDS, or (SPLIT) one
// stretch of `per` blocks of it, whose scores go to the workspace.  Bound by the
// read of the mean keys.
template <class T, int D, bool SPLIT>
__global__ __launch_bounds__(64 * NWS) void k_select_row(BlockSelectArgs p, int per) {
  extern __shared__ double sc[];
  __shared__ int sh[3 * NWS];
  const int64_t row = blockIdx.x, oi = row / p.H_kv;
  const int g = (int)(row - oi * p.H_kv);
  const RowRange r = row_range(p, oi);
  const int a = max(SPLIT ? (int)blockIdx.y * per : 0, r.f_lo), b = min(SPLIT ? (int)(blockIdx.y + 1) * per : r.nb, r.last0);
  double* out = SPLIT ? p.score + row * p.n_blk : sc;
  if (r.want > 0 && a < b) score_row<T, D>(p, query_of<T>(p, oi, g, D), means_of<T>(p, oi, g, D), a, b, out);
  if constexpr (!SPLIT) {
    __syncthreads();
    pick_row(sc, r, p.top_k, p.idx + row * p.top_k, p.count + row, sh);
  }
}

// The lists from scores in the workspace.
__global__ __launch_bounds__(64 * NWS) void k_select_pick(BlockSelectArgs p) {
  __shared__ int sh[3 * NWS];
  const int64_t row = blockIdx.x;
  pick_row(p.score + row * p.n_blk, row_range(p, row / p.H_kv), p.top_k, p.idx + row * p.top_k, p.count + row, sh);
}

__device__ __forceinline__ int pop(bool x) { return (int)__popcll(__ballot(x)); }

__device__ __forceinline__ u32x2 split_bf16(float a, float b) {   // (hi pair, lo pair)
  const uint32_t hi = pack_bf16x2(a, b);
  return u32x2{hi, pack_bf16x2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u))};
}

// TR (32, 16, 8 or 4) queries of one (object, key head) per work-group.  LDS, in
// turn: the queries, summed over their heads and split into two bf16 terms; the
// scores [TR][pitch]; fp64 scores of a hard row.
template <class T, int D>
__global__ __launch_bounds__(64 * NWS, 2) void k_select_tile(BlockSelectArgs p, int TR, int n_tile, int pitch) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NQ = D / 16;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  __shared__ float qn[32], kn[NWS];
  __shared__ int sh[3 * NWS], hard[32], n_hard;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l31 = lane & 31;
  const int64_t og = blockIdx.x / n_tile;
  const int q0 = (int)(blockIdx.x - og * n_tile) * TR, G = p.H / p.H_kv;
  const int64_t o = og / p.H_kv;
  const int g = (int)(og - o * p.H_kv), nr = min(TR, p.n_q - q0);
  const T* qbase = (const T*)p.Q + o * p.qo + (int64_t)q0 * p.qs + (int64_t)g * G * D;
  const T* km = (const T*)p.Kmean + og * p.n_blk * D;
  if (tid == 0) n_hard = 0;
  // queries: 8 channels of a row per thread
  constexpr int CPQ = D / 8;
  for (int x = tid; x < 32 * CPQ; x += 64 * NWS) {
    const int r = x / CPQ, c = x % CPQ;
    float s[8], ab = 0.f, sa[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = sa[e] = 0.f;
    if (r < nr)
      for (int h = 0; h < G; ++h) {
        const T* qp = qbase + r * p.qs + h * D + 8 * c;
#pragma unroll
        for (int y = 0; y < (BF ? 1 : 2); ++y) {
          const u32x4 v = gload((const u32x4*)qp + y);
#pragma unroll
          for (int e = 0; e < (BF ? 8 : 4); ++e) {
            const float f = chunk_val<T>(v, e);
            s[4 * y + e] += f;
            sa[4 * y + e] += __builtin_fabsf(f);
          }
        }
      }
    u32x4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u32x2 t = split_bf16(s[2 * e], s[2 * e + 1]);
      hi[e] = t[0];
      lo[e] = t[1];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ab += sa[e] * sa[e];
#pragma unroll
    for (int m = 1; m < CPQ; m <<= 1) ab += __shfl_xor(ab, m, 64);
    u32x4* qt = (u32x4*)lds + r * CPQ + (c ^ Swz<CPQ>::k(r));
    qt[0] = hi;
    qt[32 * CPQ] = lo;
    if (c == 0) qn[r] = sqrtf(ab);
  }
  // the most blocks that a row of the tile sees
  int nbm = 0;
  if (lane < nr) nbm = row_range(p, o * p.n_q + q0 + lane).nb;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) nbm = max(nbm, __shfl_xor(nbm, m, 64));
  __syncthreads();
  const bool two = !BF || G > 1;   // one bf16 head is its own first term
  u32x4 qh[NQ], ql[NQ];
#pragma unroll
  for (int k = 0; k < NQ; ++k) {
    const u32x4* qt = (const u32x4*)lds + l31 * CPQ + ((2 * k + half) ^ Swz<CPQ>::k(l31));
    qh[k] = qt[0];
    ql[k] = two ? qt[32 * CPQ] : u32x4{0, 0, 0, 0};
  }
  __syncthreads();
  float* sc = (float*)lds;
  float k2 = 0.f;   // the largest squared norm of a mean key
  for (int bt = wave; bt * 32 < nbm; bt += NWS) {
    const T* kp = km + (int64_t)min(bt * 32 + l31, nbm - 1) * D + 8 * half;
    f32x16 acc;
    float kk = 0.f;
    constexpr int KB = BF ? (NQ < 8 ? NQ : 8) : (NQ < 4 ? NQ : 4);
#pragma unroll
    for (int k0 = 0; k0 < NQ; k0 += KB) {
      u32x4 a[KB][BF ? 1 : 2];
#pragma unroll
      for (int k = 0; k < KB; ++k)
#pragma unroll
        for (int y = 0; y < (BF ? 1 : 2); ++y) a[k][y] = gload((const u32x4*)(kp + 16 * (k0 + k)) + y);
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        u32x4 ah, al = {0, 0, 0, 0};
        if constexpr (BF) {
          ah = a[k][0];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const u32x2 t = split_bf16(__uint_as_float(a[k][e / 2][2 * (e & 1)]), __uint_as_float(a[k][e / 2][2 * (e & 1) + 1]));
            ah[e] = t[0];
            al[e] = t[1];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
          const bf16x2_t v = __builtin_bit_cast(bf16x2_t, ah[e]);
          kk = __builtin_amdgcn_fdot2_f32_bf16(v, v, kk, false);
        }
        const int ks = k0 + k;
        acc = mfma32(ah, qh[ks], ks == 0 ? f32x16{} : acc);
        if (two) acc = mfma32(ah, ql[ks], acc);
        if constexpr (!BF) acc = mfma32(al, qh[ks], acc);
      }
    }
    k2 = __builtin_elementwise_maximum(k2, sum_with_partner(kk));
    if (l31 < nr)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *(f32x4*)(sc + l31 * pitch + 32 * bt + 8 * x + 4 * half) = f32x4{acc[4 * x], acc[4 * x + 1], acc[4 * x + 2], acc[4 * x + 3]};
  }
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) k2 = __builtin_elementwise_maximum(k2, __shfl_xor(k2, m, 64));
  if (lane == 0) kn[wave] = k2;
  __syncthreads();
  k2 = 0.f;
#pragma unroll
  for (int w = 0; w < NWS; ++w) k2 = __builtin_elementwise_maximum(k2, kn[w]);
  // Error of a score, relative to |q| |k| (|q| of the heads' magnitudes; 2 % for
  // the first terms' norms): an fp32 sum of D products per term, truncated at
  // worst; the heads' sum; two bf16 terms keep 2^-18 of a value.  Values below
  // 2^-60 and products below 2^-126 may count as 0.
  const float rel = 1.02f * ((float)((BF ? (two ? 2 : 1) : 3) * D + 16 + G) * 0x1p-23f + (two ? 0x1p-16f : 0.f));
  const float keps = 2.f * rel * (sqrtf(k2) + 0x1p-60f);
  const uint64_t below = (1ull << lane) - 1;
  for (int r = wave; r < nr; r += NWS) {
    const int64_t oi = o * p.n_q + q0 + r, row = oi * p.H_kv + g;
    const RowRange rr = row_range(p, oi);
    const float* srow = sc + r * pitch;
    int32_t* idx = p.idx + row * p.top_k;
    const float eps2 = keps * (qn[r] + 0x1p-60f) + 0x1p-100f;   // twice the bound
    const int seg = (rr.nb + 63) / 64;
    auto key_at = [&](int j) -> uint32_t {
      const int b = 64 * j + lane;
      return b >= rr.f_lo && b < rr.last0 ? key32(srow[b]) : 0u;
    };
    uint32_t kept[2 * VPL];
#pragma unroll
    for (int j = 0; j < 2 * VPL; ++j) kept[j] = j < seg ? key_at(j) : 0u;
    auto reach = [&](uint32_t t) {
      int n = 0;
#pragma unroll
      for (int j = 0; j < 2 * VPL; ++j)
        if (j < seg) n += pop(kept[j] >= t);
      for (int j = 2 * VPL; j < seg; ++j) n += pop(key_at(j) >= t);
      return n;
    };
    // scores above w_hi are kept, and `need` of the `cand` ones from w_lo to w_hi
    uint32_t lo = 1, hi = ~0u;
    bool is_hard = false;
    int cand = 0, need = 0;
    uint32_t w_lo = 1, w_hi = 0;
    if (rr.want > 0) {
      if (!(qn[r] * sqrtf(k2) < 1e38f)) {   // a score may leave the fp32 range, or is no number
        is_hard = true;
      } else {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * VPL; ++j) top = fmaxf(top, kept[j] ? __builtin_fabsf(of_key32(kept[j])) : 0.f);
        for (int j = 2 * VPL; j < seg; ++j) {
          const uint32_t k = key_at(j);
          top = fmaxf(top, k ? __builtin_fabsf(of_key32(k)) : 0.f);
        }
        top = wave_max(top);
        float vlo = -1.01f * top, vhi = 1.01f * top;
        bool found = false;
        for (int step = 0; step < 16 && vhi < INFINITY; ++step) {
          const float v = 0.5f * (vlo + vhi);
          const uint32_t t = key32(v);
          if (!(t > lo && t < hi)) break;
          const int n = reach(t);
          if (n >= rr.want) {
            lo = t;
            vlo = v;
          } else {
            hi = t;
            vhi = v;
          }
          if (n == rr.want) {
            found = true;
            break;
          }
        }
        while (!found && hi - lo > 1) {
          const uint32_t t = lo + ((hi - lo) >> 1);
          const int n = reach(t);
          if (n >= rr.want) lo = t;
          else hi = t;
          found = n == rr.want;
        }
        // the want-th score, and the largest below it (or equal to it)
        uint32_t kth = ~0u, next = 0;
        for (int j = 0; j < seg; ++j) {
          const uint32_t k = key_at(j);
          if (k >= lo) kth = min(kth, k);
          else next = max(next, k);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
          kth = min(kth, (uint32_t)__shfl_xor((int)kth, m, 64));
          next = max(next, (uint32_t)__shfl_xor((int)next, m, 64));
        }
        const float fk = of_key32(kth);
        if (!found || (next > 0 && !(fk - of_key32(next) > eps2))) {
          w_lo = key32(fk - eps2);
          w_hi = key32(fk + eps2);
          const int sure = reach(w_hi + 1);
          cand = reach(w_lo) - sure;
          need = rr.want - sure;
          is_hard = cand > 64;
        } else {
          w_lo = 1;
          w_hi = kth - 1;   // no block is between
        }
      }
    }
    if (is_hard) {
      if (lane == 0) hard[atomicAdd(&n_hard, 1)] = r;
      continue;
    }
    // fp64 scores of the candidates, the c-th in lane c, and its rank among them
    uint64_t win = 0;   // candidates that are kept, in their order
    if (cand > 0) {
      double mine = 0.0;
      int c = 0;
      for (int j = 0; j < seg; ++j) {
        const uint32_t k = key_at(j);
        uint64_t m = __ballot(k >= w_lo && k <= w_hi);
        for (; m; m &= m - 1, ++c) {
          const T* kp = km + (int64_t)(64 * j + __builtin_ctzll(m)) * D;
          const T* qp = qbase + r * p.qs;
          double s = 0.0;
          for (int d = lane; d < D; d += 64) {
            double qd = 0.0;
            for (int h = 0; h < G; ++h) qd += (double)to_f32<T>(qp[h * D + d]);
            s += qd * (double)to_f32<T>(kp[d]);
          }
          s = wave_sum64(s);
          if (lane == c) mine = s;
        }
      }
      const uint64_t mk = key64(mine);
      int rank = 0;
      for (int x = 0; x < cand; ++x) {
        const uint64_t other = (uint64_t)__shfl((long long)mk, x, 64);
        rank += other > mk || (other == mk && x < lane);
      }
      win = __ballot(lane < cand && rank < need);
    }
    int out = 0, c = 0;
    for (int j = 0; j < seg; ++j) {
      const int b = 64 * j + lane;
      const uint32_t k = rr.want > 0 ? key_at(j) : 0u;
      const bool in = k >= w_lo && k <= w_hi;
      const uint64_t im = __ballot(in);
      const bool keep = (b < rr.nb && (b < rr.f_lo || b >= rr.last0)) || (k > w_hi && k > 0) ||
                        (in && ((win >> (c + (int)__popcll(im & below))) & 1ull));
      c += (int)__popcll(im);
      const uint64_t m = __ballot(keep);
      if (keep) idx[out + (int)__popcll(m & below)] = b;
      out += (int)__popcll(m);
    }
    for (int t = out + lane; t < p.top_k; t += 64) idx[t] = -1;
    if (lane == 0) p.count[row] = out;
  }
  __syncthreads();
  // hard rows: every score in fp64, by the whole work-group
  double* sd = (double*)lds;
  for (int x = 0; x < n_hard; ++x) {
    const int r = hard[x];
    const int64_t oi = o * p.n_q + q0 + r, row = oi * p.H_kv + g;
    const RowRange rr = row_range(p, oi);
    score_row<T, D>(p, qbase + r * p.qs, km, rr.f_lo, rr.last0, sd);
    __syncthreads();
    pick_row(sd, rr, p.top_k, p.idx + row * p.top_k, p.count + row, sh);
    __syncthreads();
  }
}

template <class T, int D>
hipError_t launch(const BlockSelectArgs& a, const BlockSelectPlan& pl, hipStream_t st) {
  if (pl.tile) {
    const int n_tile = (a.n_q + pl.TR - 1) / pl.TR;
    const int64_t n = (int64_t)a.n_obj * a.H_kv * n_tile;
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_tile<T, D>), dim3((unsigned)n), dim3(64 * NWS), pl.lds, st, a, pl.TR,
               n_tile, pl.pitch);
  } else if (pl.split > 1) {
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_row<T, D, true>), dim3((unsigned)a.rows, pl.split), dim3(64 * NWS), 0, st,
               a, (a.n_blk + pl.split - 1) / pl.split);
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, k_select_pick, dim3((unsigned)a.rows), dim3(64 * NWS), 0, st, a);
  } else {
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_row<T, D, false>), dim3((unsigned)a.rows), dim3(64 * NWS), pl.lds, st, a,
               a.n_blk);
  }
  return hipGetLastError();
}

template <class T>
hipError_t launch_width(const BlockSelectArgs& a, const BlockSelectPlan& pl, hipStream_t st) {
  switch (a.d_h) {
    case 32: return launch<T, 32>(a, pl, st);
    case 64: return launch<T, 64>(a, pl, st);
    case 128: return launch<T, 128>(a, pl, st);
    default: return launch<T, 256>(a, pl, st);
  }
}

template <class T, int D>
static hipError_t allow() {
  const hipFuncAttribute at = hipFuncAttributeMaxDynamicSharedMemorySize;
  const hipError_t e = hipFuncSetAttribute((const void*)k_select_tile<T, D>, at, SELECT_LDS);
  return e != hipSuccess ? e : hipFuncSetAttribute((const void*)k_select_row<T, D, false>, at, SELECT_LDS);
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_select(const BlockSelectArgs& a, const BlockSelectPlan& pl, int dtype, hipStream_t st) {
  return dtype == RS3_BF16 ? launch_width<bf16_t>(a, pl, st) : launch_width<float>(a, pl, st);
}

hipError_t rs3_block_select_setup() {
  const hipError_t es[] = {allow<bf16_t, 32>(), allow<bf16_t, 64>(), allow<bf16_t, 128>(), allow<bf16_t, 256>(),
                           allow<float, 32>(), allow<float, 64>(), allow<float, 128>(), allow<float, 256>()};
  for (hipError_t e : es)
    if (e != hipSuccess) return e;
  return hipSuccess;
}

// The blocks that each query attends to: scores against the mean keys and the
// top_k of them (see rs3_block_select).
//
// The lists go by scores in fp64, so that they do not depend on the order of a
// sum.  Two forms:
//
//  k_select_row  : a work-group per (query, key head), every score in fp64.  For
//      few queries, where the read of the mean keys is the bound and the fp64
//      units have time: one token of 32 streams, up to 2048 blocks of 8 key heads of
//      128, 81 MB in 25 us (3.2 TB/s); streams of 2048 blocks each, 134 MB in 34
//      (4.0): a row per CU, the longest of which ends last.
//  k_select_tile : up to 32 queries of a key head per work-group, scores on the
//      bf16 matrix cores with a bound on their error.  A row whose top_k-th score
//      stands clear of the next by twice the bound is done; otherwise the blocks
//      within that distance of it are scored again in fp64 (a few rows in a
//      hundred, two or three blocks each), and where there are many of them (equal
//      keys, zero queries, values that are no numbers) the whole row is.  4096 prompt
//      tokens, 4 key heads of 128 and up to 512 blocks in 30 us: scores 14, the rest
//      the choice.  Bound by each wave's chain of dependent steps: two work-groups
//      per CU are all there is, vector instructions take 57 % of the SIMDs' cycles, and
//      of the waves' time 45 % waits for data or barriers, 22 % for an issue slot.
#include "block.h"

namespace rs3 {

constexpr int NWS = 8;        // waves of a work-group of k_select_tile
constexpr int NWR = 16;       // of k_select_row: more of the mean keys in flight per CU
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

// The blocks of one row: of those it sees [0, nb), [0, f_lo) and [last0, nb) are
// forced and `want` of the others are to be found.
struct RowRange {
  int nb, f_lo, last0, want;
};
__device__ __forceinline__ RowRange range_of(const BlockSelectArgs& p, int nb) {
  RowRange r;
  r.nb = nb;
  r.last0 = max(r.nb - p.n_last, 0);
  r.f_lo = min(p.n_first, r.last0);
  r.want = min(p.top_k, r.nb) - (r.f_lo + r.nb - r.last0);
  return r;
}
__device__ __forceinline__ RowRange row_range(const BlockSelectArgs& p, int64_t oi) {
  return range_of(p, (visible_keys(p.n_vis, oi, p.n_kv) + p.block - 1) / p.block);
}

// Sum over groups of N lanes (a power of two from 4 on), the same bits in every
// lane: the exchanges of wave_sum on both halves of the values.
template <int CTRL>
__device__ __forceinline__ double dppd(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, false);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <int N>
__device__ __forceinline__ double group_sum64(double v) {
  v += dppd<0xB1>(v);
  v += dppd<0x4E>(v);
  if constexpr (N >= 8) v += dppd<0x141>(v);
  if constexpr (N >= 16) v += dppd<0x140>(v);
  auto both = [](uint32_t lo, uint32_t hi) { return __longlong_as_double((long long)((uint64_t)hi << 32 | lo)); };
  if constexpr (N >= 32) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
    const auto b = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = both(a[0], b[0]) + both(a[1], b[1]);
  }
  if constexpr (N >= 64) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const auto a = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    v = both(a[0], b[0]) + both(a[1], b[1]);
  }
  return v;
}

// Minimum and maximum over the lanes by the exchanges of wave_max.
__device__ __forceinline__ float wave_min(float v) { return -wave_max(-v); }

// Bits of the 64 blocks from 64 j on that lie in [a, b).
__device__ __forceinline__ uint64_t range_bits(int j, int a, int b) {
  const int lo = min(max(a - 64 * j, 0), 64), hi = min(max(b - 64 * j, 0), 64);
  if (lo >= hi) return 0;
  return (~0ull >> (64 - (hi - lo))) << lo;
}
__device__ __forceinline__ uint64_t forced_bits(const RowRange& r, int j) {
  if (64 * j >= r.f_lo && 64 * j + 64 <= r.last0) return 0;
  return range_bits(j, 0, r.f_lo) | range_bits(j, r.last0, r.nb);
}

// LDS of pick_row: three counters in turn, a word or two per wave, and the
// counts of BINS intervals and the few scores of the short way.
constexpr int BINS = 256;
template <int NW>
struct PickLds {
  unsigned long long n[3];
  float f[2 * NW];
  uint32_t bin[BINS];
  uint64_t key[64];
  int block[64];
};

// The list of one row from its fp64 scores, by a work-group of NW waves: the
// largest key that `want` scores reach, by quartering (first of the values, which
// needs few steps for ordinary scores, then of the keys, which always ends),
// then the blocks above it and the lowest of those at it.  A wave owns a stretch
// of blocks.  The short way, for finite scores of which a few are wanted: they
// are counted in BINS intervals from the largest down, and if at most 64 lie in
// the interval of the want-th and above, one wave ranks those.
template <int NW>
__device__ void pick_row(const double* sc, const RowRange& r, int top_k, int32_t* idx, int32_t* count, PickLds<NW>& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int seg = (r.nb + 64 * NW - 1) / (64 * NW), j0 = wave * seg;
  const uint64_t below = (1ull << lane) - 1;
  auto key_at = [&](int j) -> uint64_t {
    const int b = 64 * (j0 + j) + lane;
    return b >= r.f_lo && b < r.last0 ? key64(sc[b]) : 0ull;
  };
  uint64_t kept[VPL];
#pragma unroll
  for (int j = 0; j < VPL; ++j) kept[j] = j < seg ? key_at(j) : 0ull;
  // scores at or above t[0..2], over the work-group: 21 bits of a counter each, so
  // that a wave's share of 2^21 blocks is counted one short (they are compared with
  // at most 256)
  int slot = 0;
  if (tid < 3) sh.n[tid] = 0;
  for (int x = tid; x < BINS; x += 64 * NW) sh.bin[x] = 0;
  auto reach = [&](const uint64_t (&t)[3], int (&n)[3]) {
    n[0] = n[1] = n[2] = 0;
#pragma unroll
    for (int j = 0; j < VPL; ++j)
      if (j < seg)
#pragma unroll
        for (int x = 0; x < 3; ++x) n[x] += (int)__popcll(__ballot(kept[j] >= t[x]));
    for (int j = VPL; j < seg; ++j) {
      const uint64_t k = key_at(j);
#pragma unroll
      for (int x = 0; x < 3; ++x) n[x] += (int)__popcll(__ballot(k >= t[x]));
    }
#pragma unroll
    for (int x = 0; x < 3; ++x) n[x] = min(n[x], (1 << 21) / NW - 1);
    if (lane == 0)
      atomicAdd(&sh.n[slot], (unsigned long long)n[0] | (unsigned long long)n[1] << 21 | (unsigned long long)n[2] << 42);
    __syncthreads();
    const unsigned long long all = sh.n[slot];
    // the counter of the step before last: everybody has read it
    if (tid == 0) sh.n[slot == 0 ? 2 : slot - 1] = 0;
    slot = slot == 2 ? 0 : slot + 1;
#pragma unroll
    for (int x = 0; x < 3; ++x) n[x] = (int)(all >> (21 * x)) & 0x1fffff;
  };
  uint64_t lo = 1, hi = ~0ull;   // `want` scores reach lo, fewer reach hi
  int above = 0;
  if (r.want > 0) {
    // ordinary scores: the largest finite one, and the smallest of the lanes' largest
    float top = -INFINITY, low;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const float x = kept[j] ? (float)of_key64(kept[j]) : -INFINITY;
      top = x < INFINITY ? fmaxf(top, x) : top;
    }
    low = wave_min(top == -INFINITY ? INFINITY : top);
    top = wave_max(top);
    if (lane == 0) {
      sh.f[wave] = top;
      sh.f[NW + wave] = low;
    }
    __syncthreads();
    top = wave_max(sh.f[lane % NW]);
    low = wave_min(sh.f[NW + lane % NW]);
    if (seg <= VPL && r.want <= 48 && top > low && top - low < INFINITY) {
      const float scale = (float)(BINS - 1) / (top - low);
      // interval of a score, 0 the highest; the scores below `low` (or no numbers) count as the last
      auto bin_of = [&](uint64_t k) {
        const float y = (top - (float)of_key64(k)) * scale;
        return y < (float)(BINS - 1) ? (int)fmaxf(y, 0.f) : BINS - 1;
      };
#pragma unroll
      for (int j = 0; j < VPL; ++j)
        if (j < seg && kept[j]) atomicAdd(&sh.bin[bin_of(kept[j])], 1u);
      __syncthreads();
      // every wave: the first interval that, with those before it, holds `want`
      uint32_t c[BINS / 64], mine = 0;
#pragma unroll
      for (int x = 0; x < BINS / 64; ++x) mine += c[x] = sh.bin[lane * (BINS / 64) + x];
      uint32_t incl = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(incl, d, 64);
        if (lane >= d) incl += up;
      }
      const uint64_t enough = __ballot((int)incl >= r.want);
      int last = BINS, n_few = 0;
      if (enough) {
        const int l = __builtin_ctzll(enough);
        uint32_t sum = incl - mine;
        int at = BINS;
        uint32_t total = 0;
#pragma unroll
        for (int x = BINS / 64 - 1; x >= 0; --x) {
          uint32_t upto = sum;
#pragma unroll
          for (int y = 0; y <= x; ++y) upto += c[y];
          if ((int)upto >= r.want) {
            at = lane * (BINS / 64) + x;
            total = upto;
          }
        }
        last = __builtin_amdgcn_readlane(at, l);
        n_few = __builtin_amdgcn_readlane((int)total, l);
      }
      if (last < BINS - 1 && n_few <= 64) {
        // those scores in the order of their blocks
        int n = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
          if (j < seg) n += (int)__popcll(__ballot(kept[j] && bin_of(kept[j]) <= last));
        if (lane == 0) sh.f[wave] = (float)n;
        __syncthreads();
        int at = (int)wave_sum(lane < wave ? sh.f[lane % NW] : 0.f);
#pragma unroll
        for (int j = 0; j < VPL; ++j)
          if (j < seg) {
            const bool in = kept[j] && bin_of(kept[j]) <= last;
            const uint64_t m = __ballot(in);
            const int to = at + (int)__popcll(m & below);
            if (in && to < 64) {
              sh.key[to] = kept[j];
              sh.block[to] = 64 * (j0 + j) + lane;
            }
            at += (int)__popcll(m);
          }
        __syncthreads();
        if (wave == 0) {
          const uint64_t k = lane < n_few ? sh.key[lane] : 0ull;
          const int b = sh.block[lane];
          int rank = 0;
          for (int x = 0; x < n_few; ++x) {
            const uint64_t other = sh.key[x];
            rank += other > k || (other == k && x < lane);
          }
          const uint64_t m = __ballot(lane < n_few && rank < r.want);
          const int to = r.f_lo + (int)__popcll(m & below), free_end = r.f_lo + r.want;
          for (int t = lane; t < r.f_lo; t += 64) idx[t] = t;
          if ((m >> lane & 1) && to < top_k) idx[to] = b;
          for (int t = free_end + lane; t < top_k; t += 64)
            idx[t] = r.last0 + t - free_end < r.nb ? r.last0 + t - free_end : -1;
          if (lane == 0) *count = min(top_k, r.nb);
        }
        return;
      }
    }
    const double room = 1e-3 * ((double)top - low) + 1e-6 * fabs(top);
    double vlo = low - room, vhi = top + room;
    bool found = false;
    uint64_t t[3];
    int n[3];
    for (int step = 0; step < 12 && fabs(vlo) < INFINITY && fabs(vhi) < INFINITY; ++step) {
      const double d = 0.25 * (vhi - vlo);
#pragma unroll
      for (int x = 0; x < 3; ++x) t[x] = key64(vlo + d * (x + 1));
      if (!(t[0] > lo && t[2] < hi && t[0] < t[1] && t[1] < t[2])) break;
      reach(t, n);
      const int at = (n[0] >= r.want) + (n[1] >= r.want) + (n[2] >= r.want);
      if (at > 0) lo = at == 1 ? t[0] : at == 2 ? t[1] : t[2];
      if (at < 3) hi = at == 0 ? t[0] : at == 1 ? t[1] : t[2];
      found = at > 0 && (at == 1 ? n[0] : at == 2 ? n[1] : n[2]) == r.want;
      if (found) break;
      const double base = vlo;
      if (at > 0) vlo = base + d * at;
      if (at < 3) vhi = base + d * (at + 1);
    }
    while (!found && hi - lo > 1) {
      const uint64_t q = (hi - lo) >> 2, h = (hi - lo) >> 1;
      t[0] = lo + (q ? q : 1);
      t[1] = lo + h;
      t[2] = hi - (q ? q : 1);
      reach(t, n);
      const int at = (n[0] >= r.want) + (n[1] >= r.want) + (n[2] >= r.want);
      if (at > 0) lo = at == 1 ? t[0] : at == 2 ? t[1] : t[2];
      if (at < 3) hi = at == 0 ? t[0] : at == 1 ? t[1] : t[2];
      found = at > 0 && (at == 1 ? n[0] : at == 2 ? n[1] : n[2]) == r.want;
    }
    t[0] = t[1] = t[2] = lo + 1;
    reach(t, n);
    above = n[0];
  }
  // kept: forced, above lo, and the first want - above at lo
  int n_eq = 0, n_keep = 0;
  for (int j = 0; j < seg; ++j) {
    const uint64_t k = r.want > 0 ? key_at(j) : 0ull;
    n_eq += (int)__popcll(__ballot(k == lo));
    n_keep += (int)__popcll(__ballot(k > lo) | forced_bits(r, j0 + j));
  }
  __syncthreads();
  if (lane == 0) {
    sh.f[wave] = (float)n_eq;
    sh.f[NW + wave] = (float)n_keep;
  }
  __syncthreads();
  // entries of the waves before this one
  const int eq_before = (int)wave_sum(lane < wave ? sh.f[lane % NW] : 0.f);
  const int keep_before = (int)wave_sum(lane < wave ? sh.f[NW + lane % NW] : 0.f);
  int ties = r.want - above, out = keep_before + min(max(ties, 0), eq_before);
  ties -= eq_before;
  for (int j = 0; j < seg; ++j) {
    const uint64_t k = r.want > 0 ? key_at(j) : 0ull;
    const uint64_t eq = __ballot(k == lo), at_lo = __ballot(k == lo && (int)__popcll(eq & below) < ties);
    ties -= (int)__popcll(eq);
    const uint64_t m = __ballot(k > lo) | forced_bits(r, j0 + j) | at_lo;
    const int at = out + (int)__popcll(m & below);
    if ((m >> lane & 1) && at < top_k) idx[at] = 64 * (j0 + j) + lane;
    out += (int)__popcll(m);
  }
  const int n_all = min(top_k, r.nb);
  for (int t = n_all + tid; t < top_k; t += 64 * NW) idx[t] = -1;
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
template <class T, int D, int NW>
__device__ void score_row(const BlockSelectArgs& p, const T* q, const T* km, int a, int b, double* sc) {
  constexpr int EPL = 16 / sizeof(T), LPB = D / EPL, BPP = 64 * NW / LPB;
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
      s = group_sum64<LPB>(s);
      if (__any(!(fabs(s) < INFINITY))) {
        double t = 0.0;
        for (int h = 0; h < G; ++h) {
          const u32x4 w = gload((const u32x4*)(q + h * D + c * EPL));
#pragma unroll
          for (int e = 0; e < EPL; ++e) t += (double)chunk_val<T>(w, e) * (double)chunk_val<T>(v[u], e);
        }
        t = group_sum64<LPB>(t);
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
__global__ __launch_bounds__(64 * NWR) void k_select_row(BlockSelectArgs p, int per) {
  extern __shared__ double sc[];
  __shared__ PickLds<NWR> sh;
  const int64_t row = p.row0 + folded_block(), oi = row / p.H_kv;
  if (row >= p.end) return;
  const int g = (int)(row - oi * p.H_kv);
  const RowRange r = row_range(p, oi);
  const int a = max(SPLIT ? (int)blockIdx.z * per : 0, r.f_lo), b = min(SPLIT ? (int)(blockIdx.z + 1) * per : r.nb, r.last0);
  double* out = SPLIT ? p.score + (row - p.row0) * p.n_blk : sc;
  if (r.want > 0 && a < b) score_row<T, D, NWR>(p, query_of<T>(p, oi, g, D), means_of<T>(p, oi, g, D), a, b, out);
  if constexpr (!SPLIT) {
    __syncthreads();
    pick_row<NWR>(sc, r, p.top_k, p.idx + row * p.top_k, p.count + row, sh);
  }
}

// The lists from scores in the workspace.
__global__ __launch_bounds__(64 * NWR) void k_select_pick(BlockSelectArgs p) {
  __shared__ PickLds<NWR> sh;
  const int64_t row = p.row0 + folded_block();
  if (row >= p.end) return;
  pick_row<NWR>(p.score + (row - p.row0) * p.n_blk, row_range(p, row / p.H_kv), p.top_k, p.idx + row * p.top_k, p.count + row, sh);
}

__device__ __forceinline__ int pop(bool x) { return (int)__popcll(__ballot(x)); }

__device__ __forceinline__ u32x2 split_bf16(float a, float b) {   // (hi pair, lo pair)
  const uint32_t hi = pack_bf16x2(a, b);
  return u32x2{hi, pack_bf16x2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u))};
}

// Quarters (vlo, vhi) until between `want` and `most` of the values reach vlo
// (true) or the interval is no longer than eps (false).  `want` values reach vlo
// and fewer reach vhi before and after.  NV values a lane, and more(j) for j from
// NV below seg.
template <int NV, class More>
__device__ __forceinline__ bool narrow(const float (&v)[NV], int seg, More more, int want, int most, float eps, float& vlo,
                                       float& vhi) {
  for (int step = 0; step < 64 && vhi - vlo > eps; ++step) {
    const float d = 0.25f * (vhi - vlo), t0 = vlo + d, t1 = vlo + 2.f * d, t2 = vlo + 3.f * d;
    int n0 = 0, n1 = 0, n2 = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j < seg) {
        n0 += pop(v[j] >= t0);
        n1 += pop(v[j] >= t1);
        n2 += pop(v[j] >= t2);
      }
    for (int j = NV; j < seg; ++j) {
      const float x = more(j);
      n0 += pop(x >= t0);
      n1 += pop(x >= t1);
      n2 += pop(x >= t2);
    }
    int n = most + 1;
    if (n2 >= want) {
      vlo = t2;
      n = n2;
    } else if (n1 >= want) {
      vlo = t1;
      vhi = t2;
      n = n1;
    } else if (n0 >= want) {
      vlo = t0;
      vhi = t1;
      n = n0;
    } else {
      vhi = t0;
    }
    if (n <= most) return true;
  }
  return false;
}

// TR (32, 16, 8 or 4) queries of one (object, key head) per work-group.  LDS, in
// turn: the queries, summed over their heads and split into two bf16 terms; the
// scores [TR][pitch]; fp64 scores of a hard row.  Queries of 256 channels stay in
// LDS in front of the scores: in registers they would leave room for one
// work-group per CU (1693 queries of 8 heads, 135 blocks: 36 us, so 25).
template <class T, int D>
__global__ __launch_bounds__(64 * NWS, 4) void k_select_tile(BlockSelectArgs p, int TR, int n_tile, int pitch) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NQ = D / 16;
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  __shared__ float qn[32], kn[NWS];
  __shared__ PickLds<NWS> sh;
  __shared__ int hard[32], n_hard, seen[32];
  __shared__ u32x4 room[NWS][64];   // of each wave: mean keys on their way, later a row's few scores
  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t bid = folded_block(), og = bid / n_tile;
  if (og >= (int64_t)p.n_obj * p.H_kv) return;
  const int q0 = (int)(bid - og * n_tile) * TR, G = p.H / p.H_kv;
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
  if (lane < nr) {
    nbm = row_range(p, o * p.n_q + q0 + lane).nb;
    if (wave == 0) seen[lane] = nbm;
  }
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) nbm = max(nbm, __shfl_xor(nbm, m, 64));
  __syncthreads();
  const bool two = !BF || G > 1;   // one bf16 head is its own first term
  constexpr bool QREG = D <= 128;
  auto query = [&](int k) { return (const u32x4*)lds + l31 * CPQ + ((2 * k + half) ^ Swz<CPQ>::k(l31)); };
  u32x4 qh[QREG ? NQ : 1], ql[QREG ? NQ : 1];
  if constexpr (QREG) {
#pragma unroll
    for (int k = 0; k < NQ; ++k) {
      qh[k] = query(k)[0];
      ql[k] = two ? query(k)[32 * CPQ] : u32x4{0, 0, 0, 0};
    }
    __syncthreads();
  }
  float* sc = (float*)(lds + (QREG ? 0 : select_query_lds(D)));
  float k2 = 0.f;   // the largest squared norm of a mean key
  for (int bt = wave; bt * 32 < nbm; bt += NWS) {
    const T* kp = km + (int64_t)min(bt * 32 + l31, nbm - 1) * D + 8 * half;
    // bf16: four lanes read 64 bytes of a row (a quarter of the cycles in the address
    // unit), 16 rows at a time go through LDS to the lanes of their chunks
    const T* kq[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      kq[h] = km + (int64_t)min(bt * 32 + 16 * h + (lane >> 2), nbm - 1) * D + 8 * (((lane & 3) ^ (lane >> 4)) & 3);
    u32x4* mine = room[wave];
    f32x16 acc;
    float kk = 0.f;
    constexpr int KB = BF ? (NQ < 8 ? NQ : 8) : (NQ < 4 ? NQ : 4);
#pragma unroll
    for (int k0 = 0; k0 < NQ; k0 += KB) {
      u32x4 a[KB][BF ? 1 : 2];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        if constexpr (BF) {
          a[k][0] = gload((const u32x4*)(kq[k & 1] + 16 * (k0 + (k & ~1))));
        } else {
#pragma unroll
          for (int y = 0; y < 2; ++y) a[k][y] = gload((const u32x4*)(kp + 16 * (k0 + k)) + y);
        }
      }
      if constexpr (BF) {
#pragma unroll
        for (int k = 0; k < KB; k += 2) {
          u32x4 to[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            mine[lane] = a[k + h][0];
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");   // a wave's LDS accesses take place in order
            if ((l31 >> 4) == h) {
#pragma unroll
              for (int j = 0; j < 2; ++j) to[j] = mine[(l31 & 15) * 4 + (((2 * j + half) ^ (l31 >> 2)) & 3)];
            }
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
          }
          a[k][0] = to[0];
          a[k + 1][0] = to[1];
        }
      }
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
        const u32x4 hi = QREG ? qh[QREG ? ks : 0] : query(ks)[0];
        acc = mfma32(ah, hi, ks == 0 ? f32x16{} : acc);
        if (two) acc = mfma32(ah, QREG ? ql[QREG ? ks : 0] : query(ks)[32 * CPQ], acc);
        if constexpr (!BF) acc = mfma32(al, hi, acc);
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
    const RowRange rr = range_of(p, seen[r]);
    const float* srow = sc + r * pitch;
    int32_t* idx = p.idx + row * p.top_k;
    const float eps2 = keps * (qn[r] + 0x1p-60f) + 0x1p-100f;   // twice the bound
    const int seg = (rr.nb + 63) / 64;
    auto val_at = [&](int j) {   // of the blocks that are to be chosen from
      const int b = 64 * j + lane;
      return b >= rr.f_lo && b < rr.last0 ? srow[b] : -INFINITY;
    };
    constexpr int NV = 2 * VPL;
    float kept[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) kept[j] = j < seg ? val_at(j) : -INFINITY;
    // The query in fp64, a stretch of channels per lane, for scores made again.
    constexpr int E = D < 64 ? 1 : D / 64;
    double qd[E];
    auto query64 = [&]() {
#pragma unroll
      for (int e = 0; e < E; ++e) qd[e] = 0.0;
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (lane < D) qd[e] += (double)to_f32<T>(gload(qbase + r * p.qs + h * D + lane + 64 * e));
    };
    auto score64 = [&](int b) {
      const T* kp = km + (int64_t)b * D;
      double s = 0.0;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane < D) s += qd[e] * (double)to_f32<T>(gload(kp + lane + 64 * e));
      return group_sum64<64>(s);
    };
    // The scores from t on, one per lane in the order of their blocks; false if
    // there are more than 64.
    float x = -INFINITY;
    int xb = 0;
    u32x2* few = (u32x2*)room[wave];
    auto compact_row = [&](const float (&v)[NV], int n_seg, auto more, float t) {
      int n = 0;
      auto put = [&](int j, float y) {
        const uint64_t m = __ballot(y >= t);
        if (m == 0) return;
        const int at = n + (int)__popcll(m & below);
        if (y >= t && at < 64) few[at] = u32x2{__float_as_uint(y), (uint32_t)(64 * j + lane)};
        n += (int)__popcll(m);
      };
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (j < n_seg) put(j, v[j]);
      for (int j = NV; j < n_seg; ++j) put(j, more(j));
      if (n > 64) return false;
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): written and read by this wave alone
      __builtin_amdgcn_wave_barrier();
      const u32x2 y = few[lane];
      __builtin_amdgcn_wave_barrier();
      x = lane < n ? __uint_as_float(y[0]) : -INFINITY;
      xb = (int)y[1];
      return true;
    };
    auto done_row = [&](float vlo, float vhi) {
      const float one[1] = {x};
      const bool found = narrow(one, 1, [](int) { return -INFINITY; }, rr.want, rr.want, eps2, vlo, vhi);
      uint64_t m = __ballot(x >= vlo);
      bool clear = found;
      if (found) {
        const float kth = wave_min(x >= vlo ? x : INFINITY), next = wave_max(x >= vlo ? -INFINITY : x);
        clear = kth - next > eps2;
        vlo = vhi = kth;
      }
      if (!clear) {   // between vlo - eps2 and vhi + eps2 the fp64 scores decide
        const float w_lo = vlo - eps2, w_hi = vhi + eps2;
        m = __ballot(x >= w_hi);
        const uint64_t im = __ballot(x >= w_lo && x < w_hi);
        const int need = rr.want - (int)__popcll(m);
        query64();
        double mine = 0.0;
        for (uint64_t q = im; q; q &= q - 1) {
          const int l = __builtin_ctzll(q);
          const double s = score64(__builtin_amdgcn_readlane(xb, l));
          if (lane == l) mine = s;
        }
        const uint64_t mk = key64(mine);
        int rank = 0;
        for (uint64_t q = im; q; q &= q - 1) {
          const int l = __builtin_ctzll(q);
          const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mk >> 32), l) << 32 |
                                 (uint32_t)__builtin_amdgcn_readlane((int)mk, l);
          rank += other > mk || (other == mk && l < lane);
        }
        m |= __ballot((im >> lane & 1) && rank < need);
      }
      const int n = rr.f_lo + (int)__popcll(m), at = rr.f_lo + (int)__popcll(m & below);
      for (int t = lane; t < rr.f_lo; t += 64) idx[t] = t;
      if ((m >> lane & 1) && at < p.top_k) idx[at] = xb;
      for (int t = n + lane; t < p.top_k; t += 64) idx[t] = rr.last0 + t - n < rr.nb ? rr.last0 + t - n : -1;
      if (lane == 0) p.count[row] = n + rr.nb - rr.last0;
    };
    // scores from w_hi on are kept, and `need` of the `cand` ones from w_lo to below it
    // (where the forced blocks fill the list, none: no score compares with NaN)
    bool is_hard = false;
    int cand = 0, need = 0;
    float w_lo = NAN, w_hi = NAN;
    if (rr.want > 0) {
      if (!(qn[r] * sqrtf(k2) < 1e38f)) {   // a score may leave the fp32 range, or is no number
        is_hard = true;
      } else {
        float top = kept[0];
#pragma unroll
        for (int j = 1; j < NV; ++j)
          if (j < seg) top = __builtin_elementwise_maximum(top, kept[j]);
        for (int j = NV; j < seg; ++j) top = __builtin_elementwise_maximum(top, val_at(j));
        const float low = wave_min(top);   // 64 scores reach it, if each lane has one
        float vhi = wave_max(top) + eps2, vlo = rr.want <= 64 && low > -INFINITY ? low : -1.02f * qn[r] * sqrtf(k2) - eps2;
        // few are wanted: a value that the largest of at most 32 lanes reach (about 44
        // scores, if they lie anyhow), and then on with the scores from there, one per lane
        if (rr.want <= 32 && low > -INFINITY) {
          const float one[1] = {top};
          float a = vlo, b = vhi;
          narrow(one, 1, [](int) { return -INFINITY; }, rr.want, 32, eps2, a, b);
          if (compact_row(kept, seg, val_at, a - eps2)) {
            done_row(a, vhi);
            continue;
          }
        }
        // else first a value that at most 48 scores reach, and then on with
        // those alone, one per lane
        if (rr.want <= 48 && narrow(kept, seg, val_at, rr.want, 48, eps2, vlo, vhi) &&
            compact_row(kept, seg, val_at, vlo - eps2)) {
          done_row(vlo, vhi);
          continue;
        }
        bool found = narrow(kept, seg, val_at, rr.want, rr.want, eps2, vlo, vhi);
        if (found) {   // the want-th score and the next
          float kth = INFINITY, next = -INFINITY;
#pragma unroll
          for (int j = 0; j < NV; ++j)
            if (j < seg) {
              kth = __builtin_elementwise_minimum(kth, kept[j] >= vlo ? kept[j] : INFINITY);
              next = __builtin_elementwise_maximum(next, kept[j] >= vlo ? -INFINITY : kept[j]);
            }
          for (int j = NV; j < seg; ++j) {
            const float v = val_at(j);
            kth = fminf(kth, v >= vlo ? v : INFINITY);
            next = fmaxf(next, v >= vlo ? -INFINITY : v);
          }
          kth = wave_min(kth);
          next = wave_max(next);
          if (kth - next > eps2) {
            w_lo = w_hi = kth;   // the scores from kth on are kept
          } else {
            vlo = vhi = kth;
            found = false;
          }
        }
        if (!found) {
          w_lo = vlo - eps2;
          w_hi = vhi + eps2;
          int sure = 0, reach = 0;
#pragma unroll
          for (int j = 0; j < NV; ++j)
            if (j < seg) {
              sure += pop(kept[j] >= w_hi);
              reach += pop(kept[j] >= w_lo);
            }
          for (int j = NV; j < seg; ++j) {
            const float v = val_at(j);
            sure += pop(v >= w_hi);
            reach += pop(v >= w_lo);
          }
          cand = reach - sure;
          need = rr.want - sure;
          is_hard = cand > 64;
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
      query64();
      double mine = 0.0;
      int c = 0;
      for (int j = 0; j < seg; ++j) {
        const float v = val_at(j);
        for (uint64_t m = __ballot(v >= w_lo && v < w_hi); m; m &= m - 1, ++c) {
          const double s = score64(64 * j + __builtin_ctzll(m));
          if (lane == c) mine = s;
        }
      }
      const uint64_t mk = key64(mine);
      int rank = 0;
      for (int l = 0; l < cand; ++l) {
        const uint64_t other = (uint64_t)__shfl((long long)mk, l, 64);
        rank += other > mk || (other == mk && l < lane);
      }
      win = __ballot(lane < cand && rank < need);
    }
    int out = 0, c = 0;
    auto emit = [&](int j, float v) {
      uint64_t m = __ballot(v >= w_hi) | forced_bits(rr, j);
      if (cand > 0) {
        const bool in = v >= w_lo && v < w_hi;
        const uint64_t im = __ballot(in);
        if (im) m |= __ballot(in && (win >> (c + (int)__popcll(im & below)) & 1));
        c += (int)__popcll(im);
      }
      if (m == 0) return;
      const int at = out + (int)__popcll(m & below);
      if ((m >> lane & 1) && at < p.top_k) idx[at] = 64 * j + lane;
      out += (int)__popcll(m);
    };
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j < seg) emit(j, kept[j]);
    for (int j = NV; j < seg; ++j) emit(j, val_at(j));
    for (int t = out + lane; t < p.top_k; t += 64) idx[t] = -1;
    if (lane == 0) p.count[row] = out;
  }
  __syncthreads();
  // hard rows: every score in fp64, by the whole work-group
  double* sd = (double*)lds;
  for (int x = 0; x < n_hard; ++x) {
    const int r = hard[x];
    const int64_t oi = o * p.n_q + q0 + r, row = oi * p.H_kv + g;
    const RowRange rr = range_of(p, seen[r]);
    score_row<T, D, NWS>(p, qbase + r * p.qs, km, rr.f_lo, rr.last0, sd);
    __syncthreads();
    pick_row<NWS>(sd, rr, p.top_k, p.idx + row * p.top_k, p.count + row, sh);
    __syncthreads();
  }
}

template <class T, int D>
hipError_t launch(BlockSelectArgs a, const BlockSelectPlan& pl, hipStream_t st) {
  const int64_t rows = (int64_t)a.n_obj * a.n_q * a.H_kv;
  a.row0 = 0;
  a.end = rows;
  if (pl.tile) {
    const int n_tile = (a.n_q + pl.TR - 1) / pl.TR;
    const int64_t n = (int64_t)a.n_obj * a.H_kv * n_tile;
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_tile<T, D>), folded(n), dim3(64 * NWS), pl.lds, st, a, pl.TR,
               n_tile, pl.pitch);
  } else if (pl.split > 1) {
    for (; a.row0 < rows; a.row0 += pl.at_once) {
      const int64_t n = std::min(pl.at_once, rows - a.row0);
      a.end = a.row0 + n;
      RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_row<T, D, true>), folded(n, pl.split), dim3(64 * NWR), 0, st, a,
                 (a.n_blk + pl.split - 1) / pl.split);
      RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, k_select_pick, folded(n), dim3(64 * NWR), 0, st, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  } else {
    RS3_LAUNCH(RS3_K_BLOCK_SELECT, st, (k_select_row<T, D, false>), folded(rows), dim3(64 * NWR), pl.lds, st, a, a.n_blk);
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

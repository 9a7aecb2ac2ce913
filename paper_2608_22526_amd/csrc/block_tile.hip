// Block-sparse attention of many queries: the lists are turned round, so that
// a work-group holds one block of keys and values in LDS and computes it for
// 128 of the (query, head) rows that list it.
//
//  k_block_count, k_block_scatter : the queries of every block, and the tiles;
//  k_block_tile  : softmax and value product of one block for 128 rows, a
//                  partial row (m, l, O) for each;
//  k_block_merge : the partials of a query joined.
//
// A query-major form reads its blocks anew for every query (64 KB of L2 for 64
// keys of 128 channels and one query head); here a block is read once per 128
// rows, and what moves is a row of Q and a partial row for every (query, head,
// listed block).
//
// 4096 queries, two heads of 128, 32 of 448 blocks of 64 keys in 55 us: counters 4,
// lists 5 + 6, tiles 30 (262144 rows, 0.29 PFLOP/s), merge 13.5 (67 MB, 5 TB/s); all
// pairs of these queries and keys take the dense kernel 125.  8192 prompt tokens, 16
// heads of 128 to 4 key heads, 16 of up to 512 blocks in 305 to 313: tiles 2 x 110, merge 2 x
// 45.  No one unit bounds the tiles: a row moves 256 bytes of Q, 256 of its partial and
// its share of 256 of the keys and values (address unit busy 57 % of the time; without
// the stores 24 and 80 us), vector instructions issue in 40 % of the cycles, products
// take 15 %.
#include "block.h"

namespace rs3 {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Consecutive tiles of one XCD (mostly of one block, so that its L2 serves them).
// Runs of 8 spread a chunk's long and short lists better than an eighth of the tiles
// for each XCD: tiles of the prompt, grid and fp32 grid 112/28.8/16.9 us against
// 114/30.5/18.9.
constexpr int XCD_RUN = 8;

// The blocks' counters to 0 (a kernel, which a graph can hold).
__global__ __launch_bounds__(256) void k_block_zero(uint32_t* total, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) total[i] = 0;
}

// grid (groups, runs of all chunks), 512 threads, n_blk counters in LDS.  Entries
// that take no part (out of range, not ascending, past the count, not seen) get
// no place and an empty partial.
__global__ __launch_bounds__(512) void k_block_count(BlockAttendArgs p, BlockTileArgs w, BlockPartArgs part) {
  extern __shared__ uint32_t sc[];
  const int grp = blockIdx.x, o = grp / p.H_kv, hk = grp - o * p.H_kv, tid = threadIdx.x;
  const int ch = blockIdx.y / w.runs, q0 = ch * w.chunk + (blockIdx.y - ch * w.runs) * w.run;
  const int items = max(min(w.run, min((ch + 1) * w.chunk, p.n_q) - q0), 0) * p.slots;
  for (int b = tid; b < p.n_blk; b += 512) sc[b] = 0;
  __syncthreads();
  constexpr int U = 4;   // entries of a thread in flight
  for (int e0 = tid; e0 < items; e0 += U * 512) {
    int b[U], prev[U], cnt[U], vis[U], t[U];
    int64_t row[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int e = min(e0 + 512 * k, items - 1), iq = e / p.slots;
      const int64_t oi = (int64_t)o * p.n_q + q0 + iq;
      t[k] = e - iq * p.slots;
      row[k] = oi * p.H_kv + hk;
      const int32_t* list = p.idx + row[k] * p.top_k;
      b[k] = gload(list + t[k]);
      prev[k] = gload(list + max(t[k] - 1, 0));
      cnt[k] = gload(p.count + row[k]);
      vis[k] = visible_keys(p.n_vis, oi, p.n_kv);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (e0 + 512 * k >= items) break;
      const bool ok = t[k] < min(cnt[k], p.slots) && b[k] >= 0 && b[k] < p.n_blk && (t[k] == 0 || b[k] > prev[k]) &&
                      (int64_t)b[k] * p.block < vis[k];
      uint32_t at = ~0u;
      if (ok) {
        at = atomicAdd(&sc[b[k]], 1u) * BLOCK_TILE_MAX + (uint32_t)b[k];
      } else {
        float* ml = part.ML + (row[k] * p.slots + t[k]) * p.G * 2;
        for (int g = 0; g < p.G; ++g) {
          ml[2 * g] = -INFINITY;
          ml[2 * g + 1] = 0.f;
        }
      }
      w.ord[((int64_t)grp * p.n_q + q0) * p.slots + e0 + 512 * k] = at;
    }
  }
  __syncthreads();
  // the run's place among the chunk's: in the order in which the runs come by,
  // which decides where a row is computed and nothing else
  uint32_t* total = w.total + ((int64_t)ch * w.groups + grp) * p.n_blk;
  uint32_t* base = w.base + ((int64_t)blockIdx.y * w.groups + grp) * p.n_blk;
  for (int b = tid; b < p.n_blk; b += 512)
    if (sc[b]) base[b] = atomicAdd(total + b, sc[b]);
}

// Same grid: the run's entries into the lists; each chunk's first run writes the
// tiles.  LDS: where this run's queries of each block begin, the blocks' counts
// and first tiles.
__global__ __launch_bounds__(512) void k_block_scatter(BlockAttendArgs p, BlockTileArgs w) {
  extern __shared__ uint32_t sm[];
  __shared__ uint32_t wsum[8], ntile;
  uint32_t* pre = sm;
  uint32_t* tot = sm + p.n_blk;
  const int ch = blockIdx.y / w.runs, run = blockIdx.y - ch * w.runs, grp = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t cg = (int64_t)ch * w.groups + grp;
  for (int b = tid; b < p.n_blk; b += 512) {
    tot[b] = gload(w.total + cg * p.n_blk + b);
    pre[b] = gload(w.base + ((int64_t)blockIdx.y * w.groups + grp) * p.n_blk + b);   // (anything, where it has none)
  }
  const int q0 = ch * w.chunk + run * w.run;
  const int items = max(min(w.run, min((ch + 1) * w.chunk, p.n_q) - q0), 0) * p.slots;
  const uint32_t* ord = w.ord + ((int64_t)grp * p.n_q + q0) * p.slots;
  uint32_t at4[4];   // in flight during the scan
#pragma unroll
  for (int k = 0; k < 4; ++k) at4[k] = tid + 512 * k < items ? gload(ord + tid + 512 * k) : ~0u;
  __syncthreads();
  // exclusive scan of the blocks' tiles, a stretch of blocks per thread; a tile's
  // queries begin at tq times its number in the list
  const uint32_t tq = w.tq;
  const int per = (p.n_blk + 511) / 512, b0 = min(tid * per, p.n_blk), b1 = min(b0 + per, p.n_blk);
  uint32_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += (tot[b] + tq - 1) / tq;
  uint32_t incl = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(incl, d, 64);
    if (lane >= d) incl += up;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  uint32_t at = incl - mine;
  for (int i = 0; i < wave; ++i) at += wsum[i];
  if (tid == 511) ntile = at + mine;
  uint32_t* first = sm + 2 * p.n_blk;   // first tile of each block
  for (int b = b0; b < b1; ++b) {
    first[b] = at;
    pre[b] += at * tq;
    at += (tot[b] + tq - 1) / tq;
  }
  __syncthreads();
  if (run == 0) {
    BlockTile* tiles = w.tiles + cg * w.tcap;
    for (uint32_t t = tid; t < (uint32_t)w.tcap; t += 512) {
      BlockTile e;
      e.b = -1;
      e.n = 0;
      if (t < ntile) {   // its block: the last whose first tile is not past t
        int lo = 0, hi = p.n_blk;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (first[mid] <= t) lo = mid;
          else hi = mid;
        }
        e.b = lo;
        e.n = (int)min(tot[lo] - (t - first[lo]) * tq, tq);
      }
      tiles[t] = e;
    }
  }
  uint32_t* list = w.list + cg * w.tcap * tq;
  for (int e0 = tid; e0 < items; e0 += 2048) {
    if (e0 > tid) {
#pragma unroll
      for (int k = 0; k < 4; ++k) at4[k] = e0 + 512 * k < items ? gload(ord + e0 + 512 * k) : ~0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (at4[k] != ~0u)
        list[pre[at4[k] % BLOCK_TILE_MAX] + at4[k] / BLOCK_TILE_MAX] = (uint32_t)(run * w.run * p.slots + e0 + 512 * k);
  }
}

// The (m, l) pair of a partial whose values are f16 times 2^e (device_util.h,
// at part_sum); a sum that is no number is handed on in m.
__device__ __forceinline__ void encode_ml(float m, float l, int e, float* out) {
  if (l > 0.f) {
    const int el = __builtin_amdgcn_frexp_expf(l) - 1;
    m += (float)el;
    l = __builtin_amdgcn_ldexpf(l, e - el);
  } else {
    m = l == 0.f ? -INFINITY : NAN;
    l = 0.f;
  }
  *(float2*)out = make_float2(m, l);
}

// The power of two of a row whose largest finite value is `big`: row / 2^e < 2^15.
__device__ __forceinline__ int row_exp(float big) { return max(__builtin_amdgcn_frexp_expf(big) - 15, -126); }

// One partial row by the whole wave, key by key: for rows that do not see all
// of the block where a product with weight 0 was no number (Inf or NaN in a
// value that the row does not see).
template <class T, int D>
__device__ __noinline__ void careful_row(const T* q, const T* k, int64_t ks, const T* v, int64_t vs, int keys,
                                         float qscale, void* orow, float* ml) {
  constexpr int E = D < 64 ? 1 : D / 64;
  const int lane = threadIdx.x & 63;
  const bool on = lane < D;
  float qv[E], acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    qv[e] = on ? to_f32<T>(q[lane + 64 * e]) : 0.f;
    acc[e] = 0.f;
  }
  for (int pass = 0; pass < 2; ++pass) {
    const float sub = m == -INFINITY ? 0.f : m;
    for (int j = 0; j < keys; ++j) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) s += on ? qv[e] * to_f32<T>(k[j * ks + lane + 64 * e]) : 0.f;
      s = wave_sum(s) * qscale;
      if (pass == 0) {
        m = __builtin_elementwise_maximum(m, s);
        continue;
      }
      const float w = __builtin_amdgcn_exp2f(s - sub);
      l += w;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += on ? w * to_f32<T>(v[j * vs + lane + 64 * e]) : 0.f;
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  float big = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    acc[e] *= inv;
    const float x = __builtin_fabsf(acc[e]);
    big = x < INFINITY ? fmaxf(big, x) : big;
  }
  const int ex = row_exp(wave_max(big));
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (!on) break;
    if constexpr (sizeof(T) == 2)
      ((_Float16*)orow)[lane + 64 * e] = (_Float16)__builtin_amdgcn_ldexpf(acc[e], -ex);
    else
      ((float*)orow)[lane + 64 * e] = acc[e];
  }
  if (lane == 0) {
    if constexpr (sizeof(T) == 2) encode_ml(m, l, ex, ml);
    else *(float2*)ml = make_float2(l == 0.f ? -INFINITY : m, l);
  }
}

// LDS of a work-group: the stage, and after the products for each wave 32 rows
// of a segment of its partial rows (128 bytes, or the whole of a 64-byte row); behind
// them 2 KB per wave by which the queries come.
template <class T, int D, int NT, int NW>
struct TileLayout {
  static constexpr int CPR = D * (int)sizeof(T) / 16, ROWS = 32 * NT;
  static constexpr int VOFF = ROWS * CPR * 16, STAGE = 2 * VOFF;
  static constexpr int SEG = CPR < 8 ? CPR : 8;   // chunks of a segment
  static constexpr int OUT = NW * 32 * SEG * 16;
  static constexpr int QOFF = STAGE > OUT ? STAGE : OUT, BYTES = QOFF + NW * 2048;
  // chunk c of row r lies at chunk c ^ f(r): 16 rows at one chunk, or whole rows, per LDS cycle
  static __device__ __forceinline__ int f(int r) { return (r / (16 / SEG)) & (SEG - 1); }
};

// NW waves of 32 rows; NT 32-key tiles per stage; ONE: the block is one stage.
// Logits transposed, S^T = K Q^T, so that the weights feed O^T += V^T P^T from
// their registers (in bf16 the value operand comes from the rows of V by
// transposed LDS reads); a row of the partial is one lane pair.  In bf16 the weights
// are rounded for the products and summed as rounded, and partials are f16 times a
// power of two of the row's own: 2^-11 of their largest values at most, an eighth of
// what O's rounding to bf16 takes.  The merge reads them past the caches, where this
// kernel leaves them (prompt: both plain 331 us, only stored past the caches 328, both
// past them 312, so 308; grid 60, 62, 55, 55).
template <class T, int D, int NT, int NW, bool ONE>
__global__ __launch_bounds__(64 * NW, D * sizeof(T) <= 256 ? (D * sizeof(T) <= 128 || ONE ? 4 : 3) : 1) void k_block_tile(
    BlockAttendArgs p, BlockTileArgs w, BlockPartArgs part) {
  using L = TileLayout<T, D, NT, NW>;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int CPR = L::CPR, NDT = D / 32, NQ = BF ? D / 16 : D / 8, TH = 64 * NW;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  // XCD_RUN consecutive tiles go to one XCD
  const int64_t n_item = (int64_t)w.groups * w.tcap;
  const int turn = blockIdx.x >> 3;
  const int64_t it = ((int64_t)(turn / XCD_RUN) * 8 + (blockIdx.x & 7)) * XCD_RUN + turn % XCD_RUN;
  if (it >= n_item) return;
  const int grp = (int)(it / w.tcap);
  const int64_t tile = (int64_t)w.ch * n_item + it;
  const int b = sload(&w.tiles[tile].b), rows = sload(&w.tiles[tile].n) * p.G;
  const int o = grp / p.H_kv, hk = grp - o * p.H_kv;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, l31 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // this lane's row: list entry, then query, keys seen, partial row
  const int row0 = wave * 32;
  const uint32_t lrow = (uint32_t)(row0 + l31), e = min(lrow / (uint32_t)p.G, (uint32_t)w.tq - 1);
  uint32_t ent = gload(w.list + tile * w.tq + e);   // (read beside the tile: a place without a query holds anything)
  if (b < 0) return;
  const int64_t j0 = (int64_t)b * p.block;
  const T* Kg = (const T*)p.K + o * p.ko + (int64_t)hk * D;
  const T* Vg = (const T*)p.V + o * p.vo + (int64_t)hk * D;
  // value rows: in bf16 four keys x 64 bytes per cycle, in fp32 two keys (4
  // apart) x 128 bytes
  auto fv = [](int r) { return BF ? Swz<CPR>::template v<CPR < 4 ? CPR : 4, 0>(r) : Swz<CPR>::template v<8, 2>(r); };
  // Direct-to-LDS loads: load i of a wave covers 64 chunks, RPL rows after load
  // i - 1; the swizzle repeats with every P loads, so that the lane's
  // offsets are P numbers added to uniform addresses.  Rows past the last key
  // read it again; no row sees them.
  constexpr int NL = (L::ROWS * CPR + TH - 1) / TH, RPL = TH / CPR, P = RPL >= 16 ? 1 : 16 / RPL;
  const int c0 = wave * 64 + lane, r0 = c0 / CPR, x0 = c0 % CPR;
  const int ksb = (int)p.ks * (int)sizeof(T), vsb = (int)p.vs * (int)sizeof(T);   // row strides below 2^24 bytes
  int ko[P], vo[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    ko[i] = r0 * ksb + 16 * (x0 ^ Swz<CPR>::k(r0 + i * RPL));
    vo[i] = r0 * vsb + 16 * (x0 ^ fv(r0 + i * RPL));
  }
  auto fill = [&](int st) {
    const int64_t j = j0 + st * L::ROWS;
    const uint8_t* kb = (const uint8_t*)(Kg + j * p.ks);
    const uint8_t* vb = (const uint8_t*)(Vg + j * p.vs);
    const int past = (int)max(j + L::ROWS - p.n_kv, (int64_t)0);   // rows of the stage that are not there
    if (past == 0) {
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (L::ROWS * CPR >= TH * (i + 1) || wave * 64 < L::ROWS * CPR - TH * i)
          dma16(kb + (int64_t)i * RPL * ksb + ko[i % P], lds + (wave * 64 + TH * i) * 16);
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (L::ROWS * CPR >= TH * (i + 1) || wave * 64 < L::ROWS * CPR - TH * i)
          dma16(vb + (int64_t)i * RPL * vsb + vo[i % P], lds + L::VOFF + (wave * 64 + TH * i) * 16);
    } else {
      for (int i = 0; i < NL; ++i) {
        if (wave * 64 >= L::ROWS * CPR - TH * i) break;
        const int r = r0 + i * RPL, up = max(r - max(L::ROWS - past - 1, 0), 0);   // rows back to the last key
        const int64_t back = past >= L::ROWS ? r + 1 + (past - L::ROWS) : up;
        dma16(kb + (r - back) * ksb + 16 * (x0 ^ Swz<CPR>::k(r)), lds + (wave * 64 + TH * i) * 16);
        dma16(vb + (r - back) * vsb + 16 * (x0 ^ fv(r)), lds + L::VOFF + (wave * 64 + TH * i) * 16);
      }
    }
  };
  fill(0);
  const int i0 = w.ch * w.chunk;
  const bool there = row0 + l31 < rows;
  ent = there ? ent : 0;
  const int hg = there ? (int)(lrow - e * (uint32_t)p.G) : 0;
  const int qi = (int)(ent / (uint32_t)p.slots), slot = (int)(ent - (uint32_t)qi * p.slots);
  const int64_t oi = (int64_t)o * p.n_q + i0 + qi;
  const int lim = (int)min((int64_t)visible_keys(p.n_vis, oi, p.n_kv) - j0, (int64_t)p.block);
  const int prow = (((o * w.nq + qi) * p.H_kv + hk) * p.slots + slot) * p.G + hg;
  float* ml = part.ML + 2 * (((oi * p.H_kv + hk) * p.slots + slot) * p.G + hg);
  const T* Qo = (const T*)p.Q + o * p.qo + (int64_t)i0 * p.qs + (int64_t)hk * p.G * D;
  const T* qp = Qo + qi * p.qs + hg * D;
  // Q rows: four lanes read 64 bytes of one, a quarter of the cycles in the address
  // unit that 32 rows side by side take (prompt 320 -> 312 us); the lanes' own chunks
  // come by way of LDS, a segment of 32 rows x 64 bytes at a time (chunk c of row r at
  // c ^ r / 4).
  constexpr int NSEG = CPR / 4;
  static_assert(NQ == 2 * NSEG, "two chunks of a segment per lane");
  const int64_t qown = qi * p.qs + hg * D;
  const int qr = lane >> 2, qx = ((lane & 3) ^ (qr >> 2)) & 3;
  u32x4 q[NQ];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint8_t* qs = (const uint8_t*)(Qo + __shfl(qown, qr + 16 * h, 64)) + 16 * qx;
#pragma unroll
    for (int s = 0; s < NSEG; ++s) q[2 * s + h] = gload((const u32x4*)(qs + 64 * s));
  }
  uint8_t* qb = lds + L::QOFF + wave * 2048;
#pragma unroll
  for (int s = 0; s < NSEG; ++s) {
    *(u32x4*)(qb + lane * 16) = q[2 * s];
    *(u32x4*)(qb + 1024 + lane * 16) = q[2 * s + 1];
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");   // a wave's LDS accesses take place in order
#pragma unroll
    for (int j = 0; j < 2; ++j)
      q[2 * s + j] = *(const u32x4*)(qb + l31 * 64 + (((2 * j + g) ^ (l31 >> 2)) & 3) * 16);
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
  }
  f32x16 acc[NDT];
  if constexpr (!ONE) {
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) acc[dt] = f32x16{};
  }
  float m = -INFINITY, l = 0.f;
  const int n_st = ONE ? 1 : p.block / L::ROWS;
  for (int st = 0; st < n_st; ++st) {
    if (!ONE && st > 0) {
      stage_barrier();
      fill(st);
    }
    wait_vmcnt<0>();
    stage_barrier();
    if (row0 >= rows) continue;
    f32x16 sc[NT];
#pragma unroll
    for (int kt = 0; kt < NT; ++kt) {
#pragma unroll
      for (int k = 0; k < NQ; ++k) {
        const u32x4 a = *(const u32x4*)(lds + ((32 * kt + l31) * CPR + ((2 * k + g) ^ Swz<CPR>::k(l31))) * 16);
        if constexpr (BF) sc[kt] = mfma32(a, q[k], k == 0 ? f32x16{} : sc[kt]);
        else sc[kt] = mfma32f(__builtin_bit_cast(f32x4, a), __builtin_bit_cast(f32x4, q[k]), k == 0 ? f32x16{} : sc[kt]);
      }
    }
    const int left = lim - st * L::ROWS;
    if (__any(left < L::ROWS)) {
#pragma unroll
      for (int kt = 0; kt < NT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kt][r] = 32 * kt + c_row(r, lane) < left ? sc[kt][r] : -INFINITY;
    }
    float mx = sc[0][0];
#pragma unroll
    for (int kt = 0; kt < NT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; r += 2) mx = max3f(mx, sc[kt][r], sc[kt][r + 1]);
    const float mn = __builtin_elementwise_maximum(m, max_with_partner(mx) * p.qscale);
    const float sub = mn == -INFINITY ? 0.f : mn;
    const float alpha = __builtin_amdgcn_exp2f(m - sub);
    m = mn;
    l *= alpha;
    if (!ONE && st > 0) {
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) acc[dt] *= alpha;
    }
    if constexpr (BF) {
      u32x4 pk[2 * NT];
      float ts[2] = {0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < 2 * NT; ++ks)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float s0 = sc[ks >> 1][8 * (ks & 1) + 2 * x], s1 = sc[ks >> 1][8 * (ks & 1) + 2 * x + 1];
          pk[ks][x] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(s0, p.qscale, -sub)),
                                  __builtin_amdgcn_exp2f(__builtin_fmaf(s1, p.qscale, -sub)));
          ts[ks & 1] = add_bf16x2(pk[ks][x], ts[ks & 1]);
        }
      l += ts[0] + ts[1];
      const int kr = 4 * g + ((lane & 15) >> 2), f4 = fv(kr);   // the key row whose address this lane supplies
      const uint8_t* vb = lds + L::VOFF + kr * CPR * 16 + (lane & 1) * 8;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) {
        const uint8_t* va = vb + ((4 * dt + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) ^ f4) * 16;
#pragma unroll
        for (int ks = 0; ks < 2 * NT; ++ks) {
          const u32x2 lo = lds_tr4(va + 16 * ks * CPR * 16), hi = lds_tr4(va + (16 * ks + 8) * CPR * 16);
          acc[dt] = mfma32(u32x4{lo[0], lo[1], hi[0], hi[1]}, pk[ks], ONE && ks == 0 ? f32x16{} : acc[dt]);
        }
      }
    } else {
#pragma unroll
      for (int kt = 0; kt < NT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sc[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][r], p.qscale, -sub));
          l += sc[kt][r];
        }
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int kt = 0; kt < NT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int kr = 32 * kt + c_row(r, lane);
            const float a = *(const float*)(lds + L::VOFF + (kr * CPR + ((8 * dt + (l31 >> 2)) ^ fv(kr))) * 16 + (l31 & 3) * 4);
            acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, sc[kt][r], ONE && kt == 0 && r == 0 ? f32x16{} : acc[dt], 0, 0, 0);
          }
    }
  }
  stage_barrier();   // the stage is free
  if (row0 >= rows) return;
  l = sum_with_partner(l);
  const float inv = l > 0.f ? __builtin_amdgcn_rcpf(l) : 0.f;
  float big = 0.f;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; r += 2) big = max3f(big, __builtin_fabsf(acc[dt][r]), __builtin_fabsf(acc[dt][r + 1]));
  big = max_with_partner(big);   // NaN if any value is
  bool store = there;
  if (__any(!(big < INFINITY))) {
    uint64_t todo = __ballot(store && g == 0 && !(big < INFINITY) && lim < p.block);
    while (todo) {
      const int r = __builtin_ctzll(todo);
      todo &= todo - 1;
      const int rrow = __builtin_amdgcn_readlane(prow, r), rlim = __builtin_amdgcn_readlane(lim, r);
      const int ri = __builtin_amdgcn_readlane(qi, r), rh = __builtin_amdgcn_readlane(hg, r);
      const uint64_t at = (uint64_t)(uintptr_t)ml;
      const uint64_t rml = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), r) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)at, r);
      careful_row<T, D>(Qo + ri * p.qs + rh * D, Kg + j0 * p.ks, p.ks, Vg + j0 * p.vs, p.vs, rlim, p.qscale,
                        (T*)part.Opart + (int64_t)rrow * D, (float*)rml);
      store = store && l31 != r;
    }
    big = 0.f;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = __builtin_fabsf(acc[dt][r]);
        big = x < INFINITY ? fmaxf(big, x) : big;
      }
    big = max_with_partner(big);
  }
  float f = inv;
  if constexpr (BF) {
    const int ex = row_exp(big * inv);
    f = __builtin_amdgcn_ldexpf(inv, -ex);
    if (store && g == 0) encode_ml(m, l, ex, ml);
  } else {
    if (store && g == 0) *(float2*)ml = make_float2(l == 0.f ? -INFINITY : m, l);
  }
  uint8_t* ow = lds + wave * 32 * L::SEG * 16;
  const uint32_t rows_ok = (uint32_t)__ballot(store);
  // a segment of the rows at a time through the wave's own LDS, then whole segments in 16-byte stores
  constexpr int RPS = 64 / L::SEG, RN = 32 / RPS;   // rows of a store
  const int rr0 = lane / L::SEG, xo = lane % L::SEG;
  uint8_t* ob = (uint8_t*)part.Opart + 16 * xo;
  uint64_t oo[RN];
#pragma unroll
  for (int k = 0; k < RN; ++k) oo[k] = (uint64_t)(uint32_t)__shfl(prow, rr0 + k * RPS, 64) * (CPR * 16);
#pragma unroll
  for (int sg = 0; sg < CPR / L::SEG; ++sg) {
    if constexpr (BF) {
      constexpr int DTS = L::SEG / 4;   // 32-channel blocks of a segment
#pragma unroll
      for (int d = 0; d < DTS; ++d)
#pragma unroll
        for (int x = 0; x < 4; x += 2) {
          const f32x16& a = acc[sg * DTS + d];
          auto pk2 = [&](int i) {
            typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
            const f16x2 v = {(_Float16)(a[i] * f), (_Float16)(a[i + 1] * f)};
            return __builtin_bit_cast(uint32_t, v);
          };
          // channels 8x .. 8x+3 (+4 g) and 8x+8 .. +11 (+4 g): the lane pair swaps halves,
          // so that each lane holds eight neighbours
          const auto s0 = __builtin_amdgcn_permlane32_swap(pk2(4 * x), pk2(4 * x + 4), false, false);
          const auto s1 = __builtin_amdgcn_permlane32_swap(pk2(4 * x + 2), pk2(4 * x + 6), false, false);
          *(u32x4*)(ow + (l31 * L::SEG + ((4 * d + x + g) ^ L::f(l31))) * 16) = u32x4{s0[0], s1[0], s0[1], s1[1]};
        }
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const f32x16& a = acc[sg];
        *(f32x4*)(ow + (l31 * L::SEG + ((2 * x + g) ^ L::f(l31))) * 16) =
            f32x4{a[4 * x], a[4 * x + 1], a[4 * x + 2], a[4 * x + 3]} * f;
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    u32x4 val[RN];
#pragma unroll
    for (int k = 0; k < RN; ++k) {
      const int rr = rr0 + k * RPS;
      val[k] = *(const u32x4*)(ow + (rr * L::SEG + (xo ^ L::f(rr))) * 16);
    }
#pragma unroll
    for (int k = 0; k < RN; ++k)
      if ((rows_ok >> (rr0 + k * RPS)) & 1u) gstore((u32x4*)(ob + oo[k] + sg * L::SEG * 16), val[k]);
    __builtin_amdgcn_wave_barrier();
  }
}

template <class T, int D, int NT, bool ONE>
hipError_t launch_stages(const BlockAttendArgs& a, const BlockTileArgs& t, const BlockPartArgs& w, hipStream_t st) {
  constexpr int NW = BLOCK_TILE_WAVES;
  const int64_t per = ((int64_t)t.groups * t.tcap + 8 * XCD_RUN - 1) / (8 * XCD_RUN) * XCD_RUN;
  RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, (k_block_tile<T, D, NT, NW, ONE>), dim3((unsigned)(8 * per)), dim3(64 * NW),
             (TileLayout<T, D, NT, NW>::BYTES), st, a, t, w);
  return hipGetLastError();
}

template <class T, int D, int NT>
hipError_t launch_tile(const BlockAttendArgs& a, const BlockTileArgs& t, const BlockPartArgs& w, hipStream_t st) {
  return a.block == 32 * NT ? launch_stages<T, D, NT, true>(a, t, w, st) : launch_stages<T, D, NT, false>(a, t, w, st);
}

template <class T>
hipError_t launch_width(const BlockAttendArgs& a, const BlockTileArgs& t, const BlockPartArgs& w, hipStream_t st) {
  const bool one = a.block == 32;
  switch (a.d_h) {
    case 32: return one ? launch_tile<T, 32, 1>(a, t, w, st) : launch_tile<T, 32, 2>(a, t, w, st);
    case 64: return one ? launch_tile<T, 64, 1>(a, t, w, st) : launch_tile<T, 64, 2>(a, t, w, st);
    case 128: return one ? launch_tile<T, 128, 1>(a, t, w, st) : launch_tile<T, 128, 2>(a, t, w, st);
    default:
      if (one || sizeof(T) == 4) return launch_tile<T, 256, 1>(a, t, w, st);
      if constexpr (sizeof(T) == 2) return launch_tile<T, 256, 2>(a, t, w, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace rs3

using namespace rs3;

hipError_t rs3_launch_block_lists(const BlockAttendArgs& a, const BlockTileArgs& t, const BlockPartArgs& w,
                                  hipStream_t st) {
  const dim3 grid(t.groups, t.runs * t.chunks);
  const int64_t n = (int64_t)t.chunks * t.groups * a.n_blk;
  RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, k_block_zero, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, t.total, n);
  RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, k_block_count, grid, dim3(512), a.n_blk * 4, st, a, t, w);
  RS3_LAUNCH(RS3_K_BLOCK_ATTEND, st, k_block_scatter, grid, dim3(512), a.n_blk * 12, st, a, t);
  return hipGetLastError();
}

hipError_t rs3_launch_block_tile(const BlockAttendArgs& a, const BlockTileArgs& t, const BlockPartArgs& w, int dtype,
                                 hipStream_t st) {
  return dtype == RS3_BF16 ? launch_width<bf16_t>(a, t, w, st) : launch_width<float>(a, t, w, st);
}

template <class T, int D, int NT>
static hipError_t allow() {
  constexpr int NW = BLOCK_TILE_WAVES, bytes = TileLayout<T, D, NT, NW>::BYTES;
  const hipFuncAttribute at = hipFuncAttributeMaxDynamicSharedMemorySize;
  const hipError_t e = hipFuncSetAttribute((const void*)k_block_tile<T, D, NT, NW, true>, at, bytes);
  return e != hipSuccess ? e : hipFuncSetAttribute((const void*)k_block_tile<T, D, NT, NW, false>, at, bytes);
}

hipError_t rs3_block_tile_setup() {
  const hipError_t es[] = {
      hipFuncSetAttribute((const void*)k_block_scatter, hipFuncAttributeMaxDynamicSharedMemorySize, BLOCK_TILE_MAX * 12),
      allow<bf16_t, 128, 1>(), allow<bf16_t, 128, 2>(), allow<bf16_t, 256, 1>(), allow<bf16_t, 256, 2>(),
      allow<float, 64, 2>(), allow<float, 128, 1>(), allow<float, 128, 2>(), allow<float, 256, 1>()};
  for (hipError_t e : es)
    if (e != hipSuccess) return e;
  return hipSuccess;
}

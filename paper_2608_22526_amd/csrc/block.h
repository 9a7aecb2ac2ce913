// Shared by the kernels and the host side of the block-sparse attention and
// of the norm and rotation of queries and keys.
#pragma once

#include "attn_util.h"

namespace rs3 {

struct QkNormArgs {
  const void* X[2];      // queries, keys
  void* Y[2];
  int64_t xs[2], ys[2];  // elements between rows
  const float* gain[2];  // [d_h] or null
  int heads[2], chunks[2];   // chunks: of heads that a group of lanes takes together
  int n, d_h, d_rot, halves, n_pos;
  float eps, inv_d;
  const float* table;    // [n_pos][d_rot/2][2] or null
  const int32_t* pos;    // [n] or null
};

struct BlockMeansArgs {
  const void* K;
  int64_t ks, ko;          // elements between rows, objects
  const int32_t* kv_len;   // [n_obj] or null
  void* Kmean;             // [n_obj][H_kv][n_blk][d_h]
  int n_kv, H_kv, d_h, block, n_blk, n_new;
};

struct BlockSelectArgs {
  const void* Q;
  int64_t qs, qo;
  const void* Kmean;
  const int32_t* n_vis;    // [n_obj][n_q] or null
  int32_t* idx;            // [n_obj][n_q][H_kv][top_k]
  int32_t* count;          // [n_obj][n_q][H_kv]
  double* score;           // [end - row0][n_blk] workspace, or null
  int64_t row0, end;       // rows of this launch, of the n_obj * n_q * H_kv (row forms)
  int n_obj, n_q, n_kv, H, H_kv, d_h, block, n_blk, top_k, n_first, n_last;
};

// How a call of rs3_block_select runs.
constexpr int SELECT_LDS = 131072;   // at most
// The two terms of a tile's 32 queries.
constexpr int select_query_lds(int d_h) { return 2 * 32 * d_h * 2; }
struct BlockSelectPlan {
  bool tile;         // several queries of a key head per work-group, else one
  int TR, pitch;     // tile: queries, floats of a row of scores
  int split;         // else: work-groups that share a row's blocks, whose scores go to the workspace (1: LDS)
  int64_t at_once;   //   and the rows that are there at a time
  int lds;
};

struct BlockAttendArgs {
  const void* Q;
  const void* K;
  const void* V;
  void* O;
  int64_t qs, qo, ks, ko, vs, vo, os, oo;
  const int32_t* idx;
  const int32_t* count;
  const int32_t* n_vis;
  float qscale;            // log2(e) / sqrt(d_h)
  int n_obj, n_q, n_kv, H, H_kv, G, d_h, block, n_blk, top_k;
  int slots;               // entries of a list that can take part: min(top_k, n_blk)
};

// Blocks of keys that the counters of the tiled attention hold.
constexpr int BLOCK_TILE_MAX = 8192;
// Waves of a work-group of the tiled attention, 32 (query, head) rows each (eight
// read a block half as often and took the same time).
constexpr int BLOCK_TILE_WAVES = 4;

// Workspace of the tiled attention.  A group is an (object, key head) pair; the
// queries of every object are taken `chunk` at a time, so that the partial rows
// of a chunk are still in the memory-side cache when they are merged.
struct BlockTile {
  int b, n;                // block (-1: no tile), and how many queries
};
struct BlockTileArgs {
  uint32_t* ord;           // [groups][n_q][slots] place of an entry among its run's queries of its block,
                           //   times BLOCK_TILE_MAX, + the block; ~0: none
  uint32_t* total;         // [chunks][groups][n_blk] queries that list the block
  uint32_t* base;          // [chunks * runs][groups][n_blk] where each run's begin among them
  uint32_t* list;          // [chunks][groups][tcap][tq] query of the chunk * slots + slot
  BlockTile* tiles;        // [chunks][groups][tcap]
  int chunk, chunks, ch, nq;   // queries per chunk, chunks; this launch's chunk and its queries
  int run, runs;           // queries of one counting work-group, runs per chunk
  int tq, tcap, groups;    // queries of a tile at most, tiles of a group and chunk at most
};

// Partial rows, merged by k_block_merge: O row (((o * nq + i) * H_kv + g) * S + s)
// * G + head of a chunk's nq queries, (m, l) pair of the same row among all n_q;
// s is a slot of the list (tiled form) or a split of the keys.
struct BlockPartArgs {
  void* Opart;
  float* ML;
  int S, i0, nq;
};

// Grids of many work-groups fold into two dimensions: one holds fewer than 2^32
// threads.
inline dim3 folded(int64_t n, unsigned z = 1) {
  const int64_t x = std::min<int64_t>(n, 1 << 20);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x), z);
}
__device__ __forceinline__ int64_t folded_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// How many keys query `i` (of all objects' queries) sees.
__device__ __forceinline__ int visible_keys(const int32_t* n_vis, int64_t i, int n_kv) {
  return n_vis ? min(max(gload(n_vis + i), 0), n_kv) : n_kv;
}

// LDS layout of a stage of key (value) rows: 16-byte chunk c of row r lies at
// chunk c ^ f(r) of the row, so that the rows that one LDS cycle reads fall on
// different banks.  CPR chunks a row; 16 / CPR rows share the 256 bytes of one
// cycle.  k: 16 (or more) keys at one chunk.  v: WD neighbouring chunks of the
// rows whose number differs in the bits from SH up.
template <int CPR>
struct Swz {
  static constexpr int RPB = CPR >= 16 ? 1 : 16 / CPR, W = CPR >= 16 ? 16 : CPR;
  static __device__ __forceinline__ int k(int r) { return (r / RPB) & (W - 1); }
  template <int WD, int SH>
  static __device__ __forceinline__ int v(int r) {
    return (((r >> SH) / (SH ? 1 : RPB)) & (W / WD - 1)) * WD;
  }
};

// Value operand of a bf16 product from rows of keys: lane i of 16 gets the four
// values of channel i of four keys; lane s supplies the address of channels
// 4 (s % 4) .. +3 of key s / 4.
__device__ __forceinline__ u32x2 lds_tr4(const uint8_t* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

template <class T>
__device__ __forceinline__ float to_f32(T v) {
  if constexpr (sizeof(T) == 2) return bf2f(v);
  else return v;
}

// Rounded once: to bf16 by way of the fp32 number whose last bit says whether
// anything is behind it (toward zero, set if so), which has bits to spare for that.
template <class T>
__device__ __forceinline__ T from_f64(double v) {
  const float f = (float)v;
  if constexpr (sizeof(T) == 4) return f;
  else {
    uint32_t u = __float_as_uint(f);
    if ((double)f != v) u = (u - (__builtin_fabs((double)f) > __builtin_fabs(v))) | 1u;
    return f2bf(__uint_as_float(u));
  }
}

}  // namespace rs3

hipError_t rs3_launch_qk_norm(const rs3::QkNormArgs& a, int dtype, hipStream_t st);
hipError_t rs3_launch_block_means(const rs3::BlockMeansArgs& a, int n_obj, int dtype, hipStream_t st);
hipError_t rs3_launch_block_select(const rs3::BlockSelectArgs& a, const rs3::BlockSelectPlan& pl, int dtype,
                                   hipStream_t st);
hipError_t rs3_block_select_setup();
hipError_t rs3_launch_block_row(const rs3::BlockAttendArgs& a, const rs3::BlockPartArgs& w, int dtype, hipStream_t st);
hipError_t rs3_launch_block_lists(const rs3::BlockAttendArgs& a, const rs3::BlockTileArgs& t,
                                  const rs3::BlockPartArgs& w, hipStream_t st);
hipError_t rs3_launch_block_tile(const rs3::BlockAttendArgs& a, const rs3::BlockTileArgs& t,
                                 const rs3::BlockPartArgs& w, int dtype, hipStream_t st);
hipError_t rs3_launch_block_merge(const rs3::BlockAttendArgs& a, const rs3::BlockPartArgs& w, int dtype, bool f16,
                                  hipStream_t st);
hipError_t rs3_block_setup();
hipError_t rs3_block_tile_setup();

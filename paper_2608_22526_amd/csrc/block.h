// Shared by the kernels and the host side of the block-sparse attention and
// of the norm and rotation of queries and keys.
#pragma once

#include "device_util.h"

namespace rs3 {

struct QkNormArgs {
  const void* X[2];      // queries, keys
  void* Y[2];
  int64_t xs[2], ys[2];  // elements between rows
  const float* gain[2];  // [d_h] or null
  int heads[2];
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
  double* score;           // [rows][n_blk] workspace
  int64_t rows;            // n_obj * n_q * H_kv
  int n_obj, n_q, n_kv, H, H_kv, d_h, block, n_blk, top_k, n_first, n_last;
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
};

// How many keys query `i` (of all objects' queries) sees.
__device__ __forceinline__ int visible_keys(const int32_t* n_vis, int64_t i, int n_kv) {
  return n_vis ? min(max(gload(n_vis + i), 0), n_kv) : n_kv;
}

template <class T>
__device__ __forceinline__ float to_f32(T v) {
  if constexpr (sizeof(T) == 2) return bf2f(v);
  else return v;
}
template <class T>
__device__ __forceinline__ T from_f32(float v) {
  if constexpr (sizeof(T) == 2) return f2bf(v);
  else return v;
}

}  // namespace rs3

hipError_t rs3_launch_qk_norm(const rs3::QkNormArgs& a, int dtype, hipStream_t st);
hipError_t rs3_launch_block_means(const rs3::BlockMeansArgs& a, int n_obj, int dtype, hipStream_t st);
hipError_t rs3_launch_block_select(const rs3::BlockSelectArgs& a, int dtype, hipStream_t st);
hipError_t rs3_launch_block_attend(const rs3::BlockAttendArgs& a, int dtype, hipStream_t st);

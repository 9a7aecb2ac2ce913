// Host side of the norm and rotation of queries and keys and of the
// block-sparse attention: validation and launch arguments.
#include <math.h>
#include <string.h>

#include <atomic>

#include "block.h"

using namespace rs3;

namespace {

rs3_status map_err(hipError_t e) {
  if (e == hipSuccess) return RS3_OK;
  return e == hipErrorOutOfMemory ? RS3_E_OOM : RS3_E_DEVICE;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
size_t elem(int dt) { return dt == RS3_BF16 ? 2 : 4; }

// A stride of whole 16-byte units, small enough that no row's offset leaves
// 62 bits.
bool stride_ok(int64_t s, size_t es) { return s >= 0 && s < (1ll << 36) && s * es % 16 == 0; }

bool shape_ok(const rs3_block_shape* s) {
  if (!s || (s->dt != RS3_BF16 && s->dt != RS3_F32) || s->reserved != 0) return false;
  if (s->n_obj < 1 || s->n_obj > 4096 || s->n_q < 0 || (int64_t)s->n_obj * s->n_q > (1 << 22)) return false;
  if (s->n_kv < 0 || s->n_kv > (1 << 26)) return false;
  if (s->H < 1 || s->H > 256 || s->H_kv < 1 || s->H % s->H_kv != 0) return false;
  if (s->d_h != 32 && s->d_h != 64 && s->d_h != 128 && s->d_h != 256) return false;
  if (s->block != 32 && s->block != 64 && s->block != 128 && s->block != 256) return false;
  if (s->top_k < 1 || s->top_k > 256 || s->n_first < 0 || s->n_last < 0) return false;
  return (int64_t)s->n_first + s->n_last <= s->top_k;
}

// Row layout of a tensor with `heads` heads a row.
bool rows_ok(const rs3_block_shape* s, int64_t row, int64_t obj, int heads) {
  const size_t es = elem(s->dt);
  return stride_ok(row, es) && stride_ok(obj, es) && row >= (int64_t)heads * s->d_h;
}

// The attention's lanes add up the row offsets of a block in 32 bits.
bool kv_rows_ok(const rs3_block_shape* s, int64_t row, int64_t obj) {
  return rows_ok(s, row, obj, s->H_kv) && row < (1 << 22);
}

bool out_rows_ok(const rs3_block_shape* s) {
  const int64_t w = (int64_t)s->H * s->d_h;
  if (!rows_ok(s, s->o_stride, s->o_obj_stride, s->H)) return false;
  if (s->n_obj == 1 || s->n_q == 0) return true;
  return s->o_obj_stride >= w && (s->o_obj_stride >= (int64_t)(s->n_q - 1) * s->o_stride + w ||
                                  s->o_stride >= (int64_t)(s->n_obj - 1) * s->o_obj_stride + w);
}

int n_blocks(const rs3_block_shape* s) { return (s->n_kv + s->block - 1) / s->block; }

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// How a call of rs3_block_attend runs.
struct AttendPlan {
  bool tile;         // tiled form
  int S;             // splits of a row's keys (other form)
  int objs;          // objects at a time
  int groups, chunk, chunks, run, runs, tq, tcap;   // chunks: of a section
  int64_t section;   // queries of an object whose lists are there at a time, whole chunks
  size_t ord, cnt, base, list, tiles, opart, ml, total;
};

// Partial rows of a chunk of queries, or of several objects': as much as the
// memory-side cache holds until they are merged, but every chunk reads the keys and
// values anew, so for a long cache up to twice its bytes.  537 MB of partials in chunks
// of at most 160, 256 and 540 MB (us): 8192 queries of 512 blocks, 67 MB of keys
// and values 341/318/325; of 2048 blocks, 268 MB 475/367/331; 4096 queries of 8192
// blocks, 2.1 GB 1840/1188/747.
constexpr size_t PART_LEAST = (size_t)256 << 20, PART_MOST = (size_t)1 << 30;
// Lists and (m, l) pairs of a section of the queries (chunks, one at least): their
// three launches take about 15 us, a chunk's own several times that.
constexpr size_t LISTS_MOST = (size_t)256 << 20;

void attend_plan(const rs3_block_shape* s, AttendPlan* a) {
  memset(a, 0, sizeof(*a));
  const int n_blk = (s->n_kv + s->block - 1) / s->block, G = s->H / s->H_kv;
  const int slots = std::min(s->top_k, n_blk);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += align256(bytes);
    return at;
  };
  const size_t per_q = (size_t)s->H * slots * s->d_h * elem(s->dt);   // partial rows of one query of an object
  // What the row form reads: the keys and values of each row's blocks, and as much
  // time as 128 KiB more for the row itself. The tile form reads each once, but has
  // five launches and the partial rows. Against 320 MiB and twice the cache (row and
  // tile form in us, 64-key blocks, bf16):
  //   1 x n_q, 32/8 heads of 128, 16 of 256 blocks: n_q 32 16/31, 64 28/33, 128 52/37, 256 100/43
  //   8 x n_q, the same of 128 blocks: n_q 8 34/50, 16 53/62, 32 96/75, 64 182/90
  //   1 x n_q, 8/2 heads, 16 of 4096 blocks: n_q 256 42/63, 512 77/76, 1024 144/89
  //   64 x n_q, 8/8 heads of 128, all 4 blocks: n_q 8 84/31, 64 626/43
  //   1 x n_q, 8/8 heads of 64, fp32, 16 of 128 blocks of 32: n_q 32 12/25, 64 22/26, 128 42/28
  const int64_t rows = (int64_t)s->n_obj * s->n_q * s->H_kv * ((G + 15) / 16);
  const int64_t key_bytes = (int64_t)2 * s->d_h * elem(s->dt);
  const int64_t keys = std::min<int64_t>((int64_t)slots * s->block, s->n_kv);
  const double row_reads = (double)rows * (keys * key_bytes + (128 << 10));
  const double tile_reads = (320 << 20) + 2.0 * s->n_obj * s->H_kv * s->n_kv * key_bytes;
  a->tile = s->n_q >= 8 && row_reads > tile_reads && n_blk <= BLOCK_TILE_MAX && n_blk > 0 && per_q <= (16u << 20) &&
            G <= 32 * BLOCK_TILE_WAVES;
  if (a->tile) {
    // as many whole objects as `part` holds, or one and a chunk of its queries
    const size_t part = std::min(PART_MOST, std::max(PART_LEAST, (size_t)(2 * s->H_kv * s->n_kv * key_bytes)));
    const int64_t most_o = std::max<int64_t>(1, (int64_t)(part / (per_q * s->n_q)));
    const int parts = (int)((s->n_obj + most_o - 1) / most_o);
    a->objs = (s->n_obj + parts - 1) / parts;
    const int64_t most_q = std::max<int64_t>(64, (int64_t)(part / (per_q * a->objs)));
    a->chunks = (int)((s->n_q + most_q - 1) / most_q);
    a->chunk = (s->n_q + a->chunks - 1) / a->chunks;
    a->groups = a->objs * s->H_kv;
    // queries of a counting work-group: four entries a thread, fewer while that leaves CUs
    // idle and the entries are at least four times the blocks' counters (2000 queries of
    // 16/1 heads, 4 of 7 blocks: 42 us with four work-groups, 38 with 63; 300 queries of
    // 32/8, 256 blocks each: 279 with 64 queries per work-group, 257 with 16)
    const int64_t spread = std::max<int64_t>((int64_t)a->chunk * a->chunks * a->groups / 256, 4 * n_blk / slots);
    const int least = std::max(std::max(128 / slots, 16), s->n_q >> 15);
    a->run = (int)std::max<int64_t>(least, std::min<int64_t>(2048 / slots, spread));
    a->runs = (a->chunk + a->run - 1) / a->run;
    a->tq = 32 * BLOCK_TILE_WAVES / G;
    const int64_t entries = (int64_t)a->chunk * slots;
    a->tcap = (int)(entries / a->tq + (n_blk < entries ? n_blk : entries));
    // what the launches' grids hold
    a->tile = (int64_t)a->runs * a->chunks <= 65535 && (int64_t)a->chunks * a->groups * n_blk < (1ll << 31) &&
              (int64_t)a->groups * a->tcap < (1 << 23);
  }
  if (a->tile) {
    const int64_t entries = (int64_t)a->chunk * slots;
    const size_t ord = (size_t)entries * a->groups * 4, cnt = (size_t)a->groups * n_blk * 4;   // of a chunk
    const size_t list = (size_t)a->tcap * a->groups * a->tq * 4, tiles = (size_t)a->tcap * a->groups * sizeof(BlockTile);
    const size_t ml = (size_t)entries * s->H * a->objs * 8;
    const int64_t most = std::max<int64_t>(1, (int64_t)(LISTS_MOST / (ord + cnt * (1 + a->runs) + list + tiles + ml)));
    const int64_t sections = (a->chunks + most - 1) / most;   // (several chunks are those of one object)
    a->chunks = (int)((a->chunks + sections - 1) / sections);
    a->section = (int64_t)a->chunk * a->chunks;
    a->ord = take(ord * a->chunks);
    a->cnt = take(cnt * a->chunks);
    a->base = take(cnt * a->chunks * a->runs);
    a->list = take(list * a->chunks);
    a->tiles = take(tiles * a->chunks);
    a->opart = take(entries * s->H * a->objs * s->d_h * elem(s->dt));
    a->ml = take(ml * a->chunks);
  } else {
    // a work-group per CU, each with a few pieces of 32 keys per wave (whole rows and
    // splits in us, 8 key heads of 128: one row of 64 of 2048 blocks 31/14, four rows
    // of 32 blocks 22/14, twelve 25/24; two or four splits of 256 rows 50/58/65)
    int64_t S = rows > 0 ? 256 / rows : 1;
    const int64_t most = (int64_t)slots * s->block / 32 / 8;
    S = S < most ? S : most;
    a->S = (int)(S < 1 ? 1 : S);
    if (a->S > 1) {
      a->opart = take((size_t)s->n_obj * s->n_q * s->H * a->S * s->d_h * 4);
      a->ml = take((size_t)s->n_obj * s->n_q * s->H * a->S * 8);
    }
  }
  a->total = off;
}

std::atomic<uint64_t> setup_done{0};   // one bit per device

rs3_status ensure_setup() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return RS3_E_DEVICE;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (setup_done.load(std::memory_order_acquire) & bit) return RS3_OK;
  if (rs3_block_setup() != hipSuccess) return RS3_E_DEVICE;
  setup_done.fetch_or(bit, std::memory_order_release);
  return RS3_OK;
}

// Scores in the workspace of the block choice: the rows beyond take it again (16
// rows of 2^21 blocks, the most that there can be, and what the memory-side cache holds).
constexpr size_t SCORES_MOST = (size_t)256 << 20;

void select_plan(const rs3_block_shape* s, BlockSelectPlan* a, size_t* ws) {
  memset(a, 0, sizeof(*a));
  *ws = 0;
  const int64_t n_blk = n_blocks(s), rows = (int64_t)s->n_obj * s->n_q * s->H_kv;
  a->split = 1;
  // Several queries (us, row form and tile form at 16 of 256 blocks, 8 key heads of
  // 128: 256 rows 10.5/10.1, 512 19/10, 1024 35/11, 4096 133/13). The row form has a
  // work-group per row, so up to one per CU it is no slower, and at many blocks faster
  // (256 rows of 4096 blocks 46/86). The tile: the largest whose scores leave room for
  // two work-groups per CU, smaller while that gives fewer work-groups than CUs (64
  // queries: tiles of 32 18, of 4 10.3), at least four queries.
  const int q_lds = select_query_lds(s->d_h), before = s->d_h > 128 ? q_lds : 0;   // before the scores
  a->pitch = (int)((n_blk + 31) / 32 * 32 + 4);
  if (s->n_q >= 4 && (rows > 256 || (s->n_q >= 8 && n_blk <= 256))) {
    int TR = 32;
    const int64_t heads = (int64_t)s->n_obj * s->H_kv;
    while (TR > 4 && (before + TR * a->pitch * 4 > 81920 - 10752 || TR / 2 >= s->n_q ||
                      heads * ((s->n_q + TR - 1) / TR) < 256))
      TR /= 2;
    int64_t lds = before + (int64_t)TR * a->pitch * 4;
    lds = std::max<int64_t>(lds, std::max<int64_t>(n_blk * 8, q_lds));
    if (lds <= SELECT_LDS) {
      a->tile = true;
      a->TR = TR;
      a->lds = (int)lds;
      return;
    }
  }
  // One query per work-group: its blocks over several where there are few rows
  // (whole rows and splits in us, 8 key heads of 128: one query of 2048 blocks 21/13,
  // four of 1024 14.7/13.4, twelve 14.9/14.6) or the scores do not fit the LDS.
  int64_t split = rows > 0 && rows < 128 ? std::min<int64_t>(256 / rows, n_blk / 128) : 1;
  if (n_blk * 8 > SELECT_LDS) split = std::max<int64_t>(split, (n_blk + 4095) / 4096);
  a->split = (int)(split < 1 ? 1 : split);
  if (a->split > 1) {   // rows in parts of about one size
    const int64_t most = (int64_t)(SCORES_MOST / (n_blk * sizeof(double)));
    const int64_t parts = std::max<int64_t>(1, (rows + most - 1) / most);
    a->at_once = (rows + parts - 1) / parts;
    *ws = (size_t)a->at_once * n_blk * sizeof(double);
  } else {
    a->lds = (int)std::max<int64_t>(n_blk * 8, 16);
  }
}

}  // namespace

extern "C" {

rs3_status rs3_qk_norm_rope(int32_t n, const void* Q, int64_t q_stride, int32_t H, const void* K, int64_t k_stride,
                            int32_t H_kv, int32_t d_h, rs3_dtype dt, const float* gain_q, const float* gain_k,
                            float eps, const float* table, int32_t n_pos, int32_t d_rot, int32_t pairing,
                            const int32_t* pos, void* Qo, int64_t qo_stride, void* Ko, int64_t ko_stride,
                            void* stream) {
  if (n < 0 || n > (1 << 24) || (dt != RS3_BF16 && dt != RS3_F32)) return RS3_E_INVALID;
  if (H < 0 || H_kv < 0 || H > 1024 || H_kv > 1024 - H || d_h < 16 || d_h > 256 || d_h % 16 != 0) return RS3_E_INVALID;
  if ((int64_t)n * (H + H_kv) > (1 << 27)) return RS3_E_INVALID;   // fewer than 2^32 threads
  if (!(eps > 0.f) || !isfinite(eps)) return RS3_E_INVALID;
  if (d_rot < 0 || d_rot > d_h || d_rot % 16 != 0 || (d_rot > 0) != (table != nullptr)) return RS3_E_INVALID;
  if (pairing != RS3_PAIRS_ADJACENT && pairing != RS3_PAIRS_HALVES) return RS3_E_INVALID;
  if (d_rot > 0 && (n_pos < 1 || (!pos && n > n_pos))) return RS3_E_INVALID;
  if (!aligned16(table) || !aligned16(gain_q) || !aligned16(gain_k)) return RS3_E_INVALID;
  QkNormArgs a;
  memset(&a, 0, sizeof(a));
  const struct {
    const void* x;
    void* y;
    int64_t xs, ys;
    int heads;
    const float* gain;
  } sides[2] = {{Q, Qo, q_stride, qo_stride, H, gain_q}, {K, Ko, k_stride, ko_stride, H_kv, gain_k}};
  for (int i = 0; i < 2; ++i) {
    const auto& s = sides[i];
    if (s.heads == 0) continue;
    const size_t es = elem(dt);
    if (n > 0 && (!s.x || !s.y)) return RS3_E_INVALID;
    if (!aligned16(s.x) || !aligned16(s.y) || !stride_ok(s.xs, es) || !stride_ok(s.ys, es)) return RS3_E_INVALID;
    if (s.xs < (int64_t)s.heads * d_h || s.ys < (int64_t)s.heads * d_h) return RS3_E_INVALID;
    if (s.x == s.y && s.xs != s.ys) return RS3_E_INVALID;
    a.X[i] = s.x;
    a.Y[i] = s.y;
    a.xs[i] = s.xs;
    a.ys[i] = s.ys;
    a.heads[i] = s.heads;
    a.gain[i] = s.gain;
  }
  if (n == 0 || H + H_kv == 0) return RS3_OK;
  a.n = n;
  a.d_h = d_h;
  a.d_rot = d_rot;
  a.halves = pairing == RS3_PAIRS_HALVES;
  a.n_pos = n_pos;
  a.eps = eps;
  a.inv_d = 1.f / (float)d_h;
  a.table = table;
  a.pos = pos;
  return map_err(rs3_launch_qk_norm(a, dt, (hipStream_t)stream));
}

rs3_status rs3_block_means(const rs3_block_shape* s, const void* K, const int32_t* kv_len, int32_t n_new, void* Kmean,
                           void* stream) {
  if (!shape_ok(s) || n_new < 0 || !kv_rows_ok(s, s->k_stride, s->k_obj_stride)) return RS3_E_INVALID;
  if (!aligned16(K) || !aligned16(Kmean) || (s->n_kv > 0 && (!K || !Kmean))) return RS3_E_INVALID;
  if (s->n_kv == 0) return RS3_OK;
  BlockMeansArgs a;
  memset(&a, 0, sizeof(a));
  a.K = K;
  a.ks = s->k_stride;
  a.ko = s->k_obj_stride;
  a.kv_len = kv_len;
  a.Kmean = Kmean;
  a.n_kv = s->n_kv;
  a.H_kv = s->H_kv;
  a.d_h = s->d_h;
  a.block = s->block;
  a.n_blk = n_blocks(s);
  a.n_new = n_new;
  return map_err(rs3_launch_block_means(a, s->n_obj, s->dt, (hipStream_t)stream));
}

rs3_status rs3_block_select_workspace_size(const rs3_block_shape* s, size_t* bytes) {
  if (!bytes || !shape_ok(s)) return RS3_E_INVALID;
  BlockSelectPlan pl;
  select_plan(s, &pl, bytes);
  return RS3_OK;
}

rs3_status rs3_block_select(const rs3_block_shape* s, const void* Q, const void* Kmean, const int32_t* n_vis,
                            int32_t* idx, int32_t* count, void* ws, size_t ws_bytes, void* stream) {
  if (!shape_ok(s) || !rows_ok(s, s->q_stride, s->q_obj_stride, s->H)) return RS3_E_INVALID;
  if (!aligned16(Q) || !aligned16(Kmean) || !aligned16(ws)) return RS3_E_INVALID;
  if (s->n_q == 0) return RS3_OK;
  if (!Q || !idx || !count || (s->n_kv > 0 && !Kmean)) return RS3_E_INVALID;
  BlockSelectPlan pl;
  size_t need;
  select_plan(s, &pl, &need);
  if (need > 0 && (!ws || ws_bytes < need)) return RS3_E_INVALID;
  const rs3_status st0 = ensure_setup();
  if (st0 != RS3_OK) return st0;
  BlockSelectArgs a;
  memset(&a, 0, sizeof(a));
  a.Q = Q;
  a.qs = s->q_stride;
  a.qo = s->q_obj_stride;
  a.Kmean = Kmean;
  a.n_vis = n_vis;
  a.idx = idx;
  a.count = count;
  a.score = (double*)ws;
  a.n_obj = s->n_obj;
  a.n_q = s->n_q;
  a.n_kv = s->n_kv;
  a.H = s->H;
  a.H_kv = s->H_kv;
  a.d_h = s->d_h;
  a.block = s->block;
  a.n_blk = n_blocks(s);
  a.top_k = s->top_k;
  a.n_first = s->n_first;
  a.n_last = s->n_last;
  return map_err(rs3_launch_block_select(a, pl, s->dt, (hipStream_t)stream));
}

rs3_status rs3_block_attend_workspace_size(const rs3_block_shape* s, size_t* bytes) {
  if (!bytes || !shape_ok(s)) return RS3_E_INVALID;
  AttendPlan pl;
  attend_plan(s, &pl);
  *bytes = pl.total;
  return RS3_OK;
}

rs3_status rs3_block_attend(const rs3_block_shape* s, const void* Q, const void* K, const void* V, const int32_t* idx,
                            const int32_t* count, const int32_t* n_vis, void* O, void* ws, size_t ws_bytes,
                            void* stream) {
  if (!shape_ok(s) || !rows_ok(s, s->q_stride, s->q_obj_stride, s->H) ||
      !kv_rows_ok(s, s->k_stride, s->k_obj_stride) || !kv_rows_ok(s, s->v_stride, s->v_obj_stride) || !out_rows_ok(s))
    return RS3_E_INVALID;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(ws)) return RS3_E_INVALID;
  if (s->n_q == 0) return RS3_OK;
  if (!Q || !idx || !count || !O || (s->n_kv > 0 && (!K || !V))) return RS3_E_INVALID;
  if (O == Q || (s->n_kv > 0 && (O == K || O == V))) return RS3_E_INVALID;
  AttendPlan pl;
  attend_plan(s, &pl);
  if (pl.total > 0 && (!ws || ws_bytes < pl.total)) return RS3_E_INVALID;
  const rs3_status st0 = ensure_setup();
  if (st0 != RS3_OK) return st0;
  BlockAttendArgs a;
  memset(&a, 0, sizeof(a));
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.O = O;
  a.qs = s->q_stride;
  a.qo = s->q_obj_stride;
  a.ks = s->k_stride;
  a.ko = s->k_obj_stride;
  a.vs = s->v_stride;
  a.vo = s->v_obj_stride;
  a.os = s->o_stride;
  a.oo = s->o_obj_stride;
  a.idx = idx;
  a.count = count;
  a.n_vis = n_vis;
  a.qscale = (float)(1.4426950408889634 / sqrt((double)s->d_h));
  a.n_obj = s->n_obj;
  a.n_q = s->n_q;
  a.n_kv = s->n_kv;
  a.H = s->H;
  a.H_kv = s->H_kv;
  a.G = s->H / s->H_kv;
  a.d_h = s->d_h;
  a.block = s->block;
  a.n_blk = n_blocks(s);
  a.top_k = s->top_k;
  a.slots = std::min(a.top_k, a.n_blk);
  const hipStream_t st = (hipStream_t)stream;
  uint8_t* w = (uint8_t*)ws;
  BlockPartArgs part;
  memset(&part, 0, sizeof(part));
  part.Opart = w + pl.opart;
  part.ML = (float*)(w + pl.ml);
  if (!pl.tile) {
    part.S = pl.S;
    part.nq = s->n_q;
    hipError_t e = rs3_launch_block_row(a, part, s->dt, st);
    if (e == hipSuccess && pl.S > 1) e = rs3_launch_block_merge(a, part, s->dt, false, st);
    return map_err(e);
  }
  BlockTileArgs t;
  memset(&t, 0, sizeof(t));
  t.ord = (uint32_t*)(w + pl.ord);
  t.total = (uint32_t*)(w + pl.cnt);
  t.base = (uint32_t*)(w + pl.base);
  t.list = (uint32_t*)(w + pl.list);
  t.tiles = (BlockTile*)(w + pl.tiles);
  t.chunk = pl.chunk;
  t.run = pl.run;
  t.runs = pl.runs;
  t.tq = pl.tq;
  t.tcap = pl.tcap;
  part.S = a.slots;
  hipError_t e = hipSuccess;
  for (int64_t o = 0; o < s->n_obj; o += pl.objs)
    for (int64_t q = 0; q < s->n_q && e == hipSuccess; q += pl.section) {
      const int64_t es = (int64_t)elem(s->dt), rows = o * s->n_q + q, lists = rows * s->H_kv;
      a.n_obj = (int)std::min<int64_t>(pl.objs, s->n_obj - o);
      a.n_q = (int)std::min<int64_t>(pl.section, s->n_q - q);   // all of them where there are several objects
      t.groups = a.n_obj * s->H_kv;
      t.chunks = (a.n_q + pl.chunk - 1) / pl.chunk;
      a.Q = (const uint8_t*)Q + (o * s->q_obj_stride + q * s->q_stride) * es;
      a.K = (const uint8_t*)K + o * s->k_obj_stride * es;
      a.V = (const uint8_t*)V + o * s->v_obj_stride * es;
      a.O = (uint8_t*)O + (o * s->o_obj_stride + q * s->o_stride) * es;
      a.idx = idx + lists * s->top_k;
      a.count = count + lists;
      a.n_vis = n_vis ? n_vis + rows : nullptr;
      e = rs3_launch_block_lists(a, t, part, st);
      for (t.ch = 0; t.ch < t.chunks && e == hipSuccess; ++t.ch) {
        part.i0 = t.ch * pl.chunk;
        part.nq = t.nq = std::min(pl.chunk, a.n_q - part.i0);
        e = rs3_launch_block_tile(a, t, part, s->dt, st);
        if (e == hipSuccess) e = rs3_launch_block_merge(a, part, s->dt, true, st);
      }
    }
  return map_err(e);
}

}  // extern "C"

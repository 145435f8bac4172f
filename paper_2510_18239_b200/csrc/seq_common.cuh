// Attention of the sequence path (lime_attend_history, lime_attend_tree): what its kernels share - the arguments, the work items that
// k_seq_schedule.cu makes of a batch, and where the keys of an item are.
//
// A work item is a tile of consecutive rows (tokens) of one user against a range of key tiles, for one head of keys: the Hq / Hkv query
// heads that read it are stacked, row r of the item is token r / G and query head kvh * G + r % G, so keys and values are read once for
// all of them.  The key tiles of a row tile, in the order they are walked:
//   history: key tiles 0, 1, .. up to the last one its last token sees;
//   tree:    the tiles of the user's new rows from the tile's own last row back (to the first tile, or with roots only to the tile's
//            own first row: every token walks its chain of ancestors once, backwards), then the tiles of the cached rows.
// A row tile whose keys are many, in a batch that has few row tiles, is cut into several items; k_seq_merge joins their partial results
// (running maximum, sum and unnormalised values, fp32).
#pragma once
#include "lime_common.cuh"

namespace lime {

struct SeqItem {
  int32_t row0, rows;     // first packed row, tokens
  int32_t a;              // history: packed row of the user's key 0; tree: the user
  int32_t b;              // history: the user's keys; tree: its cached rows
  int32_t c;              // history: keys that the first token sees (<= 0: none); tree: index of row0 among the user's rows
  int32_t t0, t1;         // key tiles, in the order above
  int32_t part;           // where the partial result goes; -1: the item is the whole row tile
};
struct SeqSplit { int32_t row0, rows, part0, n; };       // a row tile cut into n items, parts part0 ..
struct SeqPlan { int32_t n_items, n_split; };

struct SeqParams {
  const void *q, *k, *v;                 // history: k, v the packed keys; tree: the new rows' (nullable)
  int64_t q_stride, k_stride, v_stride, out_stride;
  void* out;
  const int32_t *off, *kv_off;           // kv_off: history only
  const int32_t *parent, *table, *ctx_len;
  const void *ck, *cv;                   // pages
  int32_t* dev_flag;
  int64_t q_rows, kv_rows, n_pages;
  int32_t B, page_rows, page_shift, max_pages;
  int32_t Hq, Hkv, G, dh;
  float scale_log2;                      // attn_scale * log2(e): scores in the log2 domain
  int32_t tok, kt;                       // tokens per row tile, keys per key tile
  // workspace
  SeqPlan* plan; SeqItem* items; SeqSplit* splits; int32_t* tile_start;
  float *part_ml, *part_acc;             // [part][kvh][2][part_rows] and [part][kvh][part_rows][dh]
  int32_t row_tiles_upper, items_upper, split_upper;
  int32_t part_rows;                     // stacked rows a row tile of the call can have
  // how row tiles are cut: key tiles per item at least; items (over all key heads) that a batch may make about; CTAs that run at once; what
  // an item costs besides its key tiles, and what its being one of several adds, in key tiles
  int32_t chunk_min, chunk_target, ctas;
  float item_cost, split_cost;
  int32_t* err;
};

// limit of what the user's range has: keys there are, of the tile kinds below
struct SeqTile {
  int kind;         // 0: packed keys, 1: cached rows, 2: new rows
  int j0;           // first key of the tile among the user's
  int n;            // keys of that kind there are (the tile may end past it)
};
__device__ __forceinline__ int seq_tree_tiles(const SeqParams& p, const SeqItem& it) {
  if (p.k == nullptr) return 0;
  const int hi = (it.c + it.rows + p.kt - 1) / p.kt, lo = p.parent != nullptr ? 0 : it.c / p.kt;
  return hi - lo;
}
// tile `t` of the walk
template <bool TREE>
__device__ __forceinline__ SeqTile seq_tile(const SeqParams& p, const SeqItem& it, int n_tree, int t) {
  SeqTile s;
  if (!TREE) {
    s.kind = 0; s.j0 = t * p.kt; s.n = it.b;
  } else if (t < n_tree) {
    s.kind = 2; s.j0 = ((it.c + it.rows + p.kt - 1) / p.kt - 1 - t) * p.kt; s.n = it.c + it.rows;
  } else {
    s.kind = 1; s.j0 = (t - n_tree) * p.kt; s.n = it.b;
  }
  return s;
}
// parent of new row i of the user whose rows start at packed row `first`: an index below i, or -1
__device__ __forceinline__ int seq_parent(const SeqParams& p, int first, int i) {
  if (p.parent == nullptr) return -1;
  const int a = __ldg(p.parent + first + i);
  return a < i ? (a < 0 ? -1 : a) : -1;
}
// the page of the user's cached row j, n_pages (a page past the last: rows that read as zeros) where the table holds none
__device__ __forceinline__ int64_t seq_page(const SeqParams& p, int user, int j) {
  const int64_t at = (int64_t)user * p.max_pages + (j >> p.page_shift);
  const int pg = __ldg(p.table + at);
  if (pg >= 0 && pg < p.n_pages) return pg;
  if (p.dev_flag != nullptr) atomicMin(p.dev_flag, (int32_t)at);
  return p.n_pages;
}

// What a result is multiplied by: 0 where the row sees nothing.  A row that sees scores of -infinity alone has a sum of 0 and values of 0,
// which the reciprocal makes NaN, as the formula has it.
__device__ __forceinline__ float seq_inverse(float sum, bool sees) { return sees ? 1.f / sum : 0.f; }

// blocks of k_seq_attn_few an SM (as many as fit without spilling much; 8 rather than 6 at d_h <= 32: 24.5 against 30.7 us for 256 events over
// 512 rows, 3 rather than 2 at d_h > 64: 180 against 201 us for 64 events over 16..16384)
constexpr int seq_few_blocks(int dh) { return dh <= 32 ? 8 : dh <= 64 ? 4 : 3; }

// ----------------------------------------------------------------------------- launchers
struct NormRotateArgs {
  const void *q, *k, *v, *gamma_q, *gamma_k;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  const int32_t *positions, *slots;
  int64_t rows, cache_rows;
  void *q_out, *k_out, *cache_k, *cache_v;
  int32_t* dev_flag;
  int dtype;
  const lime_sequence* seq;
  const uint64_t* rot_freq;
};
lime_status launch_norm_rotate(const NormRotateArgs& a, cudaStream_t st);
lime_status launch_seq_schedule(const SeqParams& p, bool tree, cudaStream_t st);
lime_status launch_seq_merge(const SeqParams& p, int dtype, cudaStream_t st);
lime_status launch_seq_attn_tc(const SeqParams& p, bool tree, cudaStream_t st);        // bf16, d_h > 64
lime_status launch_seq_attn_d64_tc(const SeqParams& p, bool tree, cudaStream_t st);    // bf16, d_h <= 64
lime_status launch_seq_attn_few(const SeqParams& p, cudaStream_t st);                   // bf16, up to 8 stacked rows, the cache alone
lime_status launch_seq_attn_simt(const SeqParams& p, bool tree, bool few_rows, cudaStream_t st);  // fp32

}  // namespace lime

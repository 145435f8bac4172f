// C-ABI entry points of the sequence path: argument validation, workspace carving and launch sequencing.
#include <algorithm>
#include <cmath>

#include "seq_common.cuh"
#include "tc_common.cuh"

namespace lime {

static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// rows of `heads` heads at this stride: 16-byte aligned throughout, and no row over another
static bool stride_ok(int64_t stride, int heads, const Ctx* c) {
  const int es = c->cfg.dtype == LIME_F32 ? 4 : 2;
  return stride >= (int64_t)heads * c->seq.d_h && stride * es % 16 == 0 && stride <= (1ll << 36);
}
static lime_status ready(const Ctx* c) {
  if (!c->have_seq) return LIME_NOT_READY;
  int dev = -1;
  LIME_CUDA(cudaGetDevice(&dev));
  return dev == c->device ? LIME_OK : LIME_INVALID_ARG;
}
constexpr int64_t kMaxRows = 0x7fff0000LL;       // row indexes and the ends of the tiles that hold them stay inside 32 bits

// How the rows of a batch are tiled, and by which kernel.
//   STREAM: up to 8 stacked rows a user on average that attend to nothing but the cache (`alone`, bf16; k_seq_attn_few).  On the tensor
//     cores' tiles of 128 rows instead: 64 events of 16 heads over 4 heads of 128 221 against 180 us, 256 of 4 over 4 of 32 53 against 24.5,
//     one of 8 over 2 of 64 17 against 11.6.
//   TENSOR: tensor cores (bf16), 128 stacked rows a CTA and two CTAs an SM, or two slots of 128 rows.
//   CUDA16, CUDA64: CUDA cores (fp32), 16 stacked rows a tile where a user has no more on average, else 64 (64 for all, d_h = 64: 64 events of
//     8 heads over 100..3000 rows 148, 16 100 us; three rows over 2000 36.9, 27.6).
enum SeqForm { STREAM, TENSOR, CUDA16, CUDA64 };
static SeqForm form_of(const Ctx* c, int32_t B, int64_t rows, bool alone) {
  const int G = c->seq.Hq / c->seq.Hkv;
  if (c->cfg.dtype == LIME_BF16) return alone && G <= 8 && rows * G <= 8ll * B ? STREAM : TENSOR;
  return G <= 16 && rows * G <= 16ll * B ? CUDA16 : CUDA64;
}
// The tiles, and how fine a batch may be cut.  Pieces are worth a merge where there are few of them or little to merge; the figures are in
// us, the other choice first.
//   streamed rows: pieces of 4 tiles and more (2: 8 events over 500..5000 rows 25.6, now 18.0; 8: one event over 1000 14.0, 12.3), four a
//     CTA (2: 64 events over 16..16384 235, 217; 8: 232);
//   tensor cores: of 8 tiles and more, which cost a merge as much as 8 more (4 and 1: 64 events behind 16..8000 rows, 16 heads over 4 of 128
//     119, 108; 2 and 1: 8 events of 16 heads over one of 64 41.2, 26.7; but a draft of 5 over 1000 rows 20.8, 21.9);
//   CUDA cores, d_h = 64: of 2 tiles and more (4: 7 users' drafts 80.3, 73.8; the events 101, 90; the three rows 27.4, 23.4).
struct SeqTiling { int tok, kt, chunk_min, chunk_target, ctas; float item_cost, split_cost; };
static SeqTiling tiling(const Ctx* c, SeqForm form) {
  const int G = c->seq.Hq / c->seq.Hkv;
  const bool narrow = c->seq.d_h <= 64;
  SeqTiling t;
  if (form == STREAM) {
    t.tok = 8 / G;
    t.kt = 64;
    t.ctas = seq_few_blocks(c->seq.d_h) * kSMs;
    t.chunk_min = 4;
    t.item_cost = 4.f;
    t.split_cost = 2.f;
  } else if (form == TENSOR) {
    t.tok = (narrow ? 1 : 2) * (128 / G);
    t.kt = narrow ? 64 : 128;
    t.ctas = (narrow ? 2 : 1) * kSMs;
    t.chunk_min = 8;
    t.item_cost = narrow ? 4.f : 6.f;
    t.split_cost = 8.f;
  } else {
    t.tok = (form == CUDA16 ? 16 : 64) / G;
    t.kt = 64;
    t.ctas = (narrow ? 2 : 1) * kSMs;
    t.chunk_min = 2;
    t.item_cost = 2.f;
    t.split_cost = 1.f;
  }
  t.chunk_target = 4 * t.ctas;
  return t;
}

// Carves the workspace; returns its size, 0 where the lists would not count that many items.  Row tiles: whole ones and one rest per user.
// What k_seq_schedule calls a chunk is at least 1 / chunk_target of all (row tile, key head) work, so the row tiles longer than that, which
// it cuts, are fewer than chunk_target / Hkv, and a row tile has at most one piece more than chunks: pieces are bounded whatever the
// lengths, and each holds no more rows than the call has (one event of 16 over 4 heads of 128 3.8 MB; 158 with whole tiles and twice the
// chunks).  For one form the size grows with B and with rows.
static size_t carve(SeqParams& p, const Ctx* c, SeqForm form, int32_t B, int64_t rows, void* base) {
  const SeqTiling t = tiling(c, form);
  p.tok = t.tok; p.kt = t.kt; p.chunk_min = t.chunk_min; p.chunk_target = t.chunk_target;
  p.ctas = t.ctas; p.item_cost = t.item_cost; p.split_cost = t.split_cost;
  const int64_t row_tiles = rows / t.tok + (B < rows ? B : rows), cut = std::min(row_tiles, (int64_t)t.chunk_target / p.Hkv);
  const int64_t pieces = t.chunk_target / p.Hkv + cut;
  if (row_tiles + pieces > kMaxRows) return 0;
  p.row_tiles_upper = (int32_t)row_tiles;
  p.items_upper = (int32_t)(row_tiles + pieces);
  p.split_upper = (int32_t)cut;
  p.part_rows = (int32_t)std::min((int64_t)t.tok, rows) * p.G;
  size_t o = 0;
  char* at = static_cast<char*>(base);
  auto take = [&](size_t n) { void* r = at ? at + o : nullptr; o += (n + 255) & ~(size_t)255; return r; };
  p.plan = (SeqPlan*)take(sizeof(SeqPlan));
  p.tile_start = (int32_t*)take(((size_t)B + 1) * 4);
  p.items = (SeqItem*)take((size_t)p.items_upper * sizeof(SeqItem));
  p.splits = (SeqSplit*)take((size_t)p.split_upper * sizeof(SeqSplit));
  const size_t part_rows = cut > 0 ? (size_t)pieces * p.Hkv * p.part_rows : 0;
  p.part_ml = (float*)take(part_rows * 2 * 4);
  p.part_acc = (float*)take(part_rows * p.dh * 4);
  return o;
}

// the shape's part of the parameters
static SeqParams shape(const Ctx* c) {
  SeqParams p{};
  p.Hq = c->seq.Hq; p.Hkv = c->seq.Hkv; p.G = p.Hq / p.Hkv; p.dh = c->seq.d_h;
  p.scale_log2 = c->seq.attn_scale * 1.4426950408889634f;
  p.err = c->dev_err;
  return p;
}

static lime_status attend(const Ctx* c, SeqParams& p, bool tree, void* ws, size_t ws_bytes, cudaStream_t st) {
  const SeqForm form = form_of(c, p.B, p.q_rows, tree && p.k == nullptr);
  char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
  const size_t need = carve(p, c, form, p.B, p.q_rows, base);
  if (need == 0) return LIME_UNSUPPORTED_SHAPE;
  if (ws == nullptr || ws_bytes < need + (size_t)(base - static_cast<char*>(ws))) return LIME_WORKSPACE_TOO_SMALL;
  // what the host knows of the keys bounds the pieces as well
  const int64_t most = tree ? (int64_t)p.max_pages * p.page_rows + (p.k ? p.q_rows + p.kt : 0) : p.kv_rows;
  const int64_t tiles = (most + p.kt - 1) / p.kt + 1, pieces = (tiles - 1) / p.chunk_min + 1;
  // (with more heads of keys than chunk_target no row tile can be: a chunk is then longer than all of them together)
  const bool may_split = tiles > p.chunk_min && p.split_upper > 0;
  const int64_t items = may_split ? p.row_tiles_upper * pieces : p.row_tiles_upper;
  if (items < p.items_upper) p.items_upper = (int32_t)items;
  if ((int64_t)p.items_upper * p.Hkv > kMaxRows) return LIME_UNSUPPORTED_SHAPE;      // (a round of CTAs past the last item stays inside 32 bits)
  lime_status s;
  if ((s = launch_seq_schedule(p, tree, st)) != LIME_OK) return s;
  if (c->cfg.dtype != LIME_BF16) s = launch_seq_attn_simt(p, tree, form == CUDA16, st);
  else if (form == STREAM) s = launch_seq_attn_few(p, st);
  else s = p.dh <= 64 ? launch_seq_attn_d64_tc(p, tree, st) : launch_seq_attn_tc(p, tree, st);
  if (s != LIME_OK) return s;
  return may_split ? launch_seq_merge(p, c->cfg.dtype, st) : LIME_OK;
}

}  // namespace lime

using namespace lime;

extern "C" {

lime_status lime_set_sequence(lime_ctx* ctx, const lime_sequence* seq) {
  if (!ctx || !seq) return LIME_INVALID_ARG;
  lime_sequence g = *seq;
  if (g.Hq <= 0 || g.Hkv <= 0 || g.d_h <= 0 || g.rot_dim < 0 || (g.rot_interleaved != 0 && g.rot_interleaved != 1)) return LIME_INVALID_ARG;
  if (!(g.attn_scale >= 0.f) || !std::isfinite(g.attn_scale) || !(g.norm_eps >= 0.f) || !std::isfinite(g.norm_eps)) return LIME_INVALID_ARG;
  if (g.rot_base == 0.0) g.rot_base = 10000.0;
  if (!(g.rot_base >= 1.0 && g.rot_base <= 1e30)) return LIME_INVALID_ARG;
  if (g.rot_dim % 2 || g.rot_dim > g.d_h || g.Hq % g.Hkv) return LIME_INVALID_ARG;
  if (g.d_h % 8 || g.d_h > 128 || g.Hq / g.Hkv > 64 || g.Hq > 1024) return LIME_UNSUPPORTED_SHAPE;
  if (g.attn_scale == 0.f) g.attn_scale = 1.0f / sqrtf((float)g.d_h);
  if (g.norm_eps == 0.f) g.norm_eps = 1e-6f;
  Ctx* c = reinterpret_cast<Ctx*>(ctx);
  // base^(-2i / rot_dim) / (2 pi) turns per position, to 64 bits after the point
  const long double two_pi = 6.283185307179586476925286766559L;
  for (int i = 0; i < 64; ++i)
    c->rot_freq[i] = 2 * i < g.rot_dim ? (uint64_t)(powl((long double)g.rot_base, -2.0L * i / g.rot_dim) / two_pi * 18446744073709551616.0L + 0.5L) : 0;
  c->seq = g;
  c->have_seq = true;
  return LIME_OK;
}

lime_status lime_norm_rotate(lime_ctx* ctx, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                             int64_t v_stride, const void* gamma_q, const void* gamma_k, const int32_t* positions, int64_t rows,
                             void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* cache_k, void* cache_v,
                             int64_t cache_rows, const int32_t* slots, int32_t* dev_flag, void* stream) {
  if (!ctx || rows < 0 || rows > kMaxRows) return LIME_INVALID_ARG;
  const Ctx* c = reinterpret_cast<const Ctx*>(ctx);
  const lime_status s = ready(c);
  if (s != LIME_OK) return s;
  if (rows == 0) return LIME_OK;
  if (!q || !k || !q_out || (!k_out && !cache_k)) return LIME_INVALID_ARG;
  if ((cache_k != nullptr) != (slots != nullptr) || (v != nullptr) != (cache_v != nullptr) || (cache_v && !cache_k)) return LIME_INVALID_ARG;
  if (cache_k && (cache_rows <= 0 || cache_rows > kMaxRows)) return LIME_INVALID_ARG;
  if (c->seq.rot_dim > 0 && !positions) return LIME_INVALID_ARG;
  if (!stride_ok(q_stride, c->seq.Hq, c) || !stride_ok(k_stride, c->seq.Hkv, c) || !stride_ok(q_out_stride, c->seq.Hq, c)) return LIME_INVALID_ARG;
  if ((v && !stride_ok(v_stride, c->seq.Hkv, c)) || (k_out && !stride_ok(k_out_stride, c->seq.Hkv, c))) return LIME_INVALID_ARG;
  for (const void* x : {q, k, v, gamma_q, gamma_k, (const void*)q_out, (const void*)k_out, (const void*)cache_k, (const void*)cache_v})
    if (!aligned16(x)) return LIME_INVALID_ARG;
  NormRotateArgs a{};
  a.q = q; a.k = k; a.v = v; a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride; a.positions = positions; a.slots = slots; a.rows = rows;
  a.cache_rows = cache_k ? cache_rows : 0; a.q_out = q_out; a.k_out = k_out; a.cache_k = cache_k; a.cache_v = cache_v; a.dev_flag = dev_flag;
  a.dtype = c->cfg.dtype; a.seq = &c->seq; a.rot_freq = c->rot_freq;
  return launch_norm_rotate(a, static_cast<cudaStream_t>(stream));
}

size_t lime_sequence_workspace_bytes(const lime_ctx* ctx, int32_t B, int64_t rows) {
  if (!ctx || B < 0 || rows < 0 || rows > kMaxRows) return 0;
  const Ctx* c = reinterpret_cast<const Ctx*>(ctx);
  if (!c->have_seq) return 0;
  // Every form that a call of at most B users and rows can take, with the most users and rows that it can have then.  Fewer users may need
  // more: their rows are then many enough for larger tiles.
  const int64_t G = c->seq.Hq / c->seq.Hkv;
  const struct { SeqForm form; bool can; int64_t B, rows; } forms[4] = {
      {STREAM, c->cfg.dtype == LIME_BF16 && G <= 8, B, std::min(rows, 8 * (int64_t)B / G)},
      {TENSOR, c->cfg.dtype == LIME_BF16, B, rows},
      {CUDA16, c->cfg.dtype != LIME_BF16 && G <= 16, B, std::min(rows, 16 * (int64_t)B / G)},
      {CUDA64, c->cfg.dtype != LIME_BF16, G <= 16 && rows > 0 ? std::min((int64_t)B, (rows * G - 1) / 16) : B, rows}};
  size_t most = 0;
  for (const auto& f : forms) {
    if (!f.can || (f.form == CUDA64 && G <= 16 && rows * G <= 16)) continue;
    SeqParams p = shape(c);
    const size_t n = carve(p, c, f.form, (int32_t)f.B, f.rows, nullptr);
    if (n == 0) return 0;
    most = std::max(most, n);
  }
  return most + 256;
}

lime_status lime_attend_history(lime_ctx* ctx, const void* q, int64_t q_stride, const int32_t* off, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, const int32_t* kv_off, int32_t B, int64_t q_rows, int64_t kv_rows,
                                void* out, int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || B < 0 || q_rows < 0 || q_rows > kMaxRows || kv_rows < 0 || kv_rows > kMaxRows) return LIME_INVALID_ARG;
  const Ctx* c = reinterpret_cast<const Ctx*>(ctx);
  const lime_status s = ready(c);
  if (s != LIME_OK) return s;
  if (!kv_off && kv_rows != q_rows) return LIME_INVALID_ARG;
  if (B == 0 || q_rows == 0) return LIME_OK;
  if (!q || !off || !out || (kv_rows > 0 && (!k || !v))) return LIME_INVALID_ARG;
  if (!stride_ok(q_stride, c->seq.Hq, c) || !stride_ok(out_stride, c->seq.Hq, c)) return LIME_INVALID_ARG;
  if (kv_rows > 0 && (!stride_ok(k_stride, c->seq.Hkv, c) || !stride_ok(v_stride, c->seq.Hkv, c))) return LIME_INVALID_ARG;
  for (const void* x : {q, k, v, (const void*)out, (const void*)ws})
    if (!aligned16(x)) return LIME_INVALID_ARG;
  SeqParams p = shape(c);
  p.q = q; p.k = k; p.v = v; p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.out = out; p.out_stride = out_stride;
  p.off = off; p.kv_off = kv_off ? kv_off : off; p.B = B; p.q_rows = q_rows; p.kv_rows = kv_rows;
  return attend(c, p, false, ws, ws_bytes, static_cast<cudaStream_t>(stream));
}

lime_status lime_attend_tree(lime_ctx* ctx, const void* q, int64_t q_stride, const int32_t* off, const int32_t* parent,
                             const void* tree_k, int64_t tree_k_stride, const void* tree_v, int64_t tree_v_stride, int32_t B,
                             int64_t rows, const void* cache_k, const void* cache_v, int64_t n_pages, int32_t page_rows,
                             const int32_t* page_table, int32_t max_pages, const int32_t* ctx_len, int32_t* dev_flag, void* out,
                             int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || B < 0 || rows < 0 || rows > kMaxRows || n_pages < 0 || n_pages > kMaxRows || max_pages < 0) return LIME_INVALID_ARG;
  if (page_rows < 16 || page_rows > 4096 || (page_rows & (page_rows - 1)) != 0) return LIME_INVALID_ARG;
  if (n_pages * page_rows > kMaxRows || (int64_t)max_pages * page_rows > kMaxRows || (int64_t)B * max_pages > 0x7fffffffLL) return LIME_INVALID_ARG;
  const Ctx* c = reinterpret_cast<const Ctx*>(ctx);
  const lime_status s = ready(c);
  if (s != LIME_OK) return s;
  if ((tree_k != nullptr) != (tree_v != nullptr) || (parent && !tree_k)) return LIME_INVALID_ARG;
  if (B == 0 || rows == 0) return LIME_OK;
  if (!q || !off || !out || !ctx_len || (max_pages > 0 && !page_table) || (n_pages > 0 && (!cache_k || !cache_v))) return LIME_INVALID_ARG;
  if (!stride_ok(q_stride, c->seq.Hq, c) || !stride_ok(out_stride, c->seq.Hq, c)) return LIME_INVALID_ARG;
  if (tree_k && (!stride_ok(tree_k_stride, c->seq.Hkv, c) || !stride_ok(tree_v_stride, c->seq.Hkv, c))) return LIME_INVALID_ARG;
  for (const void* x : {q, tree_k, tree_v, cache_k, cache_v, (const void*)out, (const void*)ws})
    if (!aligned16(x)) return LIME_INVALID_ARG;
  SeqParams p = shape(c);
  p.q = q; p.k = tree_k; p.v = tree_v; p.q_stride = q_stride; p.k_stride = tree_k_stride; p.v_stride = tree_v_stride;
  p.out = out; p.out_stride = out_stride; p.off = off; p.parent = parent; p.table = page_table; p.ctx_len = ctx_len;
  p.ck = cache_k; p.cv = cache_v; p.dev_flag = dev_flag; p.n_pages = n_pages; p.page_rows = page_rows; p.max_pages = max_pages;
  while ((1 << p.page_shift) < page_rows) ++p.page_shift;
  p.B = B; p.q_rows = rows;
  return attend(c, p, true, ws, ws_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

// Work items of the sequence path's attention, and the join of row tiles that were cut into several.
#include "seq_common.cuh"

namespace lime {

constexpr int kSeqThreads = 1024, kSeqBins = 256;

// rows of user b, cut to what there is
__device__ __forceinline__ void seq_user_rows(const int32_t* off, int b, int64_t rows, int& first, int& n) {
  const int64_t lo = min(max((int64_t)__ldg(off + b), (int64_t)0), rows), hi = min(max((int64_t)__ldg(off + b + 1), lo), rows);
  first = (int)lo;
  n = (int)(hi - lo);
}

// row tile `i` of the batch as an item with all its key tiles
template <bool TREE>
__device__ SeqItem seq_row_tile(const SeqParams& p, int i) {
  int b = 0;                                       // the user: tile_start[b] <= i < tile_start[b + 1] (written by this block: plain loads)
  for (int hi = p.B; hi - b > 1;) {
    const int mid = (b + hi) >> 1;
    if (p.tile_start[mid] <= i) b = mid; else hi = mid;
  }
  int first, n;
  seq_user_rows(p.off, b, p.q_rows, first, n);
  const int at = (i - p.tile_start[b]) * p.tok;
  SeqItem it;
  it.row0 = first + at;
  it.rows = min(p.tok, n - at);
  it.part = -1;
  it.t0 = 0;
  if (TREE) {
    it.a = b;
    it.b = (int)min((int64_t)max(__ldg(p.ctx_len + b), 0), (int64_t)p.max_pages * p.page_rows);
    it.c = at;
    it.t1 = seq_tree_tiles(p, it) + (it.b + p.kt - 1) / p.kt;
  } else {
    int key0, nk;
    seq_user_rows(p.kv_off, b, p.kv_rows, key0, nk);
    it.a = key0;
    it.b = nk;
    it.c = at + 1 + (nk - n);
    it.t1 = (max(it.c + it.rows - 1, 0) + p.kt - 1) / p.kt;          // the last token sees no more than nk
  }
  return it;
}

// One block lists the items, the longest first: blocks start in the order of the list, so the short ones fill the end (1.3 ms of ragged
// causal tiles, say, end within one short item of each other).  How long an item may be follows from the whole batch's key tiles: where
// the row tiles alone do not occupy the card, they are cut.  Positions within a bin come from shared-memory counters, so the order of
// the list may differ from run to run; what an item computes, and the order in which parts are joined, does not depend on it.
template <bool TREE>
__global__ void __launch_bounds__(kSeqThreads) k_seq_schedule(const SeqParams p) {
  __shared__ int s_scan[32];
  __shared__ int s_base, s_items, s_parts, s_split, s_longest;
  __shared__ unsigned long long s_work;
  __shared__ int s_bin[kSeqBins];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  if (tid == 0) { s_base = 0; s_parts = 0; s_split = 0; s_longest = 0; s_work = 0; p.tile_start[0] = 0; }
  for (int i = tid; i < kSeqBins; i += kSeqThreads) s_bin[i] = 0;
  __syncthreads();
  // row tiles of every user, summed up
  for (int b0 = 0; b0 < p.B; b0 += kSeqThreads) {
    const int b = b0 + tid;
    int n = 0, first;
    if (b < p.B) { seq_user_rows(p.off, b, p.q_rows, first, n); n = (n + p.tok - 1) / p.tok; }
    int sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += x; }
    if (lane == 31) s_scan[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      int x = s_scan[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
      s_scan[lane] = x;
    }
    __syncthreads();
    const int before = s_base + (warp > 0 ? s_scan[warp - 1] : 0);
    // offsets that are not non-decreasing could make more tiles than the list has room for: no more are taken
    if (b < p.B) p.tile_start[b + 1] = min(before + sum, p.row_tiles_upper);
    __syncthreads();
    if (tid == 0) s_base += s_scan[31];
    __syncthreads();
  }
  const int tiles = p.B > 0 ? p.tile_start[p.B] : 0;
  // all key tiles, and the longest row tile
  {
    unsigned long long work = 0;
    int longest = 0;
    for (int i = tid; i < tiles; i += kSeqThreads) {
      const int len = seq_row_tile<TREE>(p, i).t1;
      work += (unsigned)len;
      longest = max(longest, len);
    }
    if (work != 0) { atomicAdd(&s_work, work); atomicMax(&s_longest, longest); }
  }
  __syncthreads();
  const long long want = ((long long)s_work * p.Hkv + p.chunk_target - 1) / p.chunk_target;
  const int chunk = (int)max((long long)p.chunk_min, min(want, (long long)0x7fffffff));
  const int bin_width = min(s_longest, chunk) / kSeqBins + 1;
  for (int i = tid; i < tiles; i += kSeqThreads) {
    const int len = seq_row_tile<TREE>(p, i).t1, ns = len > chunk ? (len - 1) / chunk + 1 : 1;
    atomicAdd(&s_bin[(len / ns) / bin_width], ns);
  }
  __syncthreads();
  if (warp == 0) {                                  // first position of every bin, the longest bin first
    int total = 0;
    for (int g = kSeqBins / 32 - 1; g >= 0; --g) {
      const int i = g * 32 + 31 - lane, n = s_bin[i];
      int sum = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += x; }
      s_bin[i] = total + sum - n;
      total += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) s_items = total;
  }
  __syncthreads();
  for (int i = tid; i < tiles; i += kSeqThreads) {
    SeqItem it = seq_row_tile<TREE>(p, i);
    const int len = it.t1, ns = len > chunk ? (len - 1) / chunk + 1 : 1;
    const int at = atomicAdd(&s_bin[(len / ns) / bin_width], ns);
    int part = -1;
    if (ns > 1) {
      part = atomicAdd(&s_parts, ns);
      const SeqSplit sp = {it.row0, it.rows, part, ns};
      p.splits[atomicAdd(&s_split, 1)] = sp;
    }
    for (int s = 0; s < ns; ++s) {
      it.t0 = (int)((long long)len * s / ns);
      it.t1 = (int)((long long)len * (s + 1) / ns);
      it.part = part < 0 ? -1 : part + s;
      p.items[at + s] = it;
    }
  }
  __syncthreads();
  if (tid == 0) { p.plan->n_items = s_items; p.plan->n_split = s_split; p.plan->n_parts = s_parts; p.plan->taken = 0; }
}

lime_status launch_seq_schedule(const SeqParams& p, bool tree, cudaStream_t st) {
  ProfScope _p("k_seq_schedule", st);
  if (tree) launch_pdl(k_seq_schedule<true>, dim3(1), dim3(kSeqThreads), 0, st, p);
  else launch_pdl(k_seq_schedule<false>, dim3(1), dim3(kSeqThreads), 0, st, p);
  LIME_LAUNCH_CHECK("k_seq_schedule");
  return LIME_OK;
}

// out = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s over the parts of a row tile; one warp per row, the parts in their order.
template <typename T>
__global__ void __launch_bounds__(256) k_seq_merge(const SeqParams p) {
  pdl_wait();
  const int lane = threadIdx.x & 31, R = p.tok * p.G;
  const int64_t n = (int64_t)p.plan->n_split * p.Hkv * R;
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < n; i += (int64_t)gridDim.x * 8) {
    const int r = (int)(i % R), kvh = (int)(i / R % p.Hkv);
    const SeqSplit sp = p.splits[i / R / p.Hkv];
    if (r >= sp.rows * p.G) continue;
    float m = -INFINITY;
    for (int s = lane; s < sp.n; s += 32) m = fmaxf(m, p.part_ml[(((int64_t)(sp.part0 + s) * p.Hkv + kvh) * 2) * R + r]);
    m = warp_max(m);
    if (m == -INFINITY) m = 0.f;
    float total = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < sp.n; ++s) {
      const int64_t at = (int64_t)(sp.part0 + s) * p.Hkv + kvh;
      const float w = exp2f(p.part_ml[at * 2 * R + r] - m);
      total += w * p.part_ml[(at * 2 + 1) * R + r];
      const float* a = p.part_acc + (at * R + r) * p.dh;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c * 32 + lane < p.dh) acc[c] += w * a[c * 32 + lane];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* o = static_cast<T*>(p.out) + (int64_t)(sp.row0 + r / p.G) * p.out_stride + (kvh * p.G + r % p.G) * p.dh;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c * 32 + lane < p.dh) Store<T>::st(o + c * 32 + lane, acc[c] * inv);
  }
}

lime_status launch_seq_merge(const SeqParams& p, int dtype, cudaStream_t st) {
  const int64_t rows = (int64_t)p.split_upper * p.Hkv * p.tok * p.G;
  const int64_t blocks = (rows + 7) / 8;
  const dim3 grid((unsigned)(blocks < kSMs * 8 ? blocks : kSMs * 8));
  ProfScope _p("k_seq_merge", st);
  if (dtype == LIME_BF16) launch_pdl(k_seq_merge<__nv_bfloat16>, grid, dim3(256), 0, st, p);
  else launch_pdl(k_seq_merge<float>, grid, dim3(256), 0, st, p);
  LIME_LAUNCH_CHECK("k_seq_merge");
  return LIME_OK;
}

}  // namespace lime

// Work items of the sequence path's attention, and the join of row tiles that were cut into several.
#include "seq_common.cuh"

namespace lime {

constexpr int kSeqThreads = 1024, kSeqBins = 64, kSeqNear = 2048;

// rows of user b, cut to what there is
__device__ __forceinline__ void seq_user_rows(const int32_t* off, int b, int64_t rows, int& first, int& n) {
  const int64_t lo = min(max((int64_t)__ldg(off + b), (int64_t)0), rows), hi = min(max((int64_t)__ldg(off + b + 1), lo), rows);
  first = (int)lo;
  n = (int)(hi - lo);
}

// row tile `i` of the batch as an item with all its key tiles
template <bool TREE>
__device__ __forceinline__ SeqItem seq_row_tile(const SeqParams& p, const int32_t* tile_start, int i) {
  int b = 0;                                       // the user: tile_start[b] <= i < tile_start[b + 1]
  for (int hi = p.B; hi - b > 1;) {
    const int mid = (b + hi) >> 1;
    if (tile_start[mid] <= i) b = mid; else hi = mid;
  }
  int first, n;
  seq_user_rows(p.off, b, p.q_rows, first, n);
  const int at = (i - tile_start[b]) * p.tok;
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

// One block lists the items, the longest first, to be dealt in that order: the short ones even out the end.  How long an item may be
// follows from the whole batch's key tiles: where the row tiles alone do not occupy the card, they are cut.  Positions within a bin come
// from shared-memory counters, so the order of the list may differ from run to run; what an item computes, and the order in which parts
// are joined, does not depend on it.  What this costs is latency, every kernel of the call waits for it: row tiles are looked up in shared
// memory (up to kSeqNear users), the first one of a thread stays in registers, and small batches take a small block, whose barriers are
// shorter (100 users of 0..1000 rows: 22 us by atomics and three lookups in global memory, 8.6 us now, both cold).
template <bool TREE>
__global__ void __launch_bounds__(kSeqThreads) k_seq_schedule(const SeqParams p) {
  __shared__ int s_scan[32], s_near[kSeqNear + 1], s_bin[kSeqBins], s_longest[32], s_pieces[8], s_len[8];
  __shared__ long long s_work[32];
  __shared__ int s_items, s_parts, s_split;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  pdl_wait();
  pdl_launch_dependents();
  int32_t* tile_start = p.B <= kSeqNear ? s_near : p.tile_start;
  if (tid == 0) { s_parts = 0; s_split = 0; tile_start[0] = 0; }
  if (tid < kSeqBins) s_bin[tid] = 0;
  // row tiles of every user, summed up
  int base = 0;
  for (int b0 = 0; b0 < p.B; b0 += threads) {
    const int b = b0 + tid;
    int n = 0, first;
    if (b < p.B) { seq_user_rows(p.off, b, p.q_rows, first, n); n = (n + p.tok - 1) / p.tok; }
    int sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += x; }
    if (b0 > 0) __syncthreads();
    if (lane == 31) s_scan[warp] = sum;
    __syncthreads();
    int before = lane < warps ? s_scan[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += x; }
    const int all = __shfl_sync(0xffffffffu, before, 31), mine = __shfl_sync(0xffffffffu, before, warp > 0 ? warp - 1 : 0);
    // offsets that are not non-decreasing could make more tiles than the list has room for: no more are taken
    if (b < p.B) tile_start[b + 1] = min(base + (warp > 0 ? mine : 0) + sum, p.row_tiles_upper);
    base = min(base + all, p.row_tiles_upper);
  }
  __syncthreads();
  const int tiles = base;
  // all key tiles, and the longest row tile
  SeqItem own;
  own.t1 = 0;
  long long work = 0;
  int longest = 0;
  for (int i = tid; i < tiles; i += threads) {
    const SeqItem it = seq_row_tile<TREE>(p, tile_start, i);
    if (i == tid) own = it;
    work += it.t1;
    longest = max(longest, it.t1);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { work += __shfl_xor_sync(0xffffffffu, work, o); longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o)); }
  if (lane == 0) { s_work[warp] = work; s_longest[warp] = longest; }
  __syncthreads();
  work = lane < warps ? s_work[lane] : 0;
  longest = lane < warps ? s_longest[lane] : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { work += __shfl_xor_sync(0xffffffffu, work, o); longest = max(longest, __shfl_xor_sync(0xffffffffu, longest, o)); }
  const long long want = (work * p.Hkv + p.chunk_target - 1) / p.chunk_target;
  int chunk = (int)max((long long)p.chunk_min, min(want, (long long)0x7fffffff));
  if ((long long)tiles * p.Hkv >= 4 * p.ctas) {
    chunk = (int)max((long long)chunk, (work * p.Hkv + 2 * p.ctas - 1) / (2 * p.ctas));        // a row tile that is half a CTA's share
  } else if ((long long)tiles * p.Hkv * ((longest - 1) / chunk + 1) > p.ctas) {
    // Few row tiles, but more pieces of the least length than run at once: the length that lets the CTAs finish first.  Eight lengths in
    // equal ratios from the shortest allowed to the longest row tile; with P pieces the end comes after a piece and the cost of an item
    // where all run at once, else after the CTAs' share of everything and half a piece.  Costs in key tiles.
    if (tid < 8) {
      s_pieces[tid] = 0;
      s_len[tid] = tid == 7 ? longest : min(longest, (int)(chunk * exp2f(log2f((float)longest / chunk) * ((float)tid / 7.f)) + 0.5f));
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < tiles; i += threads) {
      int l = own.t1;
      if (i != tid) l = seq_row_tile<TREE>(p, tile_start, i).t1;
#pragma unroll 1
      for (int c = 0; c < 8; ++c) atomicAdd(&s_pieces[c], l > s_len[c] ? (l - 1) / s_len[c] + 1 : 1);
    }
    __syncthreads();
    float best = 0.f;
    int best_len = chunk;
#pragma unroll 1
    for (int c = 0; c < 8; ++c) {
      const int len = s_len[c];
      const float all = (float)s_pieces[c] * p.Hkv, item = p.item_cost + (s_pieces[c] > tiles ? p.split_cost : 0.f);
      const float cost = all <= p.ctas ? len + item : ((float)work * p.Hkv + all * item) / p.ctas + 0.5f * (len + item);
      if (c == 0 || cost < best) { best = cost; best_len = len; }
    }
    chunk = best_len;
  }
  const int bin_width = min(longest, chunk) / kSeqBins + 1;
  for (int i = tid; i < tiles; i += threads) {
    const int len = i == tid ? own.t1 : seq_row_tile<TREE>(p, tile_start, i).t1, ns = len > chunk ? (len - 1) / chunk + 1 : 1;
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
  for (int i = tid; i < tiles; i += threads) {
    SeqItem it = own;
    if (i != tid) it = seq_row_tile<TREE>(p, tile_start, i);
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
  if (tid == 0) { p.plan->n_items = s_items; p.plan->n_split = s_split; }
}

lime_status launch_seq_schedule(const SeqParams& p, bool tree, cudaStream_t st) {
  const int want = p.row_tiles_upper > p.B ? p.row_tiles_upper : p.B, threads = want <= 128 ? 128 : want <= 512 ? 512 : kSeqThreads;
  ProfScope _p("k_seq_schedule", st);
  if (tree) launch_pdl(k_seq_schedule<true>, dim3(1), dim3(threads), 0, st, p);
  else launch_pdl(k_seq_schedule<false>, dim3(1), dim3(threads), 0, st, p);
  LIME_LAUNCH_CHECK("k_seq_schedule");
  return LIME_OK;
}

// out = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s over the parts of a row tile, in their order.  A block takes 32 rows of a (row
// tile, head of keys), a warp a row at a time, four features a lane, four parts in flight.
template <typename T>
__global__ void __launch_bounds__(256, 2) k_seq_merge(const SeqParams p) {
  pdl_wait();
  const int lane = threadIdx.x & 31, R = p.part_rows, pairs = p.plan->n_split * p.Hkv;
  const bool mine = lane * 4 < p.dh;
  for (int i = blockIdx.x; i < pairs; i += gridDim.x) {
    const int kvh = i % p.Hkv;
    const SeqSplit sp = p.splits[i / p.Hkv];
    const int end = min(sp.rows * p.G, (int)(blockIdx.y + 1) * 32);
    for (int r = (int)blockIdx.y * 32 + (int)(threadIdx.x >> 5); r < end; r += 8) {
      const float* ml = p.part_ml + ((int64_t)sp.part0 * p.Hkv + kvh) * 2 * R + r;            // + s * ml_step: maximum; + R: sum
      const float* acc_in = p.part_acc + (((int64_t)sp.part0 * p.Hkv + kvh) * R + r) * p.dh + lane * 4;
      const int64_t ml_step = (int64_t)p.Hkv * 2 * R, acc_step = (int64_t)p.Hkv * R * p.dh;
      // references of the first 32 parts stay in the lanes
      const float m_lane = lane < sp.n ? ml[lane * ml_step] : -INFINITY, l_lane = lane < sp.n ? ml[lane * ml_step + R] : 0.f;
      float m = m_lane;
      for (int s = lane + 32; s < sp.n; s += 32) m = fmaxf(m, ml[s * ml_step]);
      float total = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s0 = 0; s0 < sp.n; s0 += 4) {
        float4 a[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          a[u] = s0 + u < sp.n && mine ? *reinterpret_cast<const float4*>(acc_in + (s0 + u) * acc_step) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (s0 == 0) {
          m = warp_max(m);
          if (m == -INFINITY) m = 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int s = s0 + u;
          float ms = __shfl_sync(0xffffffffu, m_lane, s & 31), ls = __shfl_sync(0xffffffffu, l_lane, s & 31);
          if (s >= 32 && s < sp.n) { ms = ml[s * ml_step]; ls = ml[s * ml_step + R]; }
          if (s >= sp.n) break;
          const float w = exp2f(ms - m);
          total = fmaf(w, ls, total);
          acc.x = fmaf(w, a[u].x, acc.x); acc.y = fmaf(w, a[u].y, acc.y); acc.z = fmaf(w, a[u].z, acc.z); acc.w = fmaf(w, a[u].w, acc.w);
        }
      }
      const float inv = seq_inverse(total, true);                 // (a row tile that is cut has more key tiles than its rows could miss)
      T* o = static_cast<T*>(p.out) + (int64_t)(sp.row0 + r / p.G) * p.out_stride + (kvh * p.G + r % p.G) * p.dh + lane * 4;
      if (mine) { Store<T>::st(o, acc.x * inv); Store<T>::st(o + 1, acc.y * inv); Store<T>::st(o + 2, acc.z * inv); Store<T>::st(o + 3, acc.w * inv); }
    }
  }
}

lime_status launch_seq_merge(const SeqParams& p, int dtype, cudaStream_t st) {
  const int64_t pairs = (int64_t)p.split_upper * p.Hkv;
  const dim3 grid((unsigned)(pairs < 2 * kSMs ? pairs : 2 * kSMs), (unsigned)((p.part_rows + 31) / 32));
  ProfScope _p("k_seq_merge", st);
  if (dtype == LIME_BF16) launch_pdl(k_seq_merge<__nv_bfloat16>, grid, dim3(256), 0, st, p);
  else launch_pdl(k_seq_merge<float>, grid, dim3(256), 0, st, p);
  LIME_LAUNCH_CHECK("k_seq_merge");
  return LIME_OK;
}

}  // namespace lime

// Attention of the sequence path on the 5th-generation tensor cores (bf16, any d_h of the sequence path):
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(scale log2(e) (<q_i, k_j> - m_i))   over the keys j that row i sees
//
// A persistent CTA per SM takes the work items of k_seq_schedule one after the other (a counter deals them, the longest first).  An item
// is up to two slots of 128 stacked rows (tokens x the query heads of one head of keys) against key tiles of 128:
//   scores [128 x 128] = Q [128 x d_h] . K_tile^T      both operands from shared memory, where TMA leaves them 128-byte swizzled
//   O [128 x d_h]     += P [128 x 128] . V_tile        P as bf16 in tensor memory, over its own scores; V as it lies (MN-major)
// Two slots because one alone is a chain (scores, softmax, values) several times its tensor time: while the softmax warps of one work,
// the pipe works for the other.  An item of no more than 128 rows puts the same rows into both slots, which take the key tiles in turn
// and are joined in the end; so a single new event streams its cache through two chains.
//  * Warp 0 loads (one lane a page where keys lie in pages), warp 1 issues the scores, warp 2 the values, warp 3 mends value tiles (below)
//    and fetches items; warps 4..7 and 8..11 are the softmax of a slot, one thread per row.  Online softmax with lazy rescale: the
//    reference maximum is raised only when exceeded by 2^8.
//  * d_h that is not 64 or 128: TMA fills the columns that are not there with zeros in shared memory only, and the contractions stop at
//    the next multiple of 16.
//  * Probabilities are rounded to bf16 for the value product (the operands of one tcgen05.mma have one type); the row sum is taken of the
//    unrounded ones in fp32.
//  * Masked positions have p = 0, but 0 * NaN and 0 * infinity are NaN.  Value rows behind the end of a cached range, which may never have
//    been written, are zeroed in shared memory.  Elsewhere such values are the exception: an item whose result has a NaN or an infinity is
//    done again with what is not finite taken out of every tile that masks anything; the rows that do see it get it added at the end.
#include "seq_common.cuh"
#include "tc_common.cuh"

namespace lime {

template <int DHP_>
struct SeqTcCfg {
  static constexpr int DHP = DHP_, KT = 128, THREADS = 384, STAGES = DHP == 128 ? 5 : 10;
  static constexpr uint32_t SUB = 128 * 128;                       // [128 rows x 64 features]
  static constexpr uint32_t TILE = (DHP / 64) * SUB;
  static constexpr uint32_t OFF_Q = 0, OFF_KV = 2 * TILE, OFF_ML = OFF_KV + STAGES * TILE, OFF_BAR = OFF_ML + 4 * 128 * 4;
  static constexpr uint32_t SMEM = OFF_BAR + 512;
  static constexpr uint32_t COL_S = 0, COL_O = 256;                // scores: two of 128 columns; accumulators: two of DHP
  static constexpr int REGS_LAUNCH = 168, REGS_CONTROL = 88, REGS_SOFTMAX = 208;
  static_assert(128 * REGS_CONTROL + 256 * REGS_SOFTMAX <= THREADS * REGS_LAUNCH, "register split");
  static_assert(SMEM <= 232448 && COL_O + 2 * DHP <= 512, "budgets of one SM");
};
constexpr float kSeqRescale = 8.0f;                                // log2 units
constexpr int kRowNowhere = 0x7fff0000;                            // a row past the end of every tensor map: reads as zeros

__device__ __forceinline__ float seq_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t seq_pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* m, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

// An item as its warps see it: key tiles t0 .. t1 (the walk of seq_common.cuh), slot s takes those of [lo[s], hi[s]), or, where both
// slots hold the same rows (`same`), every other one.
template <bool TREE>
struct SeqWork {
  SeqItem it;
  int n_tree, ts;                 // tiles of new rows; tokens per slot
  bool same;
  int lo0, hi0;                   // slot 0 (slot 1 takes all of t0 .. t1)
  __device__ __forceinline__ SeqWork(const SeqParams& p, int idx) {
    const int4* src = reinterpret_cast<const int4*>(p.items + idx);
    const int4 x = src[0], y = src[1];
    it.row0 = x.x; it.rows = x.y; it.a = x.z; it.b = x.w; it.c = y.x; it.t0 = y.y; it.t1 = y.z; it.part = y.w;
    n_tree = TREE ? seq_tree_tiles(p, it) : 0;
    ts = p.tok / 2;
    same = it.rows <= ts;
    lo0 = it.t0; hi0 = it.t1;
    if (!same) {
      if (TREE) {
        if (n_tree > 0) lo0 = max(lo0, (it.c + it.rows + 127) / 128 - (it.c + ts + 127) / 128);
      } else {
        hi0 = min(hi0, (max(it.c + ts - 1, 0) + 127) / 128);
      }
    }
  }
  __device__ __forceinline__ bool takes(int s, int t) const { return same ? ((t - it.t0) & 1) == s : s == 1 || (t >= lo0 && t < hi0); }
  __device__ __forceinline__ int first_token(int s) const { return same ? 0 : s * ts; }
  __device__ __forceinline__ int tokens(int s) const { return same ? it.rows : s == 0 ? ts : it.rows - ts; }
  // whether a row of the item does not see all keys of the tile
  __device__ __forceinline__ bool masked(const SeqTile& k) const { return k.kind == 2 || (k.kind == 0 ? k.j0 + 128 > it.c : k.j0 + 128 > k.n); }
  // whether the value tile is mended: see the top
  __device__ __forceinline__ bool mended(const SeqTile& k, bool again) const { return again ? masked(k) : TREE && k.kind == 1 && k.j0 + 128 > k.n; }
};

__device__ __forceinline__ bool not_finite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Adds to a[0..31] (columns c0.. of a row's result) the values that are not finite of the keys that the row sees in masked tiles.
template <bool TREE>
__device__ __noinline__ void seq_add_not_finite(const SeqParams& p, const SeqWork<TREE>& w, int token, int kvh, int lo, int hi, int c0, float (&a)[32]) {
  const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v);
  auto add = [&](const __nv_bfloat16* row) {
    for (int c = 0; c < 32; ++c)
      if (c0 + c < p.dh) {
        const float x = __bfloat162float(row[c0 + c]);
        if (!(fabsf(x) < INFINITY)) a[c] += x;
      }
  };
  for (int t = lo; t < hi; ++t) {
    const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
    if (!w.masked(k)) continue;
    if (TREE && k.kind == 2) {
      for (int j = w.it.c + token; j >= k.j0; j = seq_parent(p, w.it.row0 - w.it.c, j))
        if (j < k.j0 + 128) add(v + (int64_t)(w.it.row0 - w.it.c + j) * p.v_stride + kvh * p.dh);
    } else {
      const int end = min(k.j0 + 128, TREE ? k.n : w.it.c + token);
      for (int j = k.j0; j < end; ++j) {
        if (!TREE) {
          add(v + (int64_t)(w.it.a + j) * p.v_stride + kvh * p.dh);
        } else {
          const int64_t pg = seq_page(p, w.it.a, j);
          if (pg < p.n_pages) add(static_cast<const __nv_bfloat16*>(p.cv) + ((pg * p.page_rows + (j & (p.page_rows - 1))) * p.Hkv + kvh) * p.dh);
        }
      }
    }
  }
}

template <int DHP, bool TREE>
__global__ void __launch_bounds__(384, 1)
k_seq_attn_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ CUtensorMap tmCK, const __grid_constant__ CUtensorMap tmCV, const __grid_constant__ SeqParams p) {
  using namespace tc;
  using C = SeqTcCfg<DHP>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {                     // the swizzled tiles need a 1024-byte aligned base
    pdl_wait();
    if (threadIdx.x == 0) atomicCAS(p.err, 0, 110);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* kv_full = bars;            // [10] keys or values of a tile landed
  uint64_t* kv_empty = bars + 10;      // [10] every MMA that reads them has run
  uint64_t* q_full = bars + 20;
  uint64_t* s_full = bars + 21;        // [2]  scores of the slot in TMEM
  uint64_t* s_free = bars + 23;        // [2]  the values of the slot's last probabilities are issued: new scores may follow in the pipe
  uint64_t* p_ready = bars + 25;       // [2]  probabilities in TMEM (four warps)
  uint64_t* pv_done = bars + 27;       // [2]  the slot's accumulator is up to date
  uint64_t* mend_done = bars + 29;     // [10] the value tile in this stage is mended
  int* s_next = reinterpret_cast<int*>(bars + 39);          // [2 parities]
  int* s_flags = s_next + 2;           // [3] of a pass: 1 a result is not finite, 2 a wait gave up, 4 values were taken out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_flags + 3);
  float* s_ml = reinterpret_cast<float*>(smem + C::OFF_ML);   // [2 slots][2][128]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); mbar_init(&mend_done[i], 1); }
    mbar_init(q_full, 1);
    for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&s_free[i], 1); mbar_init(&p_ready[i], 4); mbar_init(&pv_done[i], 1); }
    s_flags[0] = s_flags[1] = s_flags[2] = 0;
    fence_barrier_init();
    prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    if (TREE) { prefetch_tmap(&tmCK); prefetch_tmap(&tmCV); }
  }
  if (warp == 1) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  const int n_work = p.plan->n_items * p.Hkv, G = p.G;
  const int ksteps = (p.dh + 15) / 16;                      // of 16 features
  int work = (int)blockIdx.x, turn = 0, pass_no = 0;        // an item and head of keys; how many this CTA has taken; passes over items

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CONTROL));
    const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0);
    int g = 0;                                               // K and V tiles seen so far (ring position)
    uint32_t ph0 = 0, ph1 = 0;                               // phase of the slot's barrier that this role waits for
    uint32_t q_ph = 0, mend_ph = 0;                          // mend_ph: a bit for every stage
    for (; work < n_work; ++turn) {
      const int kvh = work % p.Hkv;
      const SeqWork<TREE> w(p, work / p.Hkv);
      for (int pass = 0;; ++pass, ++pass_no) {
        const bool again = pass > 0;
        bool ok = true;
        if (warp == 0) {
          // ---------------------------------------------------------------- loads
          if (!again && w.it.t0 < w.it.t1) {
            if (lane == 0) {
              mbar_arrive_expect_tx(q_full, (w.same ? 1u : 2u) * (uint32_t)(w.ts * G) * 128u * (DHP / 64));
              for (int s = 0; s < (w.same ? 1 : 2); ++s)
                for (int c = 0; c < DHP / 64; ++c)
                  tma_load_3d(smem + C::OFF_Q + s * C::TILE + c * C::SUB, &tmQ, c * 64, kvh * G, w.it.row0 + s * w.ts, q_full);
            }
            __syncwarp();
          }
          const int box = min(p.page_rows, 128);             // rows of a page in one copy
          int row = 0;                                       // of the lane's page of the coming tile of cached rows
          auto look_up = [&](int t) {
            if (!TREE || t >= w.it.t1) return;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            const int j = k.j0 + lane * box;
            if (k.kind != 1 || lane * box >= 128 || j >= k.n) return;
            const int64_t pg = seq_page(p, w.it.a, j);
            row = pg < p.n_pages ? (int)(pg * p.page_rows + (j & (p.page_rows - 1))) : kRowNowhere;
          };
          look_up(w.it.t0);
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t) {
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            const int my_row = row;
            look_up(t + 1);
            for (int kv = 0; kv < 2; ++kv, ++g) {
              const int s = g % STAGES;
              if (!__all_sync(0xffffffffu, mbar_wait(&kv_empty[s], ((uint32_t)(g / STAGES) & 1u) ^ 1u, p.err, 111))) { ok = false; break; }
              uint8_t* dst = smem + C::OFF_KV + s * C::TILE;
              if (TREE && k.kind == 1) {
                const int n_box = min(128 / box, (k.n - k.j0 + box - 1) / box);
                if (lane == 0) mbar_arrive_expect_tx(&kv_full[s], (uint32_t)(n_box * box) * 128u * (DHP / 64));
                __syncwarp();
                if (lane < n_box)
                  for (int c = 0; c < DHP / 64; ++c)
                    tma_load_3d(dst + c * C::SUB + lane * box * 128, kv ? &tmCV : &tmCK, c * 64, kvh, my_row, &kv_full[s]);
              } else if (lane == 0) {
                mbar_arrive_expect_tx(&kv_full[s], C::TILE);
                const int r = (TREE ? w.it.row0 - w.it.c : w.it.a) + k.j0;
                for (int c = 0; c < DHP / 64; ++c) tma_load_3d(dst + c * C::SUB, kv ? &tmV : &tmK, c * 64, kvh, r, &kv_full[s]);
              }
              __syncwarp();
            }
          }
        } else if (warp == 1) {
          // ---------------------------------------------------------------- scores
          const uint32_t idesc = make_idesc_bf16(128, 128);
          const uint64_t dq0 = make_sdesc_k_sw128(smem_u32(smem) + C::OFF_Q), dk0 = make_sdesc_k_sw128(smem_u32(smem) + C::OFF_KV);
          if (!again && w.it.t0 < w.it.t1) {
            ok = __all_sync(0xffffffffu, mbar_wait(q_full, q_ph, p.err, 112));
            q_ph ^= 1u;
          }
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            const int st = g % STAGES;
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[st], (uint32_t)(g / STAGES) & 1u, p.err, 113))) { ok = false; break; }
            const uint64_t dk = dk0 + (uint64_t)((uint32_t)st * C::TILE >> 4);
            for (int s = 0; s < 2; ++s) {
              if (!w.takes(s, t)) continue;
              uint32_t& ph = s == 0 ? ph0 : ph1;
              if (!__all_sync(0xffffffffu, mbar_wait(&s_free[s], ph ^ 1u, p.err, 114))) { ok = false; break; }
              ph ^= 1u;
              tc_fence_after();
              const uint64_t dq = dq0 + (uint64_t)(w.same ? 0u : (uint32_t)s * C::TILE >> 4);
              if (elect_one()) {
                for (int kk = 0; kk < ksteps; ++kk) {
                  const uint64_t at = (uint64_t)(((kk >> 2) * C::SUB + (kk & 3) * 32) >> 4);
                  mma_bf16_ss(tmem_u + C::COL_S + (uint32_t)s * 128, dq + at, dk + at, idesc, kk != 0);
                }
                mma_commit(&s_full[s]);
              }
              __syncwarp();
            }
            if (ok && elect_one()) mma_commit(&kv_empty[st]);
            __syncwarp();
          }
        } else if (warp == 2) {
          // ---------------------------------------------------------------- values
          const uint32_t idesc = make_idesc_bf16(128, ksteps * 16, false, true);
          const uint64_t dv0 = make_sdesc_mn_sw128(smem_u32(smem) + C::OFF_KV, C::SUB);
          bool first0 = true, first1 = true;
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            const int st = (g + 1) % STAGES;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[st], (uint32_t)((g + 1) / STAGES) & 1u, p.err, 115))) { ok = false; break; }
            if (w.mended(k, again)) {
              if (!__all_sync(0xffffffffu, mbar_wait(&mend_done[st], (mend_ph >> st) & 1u, p.err, 116))) { ok = false; break; }
              mend_ph ^= 1u << st;
            }
            const uint64_t dv = dv0 + (uint64_t)((uint32_t)st * C::TILE >> 4);
            for (int s = 0; s < 2; ++s) {
              if (!w.takes(s, t)) continue;
              uint32_t& ph = s == 0 ? ph0 : ph1;
              bool& first = s == 0 ? first0 : first1;
              if (!__all_sync(0xffffffffu, mbar_wait(&p_ready[s], ph, p.err, 117))) { ok = false; break; }
              ph ^= 1u;
              tc_fence_after();
              if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                  mma_bf16_ts(tmem_u + C::COL_O + (uint32_t)(s * DHP), tmem_u + C::COL_S + (uint32_t)(s * 128 + kk * 8), dv + ((kk * 2048) >> 4), idesc,
                              kk != 0 || !first ? 1u : 0u);
                mma_commit(&pv_done[s]);
                tc_fence_before();
                mbar_arrive(&s_free[s]);
              }
              first = false;
              __syncwarp();
            }
            if (ok && elect_one()) mma_commit(&kv_empty[st]);
            __syncwarp();
          }
        } else {
          // ---------------------------------------------------------------- items and mended value tiles
          if (lane == 0) {
            s_flags[(pass_no + 1) % 3] = 0;                  // nobody reads or sets it before the next pass
            if (!again) s_next[turn & 1] = atomicAdd(&p.plan->taken, 1) + (int)gridDim.x;
          }
          // Every load of the item is waited for, so that a stage's phase is never taken for the one two before it; not at all where
          // nothing is mended (a cached range ends in the last tile).
          const bool any = w.it.t0 < w.it.t1 && (again || w.mended(seq_tile<TREE>(p, w.it, w.n_tree, w.it.t1 - 1), false));
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            if (!any) continue;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            const int st = (g + 1) % STAGES;
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[g % STAGES], (uint32_t)(g / STAGES) & 1u, p.err, 119) &&
                                             mbar_wait(&kv_full[st], (uint32_t)((g + 1) / STAGES) & 1u, p.err, 118))) { ok = false; break; }
            if (!w.mended(k, again)) continue;
            uint8_t* tile = smem + C::OFF_KV + st * C::TILE;
            const int n = k.n - k.j0;                        // rows of the tile that there are
            bool out = false;
            for (int i = lane; i < 128 * (DHP / 64) * 8; i += 32) {
              const int r = (i >> 3) & 127;
              if (r < n && !again) continue;
              uint4* at = reinterpret_cast<uint4*>(tile + (i >> 10) * C::SUB + (i & 1023) * 16);
              uint4 x = make_uint4(0, 0, 0, 0);
              if (r < n) {
                x = *at;
                uint32_t* u = reinterpret_cast<uint32_t*>(&x);
                bool any = false;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (not_finite2(u[e])) {
                    any = true;
                    if ((u[e] & 0x7f80u) == 0x7f80u) u[e] &= 0xffff0000u;
                    if ((u[e] & 0x7f800000u) == 0x7f800000u) u[e] &= 0xffffu;
                  }
                if (!any) continue;
                out = true;
              }
              *at = x;
            }
            if (out) atomicOr(&s_flags[pass_no % 3], 4);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&mend_done[st]);
          }
        }
        if (!ok && lane == 0) atomicOr(&s_flags[pass_no % 3], 2);
        __syncthreads();
        const int flags = s_flags[pass_no % 3];
        if ((flags & 2) && warp == 0) {
          // giving up: let the copies already issued land (bounded) before this CTA's shared memory goes away
          for (int j = 0; j < g && j < STAGES; ++j) mbar_wait_quiet(&kv_full[(g - 1 - j) % STAGES], (uint32_t)((g - 1 - j) / STAGES) & 1u);
        }
        __syncthreads();
        if (flags & 2) { work = n_work; break; }
        if (!(flags & 1) || again) { work = s_next[turn & 1]; ++pass_no; break; }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_SOFTMAX));
    // -------------------------------------------------------------------- softmax of a slot
    const int s = (warp - 4) >> 2, q = warp & 3;             // slot; TMEM lane quarter of this warp
    const int r = q * 32 + lane;                             // stacked row
    const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
    const uint32_t s_addr = lane_addr + C::COL_S + (uint32_t)s * 128, o_addr = lane_addr + C::COL_O + (uint32_t)(s * DHP);
    const float scale = p.scale_log2;
    uint32_t s_ph = 0, pv_ph = 0;                            // pv_ph: of the slot's next value contraction
    for (; work < n_work; ++turn) {
      const int kvh = work % p.Hkv;
      const SeqWork<TREE> w(p, work / p.Hkv);
      const int rows = w.tokens(s) * G, tok = w.first_token(s) + min(r, max(rows - 1, 0)) / G;
      const bool valid = r < rows, any_valid = q * 32 < rows;
      bool mine = false;                                     // the slot took a tile: its accumulator holds something
      for (int pass = 0;; ++pass, ++pass_no) {
        bool ok = true;
        float m = -INFINITY, l = 0.f;
        int anc = w.it.c + tok;
        mine = false;
        for (int t = w.it.t0; t < w.it.t1; ++t) {
          if (!w.takes(s, t)) continue;
          const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
          if (!__all_sync(0xffffffffu, mbar_wait(&s_full[s], s_ph, p.err, 120))) { ok = false; break; }
          s_ph ^= 1u;
          if (any_valid) {
            tc_fence_after();
            float v[128];
#pragma unroll
            for (int c = 0; c < 128; c += 32) tmem_ld_32x32(s_addr + c, *reinterpret_cast<float(*)[32]>(&v[c]));
            tmem_wait_ld();
            if (TREE && k.kind == 2) {
              uint32_t see[4] = {0u, 0u, 0u, 0u};
              while (anc >= k.j0 + 128) anc = seq_parent(p, w.it.row0 - w.it.c, anc);
              while (anc >= k.j0) {
                const int b = anc - k.j0;
#pragma unroll
                for (int i = 0; i < 4; ++i) see[i] |= (b >> 5) == i ? 1u << (b & 31) : 0u;
                anc = seq_parent(p, w.it.row0 - w.it.c, anc);
              }
#pragma unroll
              for (int j = 0; j < 128; ++j)
                if (((see[j >> 5] >> (j & 31)) & 1u) == 0) v[j] = -INFINITY;
            } else {
              const int n = (k.kind == 0 ? w.it.c + tok : k.n) - k.j0;           // keys of the tile that the row sees
              if (__any_sync(0xffffffffu, n < 128)) {
#pragma unroll
                for (int j = 0; j < 128; ++j)
                  if (j >= n) v[j] = -INFINITY;
              }
            }
            float mx0 = v[0], mx1 = v[1], mx2 = v[2], mx3 = v[3];
#pragma unroll
            for (int j = 4; j < 128; j += 4) {
              mx0 = fmaxf(mx0, v[j]); mx1 = fmaxf(mx1, v[j + 1]); mx2 = fmaxf(mx2, v[j + 2]); mx3 = fmaxf(mx3, v[j + 3]);
            }
            const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
            // raise the reference only when it is exceeded by more than the threshold, or unset
            const bool need = valid && (mx - m) * scale > kSeqRescale;
            const float m_new = need ? mx : m;
            const float factor = need && m != -INFINITY ? seq_ex2((m - m_new) * scale) : 1.f;
            if (mine && __any_sync(0xffffffffu, need)) {
              if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 121))) { ok = false; break; }
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < DHP; c += 32) {
                float a[32];
                tmem_ld_32x32(o_addr + c, a);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 32; ++j) a[j] *= factor;
                tmem_st_32x32(o_addr + c, a);
              }
            }
            l *= factor;
            m = m_new;
            const float ref = m == -INFINITY ? 0.f : m * scale;
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
            const float2 sc2 = make_float2(scale, scale), rf2 = make_float2(-ref, -ref);
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              float packed[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                float2 e = __ffma2_rn(make_float2(v[c + 2 * j], v[c + 2 * j + 1]), sc2, rf2);
                e = make_float2(seq_ex2(e.x), seq_ex2(e.y));
                if (j & 1) s1 = __fadd2_rn(s1, e); else s0 = __fadd2_rn(s0, e);
                packed[j] = __uint_as_float(seq_pack(e.x, e.y));
              }
              tmem_st_32x16(s_addr + (uint32_t)(c >> 1), packed);
            }
            s0 = __fadd2_rn(s0, s1);
            l += s0.x + s0.y;
            tmem_wait_st();
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_ready[s]);
          pv_ph ^= 1u;
          mine = true;
        }
        // the slot's result complete?  any of it not finite?
        bool bad = false;
        if (mine && ok) {
          ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 122));
          tc_fence_after();
          if (ok && any_valid && pass == 0) {
            float z = 0.f;
#pragma unroll 1
            for (int c = 0; c < ksteps * 16; c += 16) {
              float a[16];
              tmem_ld_32x16(o_addr + c, a);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; ++j) z = fmaf(a[j], 0.f, z);
            }
            bad = valid && z != 0.f;                         // 0 * infinity and 0 * NaN
          }
        }
        if (w.same) { s_ml[s * 256 + r] = m; s_ml[s * 256 + 128 + r] = mine ? l : 0.f; }
        if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(&s_flags[pass_no % 3], 1);
        if (!ok && lane == 0) atomicOr(&s_flags[pass_no % 3], 2);
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        const int flags = s_flags[pass_no % 3];
        const bool last = !(flags & 1) || pass > 0;
        if (last && !(flags & 2) && any_valid) {
          // ---------------------------------------------------------------- result: the slot's rows, or the half of the columns of both's
          float w0 = 1.f, w1 = 0.f;                          // of this slot's accumulator and the other's
          bool have0 = mine, have1 = false;
          if (w.same) {
            const float mo = s_ml[(s ^ 1) * 256 + r], lo = s_ml[(s ^ 1) * 256 + 128 + r], mm = fmaxf(m, mo);
            const float ref = mm == -INFINITY ? 0.f : mm;
            have1 = w.it.t1 - w.it.t0 > (s ^ 1);
            w0 = seq_ex2((m - ref) * scale); w1 = seq_ex2((mo - ref) * scale);
            l = l * w0 + lo * w1;
            m = mm;
          }
          const int c_lo = w.same ? s * (DHP / 2) : 0, c_hi = w.same ? c_lo + DHP / 2 : DHP;
          const uint32_t other = lane_addr + C::COL_O + (uint32_t)((s ^ 1) * DHP);
          const int64_t part = (int64_t)w.it.part * p.Hkv + kvh;
          const int R = p.tok * G, pr = w.first_token(s) * G + r;
          if (w.it.part >= 0 && valid && (s == 0 || !w.same)) {
            p.part_ml[part * 2 * R + pr] = m == -INFINITY ? m : m * scale;
            p.part_ml[(part * 2 + 1) * R + pr] = l;
          }
          const float inv = w.it.part >= 0 ? 1.f : l == 0.f ? 0.f : 1.f / l;
          uint8_t* stage = smem + C::OFF_Q + s * C::TILE + q * (C::TILE / 4);    // this warp's rows (the queries are done with)
#pragma unroll 1
          for (int c = c_lo; c < c_hi; c += 32) {
            float a[32];
            if (have0) {
              tmem_ld_32x32(o_addr + c, a);
              tmem_wait_ld();
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) a[j] = have0 ? a[j] * w0 : 0.f;
            if (have1) {
              float b[32];
              tmem_ld_32x32(other + c, b);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; ++j) a[j] = fmaf(b[j], w1, a[j]);
            }
            if ((flags & 4) && valid) seq_add_not_finite<TREE>(p, w, tok, kvh, w.same || s == 1 ? w.it.t0 : w.lo0, w.same || s == 1 ? w.it.t1 : w.hi0, c, a);
            __syncwarp();
            if (w.it.part >= 0) {
              if (valid) {
                float* dst = p.part_acc + (part * R + pr) * p.dh + c;
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                  if (c + j < p.dh) *reinterpret_cast<float4*>(dst + j) = make_float4(a[j], a[j + 1], a[j + 2], a[j + 3]);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 32; j += 8)
                *reinterpret_cast<uint4*>(stage + lane * (DHP * 2) + ((((c - c_lo + j) >> 3) ^ (lane & 7)) << 4)) =
                    make_uint4(seq_pack(a[j] * inv, a[j + 1] * inv), seq_pack(a[j + 2] * inv, a[j + 3] * inv), seq_pack(a[j + 4] * inv, a[j + 5] * inv),
                               seq_pack(a[j + 6] * inv, a[j + 7] * inv));
            }
          }
          if (w.it.part < 0) {
            __syncwarp();
            const int chunks = (c_hi - c_lo) / 8, per = 32 / chunks;             // 16-byte pieces of a row; rows a store covers
            for (int i = 0; i < 32; i += per) {
              const int rr = i + lane / chunks, ch = lane % chunks, row = q * 32 + rr;
              if (row < rows && c_lo + ch * 8 < p.dh) {
                const uint4 x = *reinterpret_cast<const uint4*>(stage + rr * (DHP * 2) + ((ch ^ (rr & 7)) << 4));
                const int token = w.first_token(s) + row / G;
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + (int64_t)(w.it.row0 + token) * p.out_stride + (kvh * G + row % G) * p.dh + c_lo + ch * 8) = x;
              }
            }
          }
        }
        tc_fence_before();
        fence_proxy_async_smem();                            // the next queries arrive by TMA where the rows were staged
        __syncthreads();
        if (flags & 2) { work = n_work; break; }
        if (last) { work = s_next[turn & 1]; ++pass_no; break; }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int DHP, bool TREE>
static lime_status launch_tc(const SeqParams& p, cudaStream_t st) {
  using C = SeqTcCfg<DHP>;
  static bool set[kMaxDeviceOrdinals] = {};
  CUtensorMap q, k, v, ck, cv;
  // maps of tensors that are not there stand on the queries and are not read inside
  const bool fresh = p.k != nullptr && (TREE ? true : p.kv_rows > 0), pages = TREE && p.n_pages > 0;
  const uint64_t rows = fresh ? (uint64_t)(TREE ? p.q_rows : p.kv_rows) : 1;
  bool ok = make_tmap_bf16_heads(&q, p.q, p.Hq, p.dh, (uint64_t)p.q_rows, p.q_stride, p.G, p.tok / 2);
  ok = ok && make_tmap_bf16_heads(&k, fresh ? p.k : p.q, p.Hkv, p.dh, rows, fresh ? p.k_stride : p.q_stride, 1, 128);
  ok = ok && make_tmap_bf16_heads(&v, fresh ? p.v : p.q, p.Hkv, p.dh, rows, fresh ? p.v_stride : p.q_stride, 1, 128);
  const uint64_t crows = pages ? (uint64_t)(p.n_pages * p.page_rows) : 1;
  const uint32_t box = TREE ? (uint32_t)(p.page_rows < 128 ? p.page_rows : 128) : 128;
  ok = ok && make_tmap_bf16_heads(&ck, pages ? p.ck : p.q, p.Hkv, p.dh, crows, (uint64_t)p.Hkv * p.dh, 1, box);
  ok = ok && make_tmap_bf16_heads(&cv, pages ? p.cv : p.q, p.Hkv, p.dh, crows, (uint64_t)p.Hkv * p.dh, 1, box);
  if (!ok) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  const lime_status s = ensure_dynamic_smem((const void*)k_seq_attn_tc<DHP, TREE>, (int)C::SMEM, set);
  if (s != LIME_OK) return s;
  const int64_t work = (int64_t)p.items_upper * p.Hkv;
  ProfScope _p("k_seq_attn_tc", st);
  launch_pdl(k_seq_attn_tc<DHP, TREE>, dim3((unsigned)(work < kSMs ? work : kSMs)), dim3(C::THREADS), C::SMEM, st, q, k, v, ck, cv, p);
  LIME_LAUNCH_CHECK("k_seq_attn_tc");
  return LIME_OK;
}

lime_status launch_seq_attn_tc(const SeqParams& p, bool tree, cudaStream_t st) {
  if (p.dh <= 64) return tree ? launch_tc<64, true>(p, st) : launch_tc<64, false>(p, st);
  return tree ? launch_tc<128, true>(p, st) : launch_tc<128, false>(p, st);
}

}  // namespace lime

// Attention of the sequence path on the 5th-generation tensor cores (bf16, any d_h of the sequence path):
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(scale log2(e) (<q_i, k_j> - m_i))   over the keys j that row i sees
//
// A persistent CTA per SM walks its share of the work items of k_seq_schedule (dealt in their order, back and forth, so the longest come
// first and rounds even out).  An item is up to two slots of 128 stacked rows (tokens x the query heads of one head of keys) against key
// tiles of 128:
//   scores [128 x 128] = Q [128 x d_h] . K_tile^T      both operands from shared memory, where TMA leaves them 128-byte swizzled
//   O [128 x d_h]     += P [128 x 128] . V_tile        P as bf16 in tensor memory, over its own scores; V as it lies (MN-major)
// Two slots because one alone is a chain (scores, softmax, values) several times its tensor time: while the softmax warps of one work,
// the pipe works for the other.  An item of no more than 128 rows puts the same rows into both slots, which take the key tiles in turn
// and are joined in the end; so a single new event streams its cache through two chains.
//  * Warp 0 loads (one lane a page where keys lie in pages), warp 1 issues the scores, warp 2 the values, warp 3 mends value tiles (below);
//    warps 4..7 and 8..11 are the softmax of a slot, one thread per row.  Online softmax with lazy rescale: the reference maximum is
//    raised only when exceeded by 2^8.
//  * Nothing waits for the end of an item but what needs it: the next one's keys and queries are loaded and its first scores formed while
//    the softmax warps write a result out (100 users of 0..1000 rows, 4 heads of 32: LIME_TODO us with a barrier of the CTA between items).
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
  static constexpr int DHP = DHP_, THREADS = 384, STAGES = DHP == 128 ? 5 : 10, QBUFS = DHP == 128 ? 1 : 2;
  static constexpr uint32_t SUB = 128 * 128;                       // [128 rows x 64 features]
  static constexpr uint32_t TILE = (DHP / 64) * SUB;
  static constexpr uint32_t OFF_Q = 0, OFF_KV = QBUFS * 2 * TILE, OFF_BAR = OFF_KV + STAGES * TILE;
  static constexpr uint32_t OFF_ML = OFF_BAR + 512;               // references and sums of joined slots: [2 slots][128] pairs
  static constexpr uint32_t OFF_BAD = OFF_ML + 2 * 128 * 8;       // a bit for every item of the CTA
  static constexpr uint32_t SMEM = OFF_BAD + 512;
  // tensor memory: scores, two of 128 columns; accumulators, two of DHP; probabilities, two of 64: their own with DHP = 64, so that the next
  // scores are formed while these are worked out; over the scores they come from with DHP = 128
  static constexpr bool OWN_P = DHP == 64;
  static constexpr uint32_t COL_S = 0, COL_P = OWN_P ? 256 : 0, P_STEP = OWN_P ? 64 : 128, COL_O = 512 - 2 * DHP;
  static constexpr int REGS_LAUNCH = 168, REGS_CONTROL = 104, REGS_SOFTMAX = 200;
  static_assert(128 * REGS_CONTROL + 256 * REGS_SOFTMAX <= THREADS * REGS_LAUNCH, "register split");
  static_assert(SMEM <= 232448, "shared memory of one SM");
};
constexpr float kSeqRescale = 8.0f, kSeqBelow = 60.0f, kSeqAbove = 100.0f;        // log2 units
constexpr int kRowNowhere = 0x7fff0000;                            // a row past the end of every tensor map: reads as zeros

__device__ __forceinline__ float seq_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float seq_max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
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
  __device__ __forceinline__ SeqWork(const SeqParams& p, int work) {
    const int4* src = reinterpret_cast<const int4*>(p.items + work / p.Hkv);
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
  // the same as a range: first tile of slot s, end, step
  __device__ __forceinline__ int first(int s) const { return same ? it.t0 + s : s == 0 ? lo0 : it.t0; }
  __device__ __forceinline__ int end(int s) const { return same || s == 1 ? it.t1 : hi0; }
  __device__ __forceinline__ int first_token(int s) const { return same ? 0 : s * ts; }
  __device__ __forceinline__ int tokens(int s) const { return same ? it.rows : s == 0 ? ts : it.rows - ts; }
  // whether a row of the item does not see all keys of the tile
  __device__ __forceinline__ bool masked(const SeqTile& k) const { return k.kind == 2 || (k.kind == 0 ? k.j0 + 128 > it.c : k.j0 + 128 > k.n); }
  // whether the value tile is mended: see the top
  __device__ __forceinline__ bool mended(const SeqTile& k, bool again) const { return again ? masked(k) : TREE && k.kind == 1 && k.j0 + 128 > k.n; }
};

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

// The items of a CTA, one after the other; in the second pass the ones whose result was not finite (a bit each in `bad`).
struct SeqWalk {
  int k, work;                      // items seen; the current (item, head of keys), -1: the end
  __device__ __forceinline__ void next(const SeqParams& p, const uint32_t* bad, bool again) {
    const int n_work = p.plan->n_items * p.Hkv;
    for (;;) {
      const int64_t first = (int64_t)k * gridDim.x;
      if (first >= n_work) { work = -1; return; }
      work = (int)first + ((k & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x);
      const int bit = min(k, 4095);
      ++k;
      if (work < n_work && (!again || ((bad[bit >> 5] >> (bit & 31)) & 1u))) break;
    }
  }
  __device__ __forceinline__ SeqWalk(const SeqParams& p, const uint32_t* bad, bool again) : k(0) { next(p, bad, again); }
};

template <int DHP, bool TREE>
__global__ void __launch_bounds__(384, 1)
k_seq_attn_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ CUtensorMap tmCK, const __grid_constant__ CUtensorMap tmCV, const __grid_constant__ SeqParams p) {
  using namespace tc;
  using C = SeqTcCfg<DHP>;
  constexpr int STAGES = C::STAGES, QBUFS = C::QBUFS;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {                     // the swizzled tiles need a 1024-byte aligned base
    pdl_wait();
    if (threadIdx.x == 0) atomicCAS(p.err, 0, 110);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* kv_full = bars;            // [10] keys or values of a tile landed
  uint64_t* kv_empty = bars + 10;      // [10] every MMA that reads them has run
  uint64_t* mend_done = bars + 20;     // [10] the value tile in this stage is mended
  uint64_t* q_full = bars + 30;        // [2]  queries of an item landed
  uint64_t* q_empty = bars + 32;       // [2]  every score MMA that reads them has run
  uint64_t* s_full = bars + 34;        // [2]  scores of the slot in TMEM
  uint64_t* s_free = bars + 36;        // [2]  new scores may be formed: the last are in registers (four warps; OWN_P), or the values of the
                                       //      probabilities over them are issued, which the pipe then takes first
  uint64_t* p_ready = bars + 38;       // [2]  probabilities in TMEM (four warps)
  uint64_t* pv_done = bars + 40;       // [2]  the slot's accumulator is up to date
  uint64_t* o_free = bars + 42;        // [2]  the slot's accumulator is read out, by its own warps (every item)
  uint64_t* x_free = bars + 44;        // [2]  and by the other slot's (items whose slots are joined)
  uint64_t* p_half = bars + 48;        // [2]  the first half of them
  uint64_t* ml_full = bars + 46;       // [2]  the slot's references and sums are in shared memory (items whose slots are joined)
  int* s_flags = reinterpret_cast<int*>(bars + 50);         // 1: some result is not finite, 2: a wait gave up
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_flags + 1);
  float2* s_ml = reinterpret_cast<float2*>(smem + C::OFF_ML);
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(smem + C::OFF_BAD);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); mbar_init(&mend_done[i], 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); mbar_init(&s_full[i], 1); mbar_init(&s_free[i], C::OWN_P ? 4 : 1); mbar_init(&pv_done[i], 1);
      mbar_init(&p_ready[i], 4); mbar_init(&p_half[i], 4); mbar_init(&o_free[i], 4); mbar_init(&x_free[i], 4); mbar_init(&ml_full[i], 4);
    }
    *s_flags = 0;
    fence_barrier_init();
    prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    if (TREE) { prefetch_tmap(&tmCK); prefetch_tmap(&tmCV); }
  }
  if (threadIdx.x >= 128 && threadIdx.x < 256) s_bad[threadIdx.x - 128] = 0;
  if (warp == 1) { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  const int G = p.G;
  const int ksteps = (p.dh + 15) / 16;                      // of 16 features

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS_CONTROL));
    const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0);
    bool ok = true;
    int g = 0, qn = 0;                                       // tiles of keys and values so far (ring position); items with key tiles
    uint32_t ph0 = 0, ph1 = 0;                               // phases of the slots' barriers that this role waits for
    uint32_t mend_ph = 0;                                    // a bit for every stage
    bool prev = false, prev_same = false;                    // an item before this one, and its slots were joined
    uint32_t o_ph = 0, x_ph = 0;                             // phases in which that item's accumulators are read out
    for (int pass = 0; pass < 2; ++pass) {
      const bool again = pass > 0;
      for (SeqWalk at(p, s_bad, again); ok && at.work >= 0; at.next(p, s_bad, again)) {
        const int kvh = at.work % p.Hkv;
        const SeqWork<TREE> w(p, at.work);
        const bool any = w.it.t0 < w.it.t1;
        const int qb = qn % QBUFS;
        const uint32_t q_ph = (uint32_t)(qn / QBUFS) & 1u;
        if (any) ++qn;
        if (warp == 0) {
          // ---------------------------------------------------------------- loads
          if (any) {
            if (!__all_sync(0xffffffffu, mbar_wait(&q_empty[qb], q_ph ^ 1u, p.err, 123))) { ok = false; break; }
            if (lane == 0) {
              mbar_arrive_expect_tx(&q_full[qb], (w.same ? 1u : 2u) * (uint32_t)(w.ts * G) * 128u * (DHP / 64));
              for (int s = 0; s < (w.same ? 1 : 2); ++s)
                for (int c = 0; c < DHP / 64; ++c)
                  tma_load_3d(smem + C::OFF_Q + (qb * 2 + s) * C::TILE + c * C::SUB, &tmQ, c * 64, kvh * G, w.it.row0 + s * w.ts, &q_full[qb]);
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
          const uint64_t dq0 = make_sdesc_k_sw128(smem_u32(smem) + C::OFF_Q + qb * 2 * C::TILE), dk0 = make_sdesc_k_sw128(smem_u32(smem) + C::OFF_KV);
          if (any && !__all_sync(0xffffffffu, mbar_wait(&q_full[qb], q_ph, p.err, 112))) { ok = false; break; }
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
#pragma unroll
                for (int kk = 0; kk < DHP / 16; ++kk)
                  if (kk < ksteps)
                    mma_bf16_ss(tmem_u + C::COL_S + (uint32_t)s * 128, dq + (((kk >> 2) * C::SUB + (kk & 3) * 32) >> 4),
                                dk + (((kk >> 2) * C::SUB + (kk & 3) * 32) >> 4), idesc, kk != 0);
                mma_commit(&s_full[s]);
              }
              __syncwarp();
            }
            if (ok && elect_one()) {
              mma_commit(&kv_empty[st]);
              if (t + 1 == w.it.t1) mma_commit(&q_empty[qb]);
            }
            __syncwarp();
          }
        } else if (warp == 2) {
          // ---------------------------------------------------------------- values
          const uint32_t idesc = make_idesc_bf16(128, ksteps * 16, false, true);
          const uint64_t dv0 = make_sdesc_mn_sw128(smem_u32(smem) + C::OFF_KV, C::SUB);
          bool first0 = true, first1 = true;
          // the accumulator of slot s as the item before left it is read out
          auto taken = [&](int s) {
            return !prev || __all_sync(0xffffffffu, mbar_wait(&o_free[s], o_ph, p.err, 124) && (!prev_same || mbar_wait(&x_free[s], x_ph, p.err, 125)));
          };
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
              if (first && !taken(s)) { ok = false; break; }
              auto half = [&](int k0) {
#pragma unroll
                for (int kk = k0; kk < k0 + 4; ++kk)
                  mma_bf16_ts(tmem_u + C::COL_O + (uint32_t)(s * DHP), tmem_u + C::COL_P + (uint32_t)(s * C::P_STEP + kk * 8), dv + ((kk * 2048) >> 4), idesc,
                              kk != 0 || !first ? 1u : 0u);
              };
              if (!__all_sync(0xffffffffu, mbar_wait(&p_half[s], ph, p.err, 128))) { ok = false; break; }
              tc_fence_after();
              if (elect_one()) half(0);
              __syncwarp();
              if (!__all_sync(0xffffffffu, mbar_wait(&p_ready[s], ph, p.err, 117))) { ok = false; break; }
              ph ^= 1u;
              tc_fence_after();
              if (elect_one()) {
                half(4);
                mma_commit(&pv_done[s]);
                if (!C::OWN_P) {
                  tc_fence_before();
                  mbar_arrive(&s_free[s]);
                }
              }
              first = false;
              __syncwarp();
            }
            if (ok && elect_one()) mma_commit(&kv_empty[st]);
            __syncwarp();
          }
          // every phase of these barriers is waited for, so that none is taken for the one two before it
          if (ok && ((first0 && !taken(0)) || (first1 && !taken(1)))) ok = false;
          if (prev) { o_ph ^= 1u; if (prev_same) x_ph ^= 1u; }
          prev = true;
          prev_same = w.same;
        } else {
          // ---------------------------------------------------------------- value tiles that need mending
          // Every load is waited for, so that a stage's phase is never taken for the one two before it (without a cache nothing is mended
          // in the first pass, and all of its loads have landed before the second).
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            if (!TREE && !again) continue;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            const int st = (g + 1) % STAGES;
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[g % STAGES], (uint32_t)(g / STAGES) & 1u, p.err, 119) &&
                                             mbar_wait(&kv_full[st], (uint32_t)((g + 1) / STAGES) & 1u, p.err, 118))) { ok = false; break; }
            if (!w.mended(k, again)) continue;
            uint8_t* tile = smem + C::OFF_KV + st * C::TILE;
            const int n = k.n - k.j0;                        // rows of the tile that there are
            for (int i = lane; i < 128 * (DHP / 64) * 8; i += 32) {
              const int r = (i >> 3) & 127;
              if (r < n && !again) continue;
              uint4* piece = reinterpret_cast<uint4*>(tile + (i >> 10) * C::SUB + (i & 1023) * 16);
              uint4 x = make_uint4(0, 0, 0, 0);
              if (r < n) {
                x = *piece;
                uint32_t* u = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  if ((u[e] & 0x7f80u) == 0x7f80u) u[e] &= 0xffff0000u;
                  if ((u[e] & 0x7f800000u) == 0x7f800000u) u[e] &= 0xffffu;
                }
              }
              *piece = x;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&mend_done[st]);
          }
        }
      }
      if (!ok && lane == 0) atomicOr(s_flags, 2);
      __syncthreads();
      const int flags = *s_flags;
      if ((flags & 2) && warp == 0) {
        // giving up: let the copies already issued land (bounded) before this CTA's shared memory goes away
        for (int j = 0; j < g && j < STAGES; ++j) mbar_wait_quiet(&kv_full[(g - 1 - j) % STAGES], (uint32_t)((g - 1 - j) / STAGES) & 1u);
        for (int j = 0; j < qn && j < QBUFS; ++j) mbar_wait_quiet(&q_full[(qn - 1 - j) % QBUFS], (uint32_t)((qn - 1 - j) / QBUFS) & 1u);
      }
      if (flags != 1) break;
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS_SOFTMAX));
    // -------------------------------------------------------------------- softmax of a slot
    const int s = (warp - 4) >> 2, q = warp & 3;             // slot; TMEM lane quarter of this warp
    const int r = q * 32 + lane;                             // stacked row
    const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
    const uint32_t s_addr = lane_addr + C::COL_S + (uint32_t)s * 128, o_addr = lane_addr + C::COL_O + (uint32_t)(s * DHP);
    const uint32_t p_addr = lane_addr + C::COL_P + (uint32_t)s * C::P_STEP;
    const uint32_t other = lane_addr + C::COL_O + (uint32_t)((s ^ 1) * DHP);
    const float scale = p.scale_log2;
    // 4 x 4 transpose of 16-byte pieces inside each group of four lanes: lane 4j + i then holds piece i of rows 4j .. 4j + 3, so that
    // every store instruction writes whole 64-byte parts of rows
    auto xchg = [&](uint4& keep_lo, uint4& keep_hi, bool upper, int dist) {
      // lanes with `upper` clear give away keep_hi and receive into it; lanes with it set give away keep_lo
      uint4 send = upper ? keep_lo : keep_hi, recv;
      recv.x = __shfl_xor_sync(0xffffffffu, send.x, dist); recv.y = __shfl_xor_sync(0xffffffffu, send.y, dist);
      recv.z = __shfl_xor_sync(0xffffffffu, send.z, dist); recv.w = __shfl_xor_sync(0xffffffffu, send.w, dist);
      if (upper) keep_lo = recv; else keep_hi = recv;
    };
    auto transpose4 = [&](uint4 (&t)[4]) {
      xchg(t[0], t[1], (lane & 1) != 0, 1);
      xchg(t[2], t[3], (lane & 1) != 0, 1);
      xchg(t[0], t[2], (lane & 2) != 0, 2);
      xchg(t[1], t[3], (lane & 2) != 0, 2);
    };
    // scores with this maximum against reference m, or against 0 where there was none yet: 2^(score - m) leaves the range that bf16 and
    // fp32 sums are safe in
    auto too_far = [](float top, float m) { return m == -INFINITY ? top < -kSeqBelow || top > kSeqAbove : top > m + kSeqAbove; };
    bool ok = true;
    uint32_t s_ph = 0, pv_ph = 0, joined = 0;                // pv_ph: of the slot's next value contraction; joined: items with joined slots
    for (int pass = 0; pass < 2; ++pass) {
      for (SeqWalk at(p, s_bad, pass > 0); ok && at.work >= 0; at.next(p, s_bad, pass > 0)) {
        bool valid, any_valid, mine = false;                 // mine: the slot took a tile, its accumulator holds something
        // m: reference of the row (log2 domain) in use, m_next: from the next tile on, l: sum so far
        float m = -INFINITY, m_next = m, l = 0.f;
        bool far = false;
        // What the tile loop needs of the item, in few registers (a tile's scores take 128); the rest is read again behind it.
        int t, end, step, n_tree, vis, anc, first_row, first_top = 0;       // vis: keys (history) or cached rows (tree) that the row sees
        {
          const SeqWork<TREE> w(p, at.work);
          const int rows = w.tokens(s) * G, tok = w.first_token(s) + min(r, max(rows - 1, 0)) / G;
          valid = r < rows; any_valid = q * 32 < rows;
          t = w.first(s); end = w.end(s); step = w.same ? 2 : 1;
          n_tree = TREE ? w.n_tree : 0;
          vis = TREE ? w.it.b : w.it.c + tok;
          anc = w.it.c + tok;
          first_row = w.it.row0 - w.it.c;
          if (TREE) { const int top = ((w.it.c + w.it.rows + 127) >> 7) - 1; first_top = top; }
        }
        for (; t < end; t += step) {
          if (!__all_sync(0xffffffffu, mbar_wait(&s_full[s], s_ph, p.err, 120))) { ok = false; break; }
          s_ph ^= 1u;
          if (any_valid) {
            tc_fence_after();
            const bool new_rows = TREE && t < n_tree;
            const int n = vis - (t - n_tree) * 128;          // keys of the tile that the row sees
            bool masked = __any_sync(0xffffffffu, n < 128);
            uint32_t see[4] = {0u, 0u, 0u, 0u};
            if (new_rows) {
              const int j0 = (first_top - t) * 128;
              while (anc >= j0 + 128) anc = seq_parent(p, first_row, anc);
              while (anc >= j0) {
                const int b = anc - j0;
#pragma unroll
                for (int i = 0; i < 4; ++i) see[i] |= (b >> 5) == i ? 1u << (b & 31) : 0u;
                anc = seq_parent(p, first_row, anc);
              }
              __syncwarp();
            } else if (masked) {
#pragma unroll
              for (int i = 0; i < 4; ++i) { const int left = n - 32 * i; see[i] = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u; }
            }
            masked |= new_rows;
            auto mask32 = [&](float (&v)[32], uint32_t bits) {
              if (masked) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (((bits >> j) & 1u) == 0) v[j] = -INFINITY;
              }
            };
            auto most32 = [&](const float (&v)[32], float mx) {
              float a = v[0], b = v[1];
#pragma unroll
              for (int j = 2; j < 30; j += 4) { a = seq_max3(a, v[j], v[j + 2]); b = seq_max3(b, v[j + 1], v[j + 3]); }
              return seq_max3(fmaxf(mx, v[30]), fmaxf(a, v[31]), b);
            };
            if (pass > 0) {
              // The second time the maximum is known first.  It is taken where the reference would be too far off, and only there: whatever
              // the item is done again for, the other rows come out as they did.
              float mx = -INFINITY;
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                float v[32];
                tmem_ld_32x32(s_addr + 32 * c, v);
                tmem_wait_ld();
                mask32(v, see[c]);
                mx = most32(v, mx);
              }
              if (mx != -INFINITY && too_far(mx * scale, m_next)) m_next = mx * scale;
            }
            const bool raise = valid && m_next != m;
            if (mine && __any_sync(0xffffffffu, raise)) {
              if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 121))) { ok = false; break; }
              tc_fence_after();
              const float factor = raise && m != -INFINITY ? seq_ex2(m - m_next) : 1.f;
#pragma unroll 1
              for (int c = 0; c < DHP; c += 32) {
                float a[32];
                tmem_ld_32x32(o_addr + c, a);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 32; ++j) a[j] *= factor;
                tmem_st_32x32(o_addr + c, a);
              }
              l *= factor;
            }
            m = m_next;
            const float ref = m == -INFINITY ? 0.f : m;
            float mx = -INFINITY;
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
            const float2 sc2 = make_float2(scale, scale), rf2 = make_float2(-ref, -ref);
            // 32 keys of the tile: probabilities, their sum, the maximum
            auto chunk = [&](float (&x)[32], uint32_t bits, uint32_t to, bool first) {
              mask32(x, bits);
              float packed[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                float2 e = __ffma2_rn(make_float2(x[2 * j], x[2 * j + 1]), sc2, rf2);
                e = make_float2(seq_ex2(e.x), seq_ex2(e.y));
                if (j & 1) s1 = __fadd2_rn(s1, e); else s0 = __fadd2_rn(s0, e);
                packed[j] = __uint_as_float(seq_pack(e.x, e.y));
              }
              mx = most32(x, mx);
              if (C::OWN_P && first && mine) {               // the last probabilities are read
                ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 129));
                tc_fence_after();
              }
              tmem_st_32x16(to, packed);
            };
            // Rolled up: unrolled over the tile, the code of the roles does not stay in the instruction caches (twice the time).
            float x0[32], x1[32];
            tmem_ld_32x32(s_addr, x0);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              tmem_wait_ld();
              tmem_ld_32x32(s_addr + 64 * h + 32, x1);
              chunk(x0, h ? see[2] : see[0], p_addr + 32 * h, h == 0);
              tmem_wait_ld();
              if (h == 0) {
                tmem_ld_32x32(s_addr + 64, x0);
              } else if (C::OWN_P) {                         // all scores are in registers
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_free[s]);
                __syncwarp();                                // (the whole warp loads from and stores to tensor memory)
              }
              chunk(x1, h ? see[3] : see[1], p_addr + 32 * h + 16, false);
              if (h == 0) {
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_half[s]);
                __syncwarp();
              }
            }
            s0 = __fadd2_rn(s0, s1);
            l += s0.x + s0.y;
            // the reference of the next tile
            const float top = mx * scale;
            if (mx != -INFINITY) {
              far |= too_far(top, m);
              if (m == -INFINITY) {
                m = 0.f;
                m_next = fabsf(top) > kSeqRescale ? top : 0.f;
              } else {
                m_next = top > m + kSeqRescale ? top : m;
              }
            }
            tmem_wait_st();
            tc_fence_before();
          } else {
            // a warp without rows keeps step: with scores ahead of the probabilities it could else arrive for a tile too early
            if (lane == 0 && C::OWN_P) mbar_arrive(&s_free[s]);
            if (C::OWN_P && mine) ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 130));
            if (lane == 0) mbar_arrive(&p_half[s]);
          }
          if (!ok) break;
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_ready[s]);
          pv_ph ^= 1u;
          mine = true;
        }
        if (!ok) break;
        const SeqWork<TREE> w(p, at.work);
        const int kvh = at.work % p.Hkv, tok = w.first_token(s) + min(r, max(w.tokens(s) * G - 1, 0)) / G;
        if (mine && !__all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 122))) { ok = false; break; }
        // ------------------------------------------------------------------ result: the slot's rows, or of joined slots half the columns
        float w0 = 1.f, w1 = 0.f;                            // of this slot's accumulator and the other's
        const bool have0 = mine, have1 = w.same && w.it.t1 - w.it.t0 > (s ^ 1);
        if (w.same) {
          // (read for the joined item before this one: its value contractions were behind that, but this slot may have had no tile)
          if (joined > 0 && !__all_sync(0xffffffffu, mbar_wait(&x_free[s], (joined - 1) & 1u, p.err, 127))) { ok = false; break; }
          s_ml[s * 128 + r] = make_float2(m, mine ? l : 0.f);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ml_full[s]);
          if (!__all_sync(0xffffffffu, mbar_wait(&ml_full[s ^ 1], joined & 1u, p.err, 126))) { ok = false; break; }
          ++joined;
          const float2 o = s_ml[(s ^ 1) * 128 + r];
          const float mm = fmaxf(m, o.x), ref = mm == -INFINITY ? 0.f : mm;
          w0 = seq_ex2(m - ref); w1 = seq_ex2(o.x - ref);
          l = l * w0 + o.y * w1;
          m = mm;
        }
        tc_fence_after();
        if (any_valid) {
          const int c_lo = w.same ? s * (DHP / 2) : 0, c_hi = min(w.same ? c_lo + DHP / 2 : DHP, p.dh);
          const bool whole = w.it.part < 0;
          const int64_t part = (int64_t)w.it.part * p.Hkv + kvh;
          const int R = p.tok * G, pr = w.first_token(s) * G + r;
          if (!whole && valid && (s == 0 || !w.same)) {
            p.part_ml[part * 2 * R + pr] = m;
            p.part_ml[(part * 2 + 1) * R + pr] = l;
          }
          const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
          w0 *= inv; w1 *= inv;
          // where this row goes (element offset in the output, or in the partial results); -1: nowhere
          const int64_t to = !valid ? -1 : whole ? (int64_t)(w.it.row0 + tok) * p.out_stride + (kvh * G + r % G) * p.dh : (part * R + pr) * p.dh;
          int64_t to4[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) to4[i] = __shfl_sync(0xffffffffu, to, (lane & ~3) + i);
          float z = pass > 0 ? 0.f : far ? 1.f : l * 0.f;         // not 0: not finite, or too far from the reference
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
            if (pass > 0) {
              if (valid) seq_add_not_finite<TREE>(p, w, tok, kvh, w.same || s == 1 ? w.it.t0 : w.lo0, w.same || s == 1 ? w.it.t1 : w.hi0, c, a);
              __syncwarp();
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (c + (j & ~7) < p.dh) z = fmaf(a[j], 0.f, z);               // 0 * infinity and 0 * NaN
            }
            if (whole) {
              uint4 t4[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                t4[i] = make_uint4(seq_pack(a[8 * i], a[8 * i + 1]), seq_pack(a[8 * i + 2], a[8 * i + 3]), seq_pack(a[8 * i + 4], a[8 * i + 5]), seq_pack(a[8 * i + 6], a[8 * i + 7]));
              transpose4(t4);
              const int col = c + (lane & 3) * 8;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (to4[i] >= 0 && col < p.dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + to4[i] + col) = t4[i];
            } else {
#pragma unroll
              for (int h = 0; h < 32; h += 16) {
                uint4 t4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  t4[i] = make_uint4(__float_as_uint(a[h + 4 * i]), __float_as_uint(a[h + 4 * i + 1]), __float_as_uint(a[h + 4 * i + 2]), __float_as_uint(a[h + 4 * i + 3]));
                transpose4(t4);
                const int col = c + h + (lane & 3) * 4;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (to4[i] >= 0 && col < p.dh) *reinterpret_cast<uint4*>(p.part_acc + to4[i] + col) = t4[i];
              }
            }
          }
          if (__any_sync(0xffffffffu, valid && z != 0.f) && lane == 0) {
            const int bit = min(at.k - 1, 4095);
            atomicOr(&s_bad[bit >> 5], 1u << (bit & 31));
            atomicOr(s_flags, 1);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&o_free[s]);
          if (w.same) mbar_arrive(&x_free[s ^ 1]);
        }
      }
      if (!ok && lane == 0) atomicOr(s_flags, 2);
      __syncthreads();
      if (*s_flags != 1) break;
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

// Attention of the sequence path on the 5th-generation tensor cores for d_h of 72 .. 128 (bf16; k_seq_attn_d64_tc.cu has the narrower):
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
// and are joined in the end; so a few new rows stream their cache through two chains.
//  * Warp 0 loads (one lane a page where keys lie in pages), warp 1 issues the scores, warp 2 the values, warp 3 mends value tiles (below);
//    warps 4..7 and 8..11 are the softmax of a slot, one thread per row.  Online softmax with lazy rescale: the reference maximum is
//    raised only when exceeded by 2^8.
//  * Nothing waits for the end of an item but what needs it: the next one's keys and queries are loaded and its first scores formed while
//    the softmax warps write a result out (64 single events, 16..16384 keys: 244 -> 227 us; with a barrier of the CTA between items before).
//  * d_h under 128: TMA fills the columns that are not there with zeros in shared memory only, and the contractions stop at the next
//    multiple of 16.
//  * Probabilities are rounded to bf16 for the value product (the operands of one tcgen05.mma have one type); the row sum is taken of the
//    unrounded ones in fp32.
//  * Masked positions have p = 0, but 0 * NaN and 0 * infinity are NaN.  Value rows behind the end of a cached range, which may never have
//    been written, are zeroed in shared memory.  Elsewhere such values are the exception: an item whose result has a NaN or an infinity is
//    done again with what is not finite taken out of every tile that masks anything; the rows that do see it get it added at the end.
// What bounds it: 16384 causal rows of 16 heads of 128 over 4 heads of keys take 1.08 to 1.12 ms, 0.98 to 1.02 PFLOP/s at 950 to 1000 W, the
// power cap: 1825 active cycles of an SM for a tile of 128 x 128 (counted in a call alone: 1.03 ms at 1.58 GHz), of which its contractions
// fill 1024 of the tensor pipe (56 %) and its exponentials 1024 of the special-function unit (57 %).  A slot's chain (scores, maximum,
// exponentials, values) is longer than a tile's share of either, and with two slots the one fills the gaps of the other only in part.
// Measured and dropped: probabilities against the reference of the tiles before, without waiting for the maximum (1.15 ms); 64-key tiles
// with two score buffers a slot, which take the scores out of the chain (1.24 ms); two threads a row, 16 softmax warps (1.18 ms); the first
// half of the probabilities handed over early, polling without a pause (no change).
// A few rows stream their keys at 0.70 of the copy rate (64 users' 4 drafts over 16..16384 rows, 1.07 GB: 234 us).
#include "seq_tc.cuh"

namespace lime {

struct SeqTcCfg {
  static constexpr int DHP = 128, THREADS = 384, STAGES = 5;
  static constexpr uint32_t SUB = 128 * 128;                       // [128 rows x 64 features]
  static constexpr uint32_t TILE = (DHP / 64) * SUB;
  static constexpr uint32_t OFF_Q = 0, OFF_KV = 2 * TILE, OFF_BAR = OFF_KV + STAGES * TILE;
  static constexpr uint32_t OFF_ML = OFF_BAR + 512;               // references and sums of joined slots: [2 slots][128] pairs
  static constexpr uint32_t OFF_BAD = OFF_ML + 2 * 128 * 8;       // a bit for every item of the CTA
  static constexpr uint32_t SMEM = OFF_BAD + 512;
  static constexpr uint32_t COL_S = 0, COL_O = 256;                // scores: two of 128 columns; accumulators: two of DHP
  static constexpr int REGS_LAUNCH = 168, REGS_CONTROL = 56, REGS_SOFTMAX = 224;
  static_assert(128 * REGS_CONTROL + 256 * REGS_SOFTMAX <= THREADS * REGS_LAUNCH, "register split");
  static_assert(SMEM <= 232448 && COL_O + 2 * DHP <= 512, "budgets of one SM");
};
// An item as its warps see it: key tiles t0 .. t1 (the walk of seq_common.cuh), slot s takes those of [lo[s], hi[s]), or, where both
// slots hold the same rows (`same`), every other one.
template <bool TREE>
struct SeqWork {
  SeqItem it;
  int n_tree, ts;                 // tiles of new rows; tokens per slot
  bool same;
  int lo0, hi0;                   // slot 0 (slot 1 takes all of t0 .. t1)
  __device__ __forceinline__ SeqWork(const SeqParams& p, int work) {
    it = seq_item(p, work);
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
  __device__ __forceinline__ bool masked(const SeqTile& k) const { return seq_masked(it, k, 128); }
  // whether the value tile is mended: see the top
  __device__ __forceinline__ bool mended(const SeqTile& k, bool again) const { return again ? masked(k) : TREE && k.kind == 1 && k.j0 + 128 > k.n; }
};

template <bool TREE>
__global__ void __launch_bounds__(384, 1)
k_seq_attn_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
              const __grid_constant__ CUtensorMap tmCK, const __grid_constant__ CUtensorMap tmCV, const __grid_constant__ SeqParams p) {
  using namespace tc;
  using C = SeqTcCfg;
  constexpr int DHP = C::DHP, STAGES = C::STAGES;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {                     // the swizzled tiles need a 1024-byte aligned base
    pdl_wait();
    if (threadIdx.x == 0) atomicCAS(p.err, 0, 110);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* kv_full = bars;            // [5]  keys or values of a tile landed
  uint64_t* kv_empty = bars + 10;      // [5]  every MMA that reads them has run
  uint64_t* mend_ask = bars + 20;      //      the next value tile to be mended is on its way
  uint64_t* mend_done = bars + 21;     //      it is mended
  uint64_t* q_full = bars + 30;        //      queries of an item landed
  uint64_t* q_empty = bars + 32;       //      every score MMA that reads them has run
  uint64_t* s_full = bars + 34;        // [2]  scores of the slot in TMEM
  uint64_t* s_free = bars + 36;        // [2]  the values of the slot's last probabilities are issued: new scores may follow in the pipe
  uint64_t* p_ready = bars + 38;       // [2]  probabilities in TMEM (four warps)
  uint64_t* pv_done = bars + 40;       // [2]  the slot's accumulator is up to date
  // (of items that have key tiles; the first two of those in which the slot has one, so that none runs ahead of the values by two phases)
  uint64_t* o_free = bars + 42;        // [2]  the slot's accumulator is read out, by its own warps
  uint64_t* x_free = bars + 44;        // [2]  and by the other slot's (items whose slots are joined)
  uint64_t* ml_full = bars + 46;       // [2]  the slot's references and sums are in shared memory (items whose slots are joined)
  uint64_t* ml_free = bars + 48;       // [2]  and read by the other slot
  int* s_flags = reinterpret_cast<int*>(bars + 50);         // 1: some result is not finite, 2: a wait gave up
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_flags + 1);
  float2* s_ml = reinterpret_cast<float2*>(smem + C::OFF_ML);
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(smem + C::OFF_BAD);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
    mbar_init(mend_ask, 1); mbar_init(mend_done, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); mbar_init(&s_full[i], 1); mbar_init(&s_free[i], 1); mbar_init(&pv_done[i], 1);
      mbar_init(&p_ready[i], 4); mbar_init(&o_free[i], 4); mbar_init(&x_free[i], 4); mbar_init(&ml_full[i], 4); mbar_init(&ml_free[i], 4);
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
    uint32_t mend_ph = 0;
    // values: a bit for every slot whose accumulator an item before left to be read out, by its own warps and by the other slot's; phases
    uint32_t own_out = 0, cross_out = 0, o_ph = 0, x_ph = 0;
    for (int pass = 0; pass < 2; ++pass) {
      const bool again = pass > 0;
      for (SeqWalk at(p, s_bad, again); ok && at.work >= 0; at.next(p, s_bad, again)) {
        const int kvh = at.work % p.Hkv;
        const SeqWork<TREE> w(p, at.work);
        if (w.it.t0 >= w.it.t1) continue;                    // nothing to see: its rows are zeros, without any of this
        const uint32_t q_ph = (uint32_t)qn & 1u;
        ++qn;
        if (warp == 0) {
          // ---------------------------------------------------------------- loads
          if (!__all_sync(0xffffffffu, mbar_wait(q_empty, q_ph ^ 1u, p.err, 123))) { ok = false; break; }
          if (lane == 0) {
            mbar_arrive_expect_tx(q_full, (w.same ? 1u : 2u) * (uint32_t)(w.ts * G) * 128u * (DHP / 64));
            for (int s = 0; s < (w.same ? 1 : 2); ++s)
              for (int c = 0; c < DHP / 64; ++c)
                tma_load_3d(smem + C::OFF_Q + s * C::TILE + c * C::SUB, &tmQ, c * 64, kvh * G, w.it.row0 + s * w.ts, q_full);
          }
          __syncwarp();
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
          if (!__all_sync(0xffffffffu, mbar_wait(q_full, q_ph, p.err, 112))) { ok = false; break; }
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
                  const uint64_t at_k = (uint64_t)(((kk >> 2) * C::SUB + (kk & 3) * 32) >> 4);
                  mma_bf16_ss(tmem_u + C::COL_S + (uint32_t)s * 128, dq + at_k, dk + at_k, idesc, kk != 0);
                }
                mma_commit(&s_full[s]);
              }
              __syncwarp();
            }
            if (ok && elect_one()) {
              mma_commit(&kv_empty[st]);
              if (t + 1 == w.it.t1) mma_commit(q_empty);
            }
            __syncwarp();
          }
        } else if (warp == 2) {
          // ---------------------------------------------------------------- values
          const uint32_t idesc = make_idesc_bf16(128, ksteps * 16, false, true);
          const uint64_t dv0 = make_sdesc_mn_sw128(smem_u32(smem) + C::OFF_KV, C::SUB);
          bool first0 = true, first1 = true;
          // the accumulator of slot s as an item before left it is read out
          auto taken = [&](int s) {
            const uint32_t bit = 1u << s;
            const bool done = (!(own_out & bit) || mbar_wait(&o_free[s], (o_ph >> s) & 1u, p.err, 124)) &&
                              (!(cross_out & bit) || mbar_wait(&x_free[s], (x_ph >> s) & 1u, p.err, 125));
            o_ph ^= own_out & bit;
            x_ph ^= cross_out & bit;
            own_out |= bit;
            cross_out = w.same ? cross_out | bit : cross_out & ~bit;
            return __all_sync(0xffffffffu, done);
          };
          // a tile is asked for one ahead, when the stage's load before this one has landed and the mending before it is done
          auto ask = [&](int t) {
            if ((TREE || again) && t < w.it.t1 && w.mended(seq_tile<TREE>(p, w.it, w.n_tree, t), again) && lane == 0) mbar_arrive(mend_ask);
            __syncwarp();
          };
          ask(w.it.t0);
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            const int st = (g + 1) % STAGES;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[st], (uint32_t)((g + 1) / STAGES) & 1u, p.err, 115))) { ok = false; break; }
            if (w.mended(k, again)) {
              if (!__all_sync(0xffffffffu, mbar_wait(mend_done, mend_ph, p.err, 116))) { ok = false; break; }
              mend_ph ^= 1u;
            }
            ask(t + 1);
            const uint64_t dv = dv0 + (uint64_t)((uint32_t)st * C::TILE >> 4);
            for (int s = 0; s < 2; ++s) {
              if (!w.takes(s, t)) continue;
              uint32_t& ph = s == 0 ? ph0 : ph1;
              bool& first = s == 0 ? first0 : first1;
              if (first && !taken(s)) { ok = false; break; }
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
          // ---------------------------------------------------------------- value tiles that need mending
          // Asked for one at a time by the warp that will use it: the ring waits for that warp and not for this one, which could
          // otherwise fall a round behind and take a stage's phase for the one two before it.
          for (int t = w.it.t0; t < w.it.t1 && ok; ++t, g += 2) {
            if (!TREE && !again) continue;
            const SeqTile k = seq_tile<TREE>(p, w.it, w.n_tree, t);
            if (!w.mended(k, again)) continue;
            const int st = (g + 1) % STAGES;
            // The tiles and items before the next one to be mended may take seconds (histories that fill their tiles, then one that does not).
            // They are not this warp's to watch: what gets stuck is seen by a warp that waits for a step of it, and the error word ends this
            // wait too.
            if (!__all_sync(0xffffffffu, mbar_wait_limit(mend_ask, mend_ph, p.err, 119, 60 * kWaitLimitNs) &&
                                             mbar_wait(&kv_full[st], (uint32_t)((g + 1) / STAGES) & 1u, p.err, 118))) { ok = false; break; }
            mend_ph ^= 1u;
            uint8_t* tile = smem + C::OFF_KV + st * C::TILE;
            const int n = k.n - k.j0;                        // rows of the tile that there are
            for (int i = lane; i < 128 * (DHP / 64) * 8; i += 32) {
              const int r = (i >> 3) & 127;
              if (r < n && !again) continue;
              uint4* piece = reinterpret_cast<uint4*>(tile + (i >> 10) * C::SUB + (i & 1023) * 16);
              uint4 x = make_uint4(0, 0, 0, 0);
              if (r < n) {
                x = seq_finite8(*piece);
              }
              *piece = x;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(mend_done);
          }
        }
      }
      if (!ok && lane == 0) atomicOr(s_flags, 2);
      __syncthreads();
      const int flags = *s_flags;
      if ((flags & 2) && warp == 0) {
        // giving up: let the copies already issued land (bounded) before this CTA's shared memory goes away
        for (int j = 0; j < g && j < STAGES; ++j) mbar_wait_quiet(&kv_full[(g - 1 - j) % STAGES], (uint32_t)((g - 1 - j) / STAGES) & 1u);
        if (qn > 0) mbar_wait_quiet(q_full, (uint32_t)(qn - 1) & 1u);
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
    const uint32_t other = lane_addr + C::COL_O + (uint32_t)((s ^ 1) * DHP);
    const float scale = p.scale_log2;
    bool ok = true;
    uint32_t s_ph = 0, pv_ph = 0, joined = 0;                // pv_ph: of the slot's next value contraction; joined: items with joined slots
    for (int pass = 0; pass < 2; ++pass) {
      for (SeqWalk at(p, s_bad, pass > 0); ok && at.work >= 0; at.next(p, s_bad, pass > 0)) {
        bool valid, any_valid, mine = false;                 // mine: the slot took a tile, its accumulator holds something
        float m = -INFINITY, l = 0.f;
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
            float v[128];
#pragma unroll
            for (int c = 0; c < 128; c += 32) tmem_ld_32x32(s_addr + c, *reinterpret_cast<float(*)[32]>(&v[c]));
            tmem_wait_ld();
            if (TREE && t < n_tree) {
              const int j0 = (first_top - t) * 128;
              uint32_t see[4] = {0u, 0u, 0u, 0u};
              while (anc >= j0 + 128) anc = seq_parent(p, first_row, anc);
              while (anc >= j0) {
                const int b = anc - j0;
#pragma unroll
                for (int i = 0; i < 4; ++i) see[i] |= (b >> 5) == i ? 1u << (b & 31) : 0u;
                anc = seq_parent(p, first_row, anc);
              }
              __syncwarp();                                // (tensor memory is read and written by whole warps)
#pragma unroll
              for (int j = 0; j < 128; ++j)
                if (((see[j >> 5] >> (j & 31)) & 1u) == 0) v[j] = -INFINITY;
            } else {
              const int n = vis - (t - n_tree) * 128;                            // keys of the tile that the row sees
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
        if (!ok) break;
        const SeqWork<TREE> w(p, at.work);
        const int kvh = at.work % p.Hkv, tok = w.first_token(s) + min(r, max(w.tokens(s) * G - 1, 0)) / G;
        if (mine && !__all_sync(0xffffffffu, mbar_wait(&pv_done[s], pv_ph ^ 1u, p.err, 122))) { ok = false; break; }
        // ------------------------------------------------------------------ result: the slot's rows, or of joined slots half the columns
        float w0 = 1.f, w1 = 0.f;                            // of this slot's accumulator and the other's
        const bool have0 = mine, have1 = w.same && w.it.t1 - w.it.t0 > (s ^ 1);
        if (w.same && w.it.t0 < w.it.t1) {
          if (joined > 0 && !__all_sync(0xffffffffu, mbar_wait(&ml_free[s], (joined - 1) & 1u, p.err, 127))) { ok = false; break; }
          s_ml[s * 128 + r] = make_float2(m, mine ? l : 0.f);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ml_full[s]);
          if (!__all_sync(0xffffffffu, mbar_wait(&ml_full[s ^ 1], joined & 1u, p.err, 126))) { ok = false; break; }
          ++joined;
          const float2 o = s_ml[(s ^ 1) * 128 + r];
          __syncwarp();
          if (lane == 0) mbar_arrive(&ml_free[s ^ 1]);
          const float mm = fmaxf(m, o.x), ref = mm == -INFINITY ? 0.f : mm;
          w0 = seq_ex2((m - ref) * scale); w1 = seq_ex2((o.x - ref) * scale);
          l = l * w0 + o.y * w1;
          m = mm;
        }
        tc_fence_after();
        if (any_valid) {
          const int c_lo = w.same ? s * (DHP / 2) : 0, c_hi = min(w.same ? c_lo + DHP / 2 : DHP, p.dh);
          const bool whole = w.it.part < 0;
          const int64_t part = (int64_t)w.it.part * p.Hkv + kvh;
          const int R = p.part_rows, pr = w.first_token(s) * G + r;
          if (!whole && valid && (s == 0 || !w.same)) {
            p.part_ml[part * 2 * R + pr] = m == -INFINITY ? m : m * scale;
            p.part_ml[(part * 2 + 1) * R + pr] = l;
          }
          const float inv = !whole ? 1.f : seq_inverse(l, TREE ? w.it.b > 0 || p.k != nullptr : w.it.c + tok > 0);
          w0 *= inv; w1 *= inv;
          // where this row goes (element offset in the output, or in the partial results); -1: nowhere
          const int64_t to = !valid ? -1 : whole ? (int64_t)(w.it.row0 + tok) * p.out_stride + (kvh * G + r % G) * p.dh : (part * R + pr) * p.dh;
          float z = 0.f;
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
              if (valid) seq_add_not_finite<TREE>(p, at.work, tok, w.same ? w.it.t0 : w.first(s), w.end(s), c, a);
              __syncwarp();
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (c + (j & ~7) < p.dh) z = fmaf(a[j], 0.f, z);               // 0 * infinity and 0 * NaN
            }
            seq_store32(p, whole, a, to, c, lane);
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
          if (have0) mbar_arrive(&o_free[s]);
          if (have1) mbar_arrive(&x_free[s ^ 1]);
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

template <bool TREE>
static lime_status launch_tc(const SeqParams& p, cudaStream_t st) {
  using C = SeqTcCfg;
  static bool set[kMaxDeviceOrdinals] = {};
  SeqMaps m;
  if (!seq_make_maps(m, p, TREE, p.tok / 2, 128)) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  const lime_status s = ensure_dynamic_smem((const void*)k_seq_attn_tc<TREE>, (int)C::SMEM, set);
  if (s != LIME_OK) return s;
  const int64_t work = (int64_t)p.items_upper * p.Hkv;
  ProfScope _p("k_seq_attn_tc", st);
  launch_pdl(k_seq_attn_tc<TREE>, dim3((unsigned)(work < kSMs ? work : kSMs)), dim3(C::THREADS), C::SMEM, st, m.q, m.k, m.v, m.ck, m.cv, p);
  LIME_LAUNCH_CHECK("k_seq_attn_tc");
  return LIME_OK;
}

lime_status launch_seq_attn_tc(const SeqParams& p, bool tree, cudaStream_t st) {
  return tree ? launch_tc<true>(p, st) : launch_tc<false>(p, st);
}

}  // namespace lime

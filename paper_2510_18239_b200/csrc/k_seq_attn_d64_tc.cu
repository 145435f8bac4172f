// Attention of the sequence path on the 5th-generation tensor cores for d_h <= 64 (bf16):
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(scale log2(e) (<q_i, k_j> - m_i))   over the keys j that row i sees
//
// With so few features a tile is little work for the tensor cores and a long chain of latencies - scores, TMEM loads, maximum,
// exponentials, probabilities, values.  So two independent CTAs share an SM, each with a chain of its own: 128 stacked rows (tokens x the
// query heads of one head of keys) against key tiles of 64,
//   scores [128 x 64] = Q [128 x d_h] . K_tile^T       O [128 x d_h] += P [128 x 64] . V_tile
// in 128 columns of tensor memory and six warps: 0 loads (one lane a page where keys lie in pages), 1 issues both products, 2..5 are the
// softmax, one thread per row.  The CTAs are persistent and walk the work items of k_seq_schedule back and forth.
// d_h <= 32 leaves columns for the probabilities, so that the next scores are formed while these are worked out.
// What bounds it: the hand-overs between the warps, tile by tile.  With loads and contractions issued by one warp and three CTAs an SM,
// candidate roots (32 users of 1000 behind 1024 rows, 8 heads of 32) took 189 us; without their exponentials and contractions still 178; with nothing
// left but the hand-overs 130.  The exponentials alone would take about 70.  As it stands they take 161 and 100 ragged users of 0..1000
// rows 62, with the special-function unit at 0.49 and 0.39 and the tensor pipe at 0.12 and 0.10.  More CTAs an SM do not help (beside 172 and
// 65 with two): four with 80 registers a thread, the scores loaded twice, 180 and 63..67; three as above 189 and 69; both slots of
// k_seq_attn_tc.cu in one CTA 172 and 72.
// The rest is as in k_seq_attn_tc.cu: online softmax with lazy rescale, probabilities rounded to bf16 for the value product and summed
// unrounded, features past d_h as zeros in shared memory only, value rows behind the end of a cached range zeroed there, items whose
// result is not finite done again with what is not finite taken out of the tiles that mask anything.
#include "seq_tc.cuh"

namespace lime {

constexpr int kD64Keys = 64, kD64Stages = 8, kD64Ctas = 2;
constexpr uint32_t kD64Tile = kD64Keys * 128, kD64OffKv = 128 * 128, kD64OffBar = kD64OffKv + kD64Stages * kD64Tile, kD64OffBad = kD64OffBar + 256,
                   kD64Smem = kD64OffBad + 512;

// OWN_P (d_h <= 32): the probabilities have columns of their own, so that the next scores are formed while these are worked out
template <bool TREE, bool OWN_P>
__global__ void __launch_bounds__(192, kD64Ctas)
k_seq_attn_d64_tc(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ CUtensorMap tmCK, const __grid_constant__ CUtensorMap tmCV, const __grid_constant__ SeqParams p) {
  using namespace tc;
  constexpr int KEYS = kD64Keys, STAGES = kD64Stages;
  extern __shared__ __align__(1024) uint8_t smem[];
  if ((smem_u32(smem) & 1023u) != 0) {                     // the swizzled tiles need a 1024-byte aligned base
    pdl_wait();
    if (threadIdx.x == 0) atomicCAS(p.err, 0, 140);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kD64OffBar);
  uint64_t* kv_full = bars;            // [8] keys or values of a tile landed
  uint64_t* kv_empty = bars + 8;       // [8] every MMA that reads them has run
  uint64_t* q_full = bars + 16;        //     queries of an item landed
  uint64_t* q_empty = bars + 17;       //     every score MMA that reads them has run
  uint64_t* s_full = bars + 18;        //     scores in TMEM
  uint64_t* p_ready = bars + 19;       //     probabilities in TMEM (four warps)
  uint64_t* pv_done = bars + 20;       //     their values are in the accumulator
  uint64_t* o_free = bars + 21;        //     the accumulator of an item with key tiles is read out (four warps)
  uint64_t* s_free = bars + 22;        //     the scores of a tile are in registers (four warps; OWN_P)
  int* s_flags = reinterpret_cast<int*>(bars + 23);         // 1: some result is not finite, 2: a wait gave up
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_flags + 1);
  uint32_t* s_bad = reinterpret_cast<uint32_t*>(smem + kD64OffBad);   // a bit for every item of the CTA

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
    mbar_init(q_full, 1); mbar_init(q_empty, 1); mbar_init(s_full, 1); mbar_init(pv_done, 1);
    mbar_init(p_ready, 4); mbar_init(o_free, 4); mbar_init(s_free, 4);
    *s_flags = 0;
    fence_barrier_init();
    prefetch_tmap(&tmQ); prefetch_tmap(&tmK); prefetch_tmap(&tmV);
    if (TREE) { prefetch_tmap(&tmCK); prefetch_tmap(&tmCV); }
  }
  if (threadIdx.x >= 64) s_bad[threadIdx.x - 64] = 0;
  if (warp == 1) { tmem_alloc(tmem_slot, 128); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  const int G = p.G, ksteps = (p.dh + 15) / 16;             // of 16 features
  constexpr uint32_t COL_P = OWN_P ? 64 : 0, COL_O = OWN_P ? 96 : 64;          // scores: columns 0..63
  // Every role has its own loop over the items (twice: see the second pass), so that none keeps registers for another's state.
  auto end_of_pass = [&](bool ok) {
    if (!ok && lane == 0) atomicOr(s_flags, 2);
    __syncthreads();
    return *s_flags;
  };
  if (warp == 0) {
    bool ok = true;
    int g = 0, qn = 0;                                       // loads of keys and values so far (ring position); items with key tiles
    for (int pass = 0; pass < 2; ++pass) {
      for (SeqWalk at(p, s_bad, pass > 0); ok && at.work >= 0; at.next(p, s_bad, pass > 0)) {
        const SeqItem it = seq_item(p, at.work);
        const int kvh = at.work % p.Hkv, n_tree = TREE ? seq_tree_tiles(p, it) : 0;
        if (it.t0 >= it.t1) continue;                        // nothing to see: its rows are zeros, without any of this
        // ------------------------------------------------------------------ loads
        if (!__all_sync(0xffffffffu, mbar_wait(q_empty, ((uint32_t)qn & 1u) ^ 1u, p.err, 141))) { ok = false; break; }
        if (lane == 0) {
          mbar_arrive_expect_tx(q_full, (uint32_t)(p.tok * G) * 128u);
          tma_load_3d(smem, &tmQ, 0, kvh * G, it.row0, q_full);
        }
        __syncwarp();
        ++qn;
        const int box = min(p.page_rows, KEYS);              // rows of a page in one copy
        int row = 0;                                         // of the lane's page of the coming tile of cached rows
        auto look_up = [&](int t) {
          if (!TREE || t >= it.t1) return;
          const SeqTile k = seq_tile<TREE>(p, it, n_tree, t);
          const int j = k.j0 + lane * box;
          if (k.kind != 1 || lane * box >= KEYS || j >= k.n) return;
          const int64_t pg = seq_page(p, it.a, j);
          row = pg < p.n_pages ? (int)(pg * p.page_rows + (j & (p.page_rows - 1))) : kRowNowhere;
        };
        look_up(it.t0);
        for (int t = it.t0; t < it.t1 && ok; ++t) {
          const SeqTile k = seq_tile<TREE>(p, it, n_tree, t);
          const int my_row = row;
          look_up(t + 1);
          for (int kv = 0; kv < 2; ++kv, ++g) {
            const int s = g % STAGES;
            if (!__all_sync(0xffffffffu, mbar_wait(&kv_empty[s], ((uint32_t)(g / STAGES) & 1u) ^ 1u, p.err, 142))) { ok = false; break; }
            uint8_t* dst = smem + kD64OffKv + s * kD64Tile;
            if (TREE && k.kind == 1) {
              const int n_box = min(KEYS / box, (k.n - k.j0 + box - 1) / box);
              if (lane == 0) mbar_arrive_expect_tx(&kv_full[s], (uint32_t)(n_box * box) * 128u);
              __syncwarp();
              if (lane < n_box) tma_load_3d(dst + lane * box * 128, kv ? &tmCV : &tmCK, 0, kvh, my_row, &kv_full[s]);
            } else if (lane == 0) {
              mbar_arrive_expect_tx(&kv_full[s], kD64Tile);
              tma_load_3d(dst, kv ? &tmV : &tmK, 0, kvh, (TREE ? it.row0 - it.c : it.a) + k.j0, &kv_full[s]);
            }
            __syncwarp();
          }
        }
      }
      const int flags = end_of_pass(ok);
      if (flags & 2) {
        // giving up: let the copies already issued land (bounded) before this CTA's shared memory goes away
        for (int j = 0; j < g && j < STAGES; ++j) mbar_wait_quiet(&kv_full[(g - 1 - j) % STAGES], (uint32_t)((g - 1 - j) / STAGES) & 1u);
        if (qn > 0) mbar_wait_quiet(q_full, (uint32_t)(qn - 1) & 1u);
      }
      if (flags != 1) break;
    }
  } else if (warp == 1) {
    bool ok = true;
    int g = 0, qn = 0;
    uint32_t n = 0, done = 0;                                // tiles so far; items with tiles so far
    for (int pass = 0; pass < 2; ++pass) {
      const bool again = pass > 0;
      for (SeqWalk at(p, s_bad, again); ok && at.work >= 0; at.next(p, s_bad, again)) {
        const SeqItem it = seq_item(p, at.work);
        const int n_tree = TREE ? seq_tree_tiles(p, it) : 0;
        if (it.t0 >= it.t1) continue;
        // ------------------------------------------------------------------ both products: values of a tile, then scores of the next
        const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0), idesc_s = make_idesc_bf16(128, KEYS), idesc_o = make_idesc_bf16(128, ksteps * 16, false, true);
        const uint64_t dq = make_sdesc_k_sw128(smem_u32(smem)), dk0 = make_sdesc_k_sw128(smem_u32(smem) + kD64OffKv), dv0 = make_sdesc_mn_sw128(smem_u32(smem) + kD64OffKv, kD64Tile);
        // loads come as keys 0, values 0, keys 1, ..: tile t's keys are load `k0 + 2 (t - t0)`
        const int k0 = g;
        auto scores = [&](int t) {
          const int at_load = k0 + 2 * (t - it.t0), s = at_load % STAGES;
          const bool last = t + 1 == it.t1;
          if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[s], (uint32_t)(at_load / STAGES) & 1u, p.err, 143))) return false;
          tc_fence_after();
          const uint64_t dk = dk0 + (uint64_t)((uint32_t)s * kD64Tile >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              if (kk < ksteps) mma_bf16_ss(tmem_u, dq + ((kk * 32) >> 4), dk + ((kk * 32) >> 4), idesc_s, kk != 0);
            mma_commit(s_full);
            mma_commit(&kv_empty[s]);
            if (last) mma_commit(q_empty);
          }
          __syncwarp();
          return true;
        };
        // the accumulator as the item before left it is read out
        auto taken = [&] { return done == 0 || __all_sync(0xffffffffu, mbar_wait(o_free, (done - 1) & 1u, p.err, 146)); };
        if (!__all_sync(0xffffffffu, mbar_wait(q_full, (uint32_t)qn & 1u, p.err, 144))) { ok = false; break; }
        ++qn;
        if (!scores(it.t0)) { ok = false; break; }
        for (int t = it.t0; t < it.t1; ++t, ++n) {
          if (OWN_P && !(__all_sync(0xffffffffu, mbar_wait(s_free, n & 1u, p.err, 151)) && (t + 1 >= it.t1 || scores(t + 1)))) { ok = false; break; }
          g = k0 + 2 * (t - it.t0) + 1;                      // its values
          const int s = g % STAGES;
          const SeqTile k = seq_tile<TREE>(p, it, n_tree, t);
          if (!__all_sync(0xffffffffu, mbar_wait(&kv_full[s], (uint32_t)(g / STAGES) & 1u, p.err, 145))) { ok = false; break; }
          if (again ? seq_masked(it, k, KEYS) : TREE && k.kind == 1 && k.j0 + KEYS > k.n) {
            uint8_t* tile = smem + kD64OffKv + s * kD64Tile;
            for (int i = lane; i < KEYS * 8; i += 32) {
              uint4* piece = reinterpret_cast<uint4*>(tile + i * 16);
              if ((i >> 3) >= k.n - k.j0) *piece = make_uint4(0, 0, 0, 0);
              else if (again) *piece = seq_finite8(*piece);
            }
            fence_proxy_async_smem();
            __syncwarp();
          }
          if (t == it.t0 && !taken()) { ok = false; break; }
          if (!__all_sync(0xffffffffu, mbar_wait(p_ready, n & 1u, p.err, 147))) { ok = false; break; }
          tc_fence_after();
          const uint64_t dv = dv0 + (uint64_t)((uint32_t)s * kD64Tile >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < KEYS / 16; ++kk)
              mma_bf16_ts(tmem_u + COL_O, tmem_u + COL_P + (uint32_t)(kk * 8), dv + ((kk * 2048) >> 4), idesc_o, kk != 0 || t != it.t0 ? 1u : 0u);
            mma_commit(pv_done);
            mma_commit(&kv_empty[s]);
          }
          __syncwarp();
          if (!OWN_P && t + 1 < it.t1 && !scores(t + 1)) { ok = false; break; }
        }
        ++g;
        ++done;
      }
      if (end_of_pass(ok) != 1) break;
    }
  } else {
    const int q = warp & 3, r = q * 32 + lane;               // TMEM lane quarter; stacked row
    const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
    const float scale = p.scale_log2;
    bool ok = true;
    uint32_t n = 0;                                          // tiles so far
    for (int pass = 0; pass < 2; ++pass) {
      const bool again = pass > 0;
      for (SeqWalk at(p, s_bad, again); ok && at.work >= 0; at.next(p, s_bad, again)) {
        // ------------------------------------------------------------------ softmax
        // What the tile loop needs of the item, in few registers; the rest is read again behind it.
        int t, end, n_tree, vis, anc, first_row, top_tile;   // vis: keys (history) or cached rows (tree) that the row sees
        bool valid, any_valid;
        {
          const SeqItem it = p.items[at.work / p.Hkv];
          const int rows = it.rows * G, tok = min(r, rows - 1) / G;
          valid = r < rows; any_valid = q * 32 < rows;
          t = it.t0; end = it.t1;
          n_tree = TREE ? seq_tree_tiles(p, it) : 0;
          vis = TREE ? it.b : it.c + tok;
          anc = it.c + tok;
          first_row = it.row0 - it.c;
          top_tile = TREE ? (it.c + it.rows + KEYS - 1) / KEYS - 1 : 0;
        }
        bool first = true;
        float m = -INFINITY, l = 0.f;                        // reference maximum (scores as they are), sum
        for (; t < end; ++t, ++n, first = false) {
          if (!__all_sync(0xffffffffu, mbar_wait(s_full, n & 1u, p.err, 148))) { ok = false; break; }
          // the values of the tile before are in the accumulator: its probabilities may be overwritten (every tile is waited for, so that no
          // phase is missed; without OWN_P they were ahead of these scores in the pipe)
          auto before = [&] { return first || __all_sync(0xffffffffu, mbar_wait(pv_done, (n & 1u) ^ 1u, p.err, 149)); };
          if (!any_valid) {
            if (OWN_P && lane == 0) mbar_arrive(s_free);
            if (!before()) { ok = false; break; }
          } else {
            tc_fence_after();
            // keys that the row sees, a bit each
            uint32_t see0 = 0xffffffffu, see1 = 0xffffffffu;
            bool masked = TREE && t < n_tree;
            if (masked) {
              const int j0 = (top_tile - t) * KEYS;
              see0 = see1 = 0u;
              while (anc >= j0 + KEYS) anc = seq_parent(p, first_row, anc);
              while (anc >= j0) {
                const int b = anc - j0;
                if (b < 32) see0 |= 1u << b; else see1 |= 1u << (b - 32);
                anc = seq_parent(p, first_row, anc);
              }
              __syncwarp();
            } else {
              const int left = vis - (t - n_tree) * KEYS;
              masked = __any_sync(0xffffffffu, left < KEYS);
              if (left < KEYS) {
                see0 = left >= 32 ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u;
                see1 = left > 32 ? (1u << (left - 32)) - 1u : 0u;
              }
            }
            float v[64];
            tmem_ld_32x32(lane_addr, *reinterpret_cast<float(*)[32]>(&v[0]));
            tmem_ld_32x32(lane_addr + 32, *reinterpret_cast<float(*)[32]>(&v[32]));
            tmem_wait_ld();
            if (OWN_P) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(s_free);
              __syncwarp();                                  // (the whole warp loads from and stores to tensor memory)
            }
            if (masked) {
#pragma unroll
              for (int j = 0; j < 64; ++j)
                if ((((j < 32 ? see0 : see1) >> (j & 31)) & 1u) == 0) v[j] = -INFINITY;
            }
            float mx0 = v[0], mx1 = v[1], mx2 = v[2], mx3 = v[3];
#pragma unroll
            for (int j = 4; j < 60; j += 8) {
              mx0 = seq_max3(mx0, v[j], v[j + 4]); mx1 = seq_max3(mx1, v[j + 1], v[j + 5]);
              mx2 = seq_max3(mx2, v[j + 2], v[j + 6]); mx3 = seq_max3(mx3, v[j + 3], v[j + 7]);
            }
            const float mx = seq_max3(seq_max3(mx0, mx1, v[60]), seq_max3(mx2, mx3, v[61]), fmaxf(v[62], v[63]));
            if (!before()) { ok = false; break; }
            tc_fence_after();
            // raise the reference only when it is exceeded by more than the threshold, or unset
            const bool need = valid && (mx - m) * scale > kSeqRescale;
            const float m_new = need ? mx : m;
            if (!first && __any_sync(0xffffffffu, need)) {
              const float factor = need && m != -INFINITY ? seq_ex2((m - m_new) * scale) : 1.f;
#pragma unroll 1
              for (int c = 0; c < ksteps * 16; c += 16) {
                float a[16];
                tmem_ld_32x16(lane_addr + COL_O + c, a);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) a[j] *= factor;
                tmem_st_32x16(lane_addr + COL_O + c, a);
              }
              l *= factor;
            }
            m = m_new;
            const float ref = m == -INFINITY ? 0.f : m * scale;
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
            const float2 sc2 = make_float2(scale, scale), rf2 = make_float2(-ref, -ref);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float packed[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                float2 e = __ffma2_rn(make_float2(v[16 * c + 2 * j], v[16 * c + 2 * j + 1]), sc2, rf2);
                e = make_float2(seq_ex2(e.x), seq_ex2(e.y));
                if (j & 1) s1 = __fadd2_rn(s1, e); else s0 = __fadd2_rn(s0, e);
                packed[j] = __uint_as_float(seq_pack(e.x, e.y));
              }
              tmem_st_32x8(lane_addr + COL_P + 8 * c, packed);             // (without OWN_P over scores that have been read)
            }
            s0 = __fadd2_rn(s0, s1);
            l += s0.x + s0.y;
            tmem_wait_st();
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(p_ready);
        }
        const SeqItem it = p.items[at.work / p.Hkv];
        const bool any = it.t0 < it.t1;
        if (!ok || (any && !__all_sync(0xffffffffu, mbar_wait(pv_done, (n & 1u) ^ 1u, p.err, 150)))) { ok = false; break; }
        tc_fence_after();
        if (any_valid) {
          const bool whole = it.part < 0;
          const int R = p.part_rows, kvh = at.work % p.Hkv, tok = min(r, it.rows * G - 1) / G;
          const int64_t piece = (int64_t)it.part * p.Hkv + kvh;
          if (!whole && valid) {
            p.part_ml[piece * 2 * R + r] = m == -INFINITY ? m : m * scale;
            p.part_ml[(piece * 2 + 1) * R + r] = l;
          }
          const float inv = !whole ? 1.f : seq_inverse(l, TREE ? it.b > 0 || p.k != nullptr : it.c + tok > 0);
          const int64_t to = !valid ? -1 : whole ? (int64_t)(it.row0 + tok) * p.out_stride + (kvh * G + r % G) * p.dh : (piece * R + r) * p.dh;
          float z = 0.f;
#pragma unroll 1
          for (int c = 0; c < p.dh; c += 32) {
            float a[32];
            if (any) {
              tmem_ld_32x32(lane_addr + COL_O + c, a);
              tmem_wait_ld();
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) a[j] = any ? a[j] * inv : 0.f;
            if (again) {
              if (valid) seq_add_not_finite<TREE>(p, at.work, tok, it.t0, it.t1, c, a);
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
        if (any && lane == 0) mbar_arrive(o_free);
      }
      if (end_of_pass(ok) != 1) break;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 128);
  }
}

template <bool TREE, bool OWN_P>
static lime_status launch_d64(const SeqParams& p, cudaStream_t st) {
  static bool set[kMaxDeviceOrdinals] = {};
  SeqMaps m;
  if (!seq_make_maps(m, p, TREE, p.tok, kD64Keys)) return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  const lime_status s = ensure_dynamic_smem((const void*)k_seq_attn_d64_tc<TREE, OWN_P>, (int)kD64Smem, set);
  if (s != LIME_OK) return s;
  const int64_t work = (int64_t)p.items_upper * p.Hkv;
  ProfScope _p("k_seq_attn_d64_tc", st);
  launch_pdl(k_seq_attn_d64_tc<TREE, OWN_P>, dim3((unsigned)(work < kD64Ctas * kSMs ? work : kD64Ctas * kSMs)), dim3(192), kD64Smem, st, m.q, m.k, m.v, m.ck, m.cv, p);
  LIME_LAUNCH_CHECK("k_seq_attn_d64_tc");
  return LIME_OK;
}

lime_status launch_seq_attn_d64_tc(const SeqParams& p, bool tree, cudaStream_t st) {
  if (p.dh <= 32) return tree ? launch_d64<true, true>(p, st) : launch_d64<false, true>(p, st);
  return tree ? launch_d64<true, false>(p, st) : launch_d64<false, false>(p, st);
}

}  // namespace lime

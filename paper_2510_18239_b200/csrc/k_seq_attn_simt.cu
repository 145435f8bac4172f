// Attention of the sequence path on CUDA cores (fp32):
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(scale log2(e) <q_i, k_j> - m_i)   over the keys j that row i sees
//
// One block of 256 threads per work item (seq_common.cuh) and head of keys: RT stacked query rows against tiles of 64 keys, all in fp32
// (FFMA), running maximum and sum per row, one pass over keys and values.  Threads are 16 x 16: thread (ty, tx) forms the scores of rows
// ty, ty + 16, .. with keys tx, tx + 16, .., and owns 16 / VW-wide column groups of the same rows' results, so maxima and sums stay
// within half a warp and the probabilities pass through shared memory without a block barrier.  The next tile's keys and values are
// copied (cp.async) while a tile is worked on.
// A masked position is -1 among the probabilities of a tile that has one: its value row is then not touched at all, so that infinities
// and NaN there stay there.
// What bounds it: with many items FFMA and the shared-memory reads that feed it (64 histories of 512 rows, 8 heads of 64: 0.60 ms,
// 29 of 74 TFLOP/s); with few the chain of a tile, about 5 us for a block that has an SM to itself, so two blocks share one where they fit (drafts
// of 7 users 91 -> 74 us with pairs of products and predicates for what is masked; the FMA pipe is then busy in 0.47 of the cycles, the
// paths to shared memory in 0.51).
#include <type_traits>

#include "seq_common.cuh"
#include "tc_common.cuh"

namespace lime {

constexpr int kSimtKeys = 64;

template <int DHP, int RT>
struct SimtCfg {
  static constexpr int LD = DHP + 4, PLD = kSimtKeys + 4;
  static constexpr int VW = DHP >= 64 ? 4 : 2, DC = DHP / (16 * VW), RI = RT / 16;
  static constexpr int OFF_K = RT * LD, OFF_V = OFF_K + 2 * kSimtKeys * LD, OFF_P = OFF_V + 2 * kSimtKeys * LD;
  static constexpr int OFF_MASK = OFF_P + RT * PLD;                               // [2 tile parities][RT] of two words
  static constexpr int SMEM = (OFF_MASK + 4 * RT) * 4;
  static_assert(SMEM <= 232448, "shared memory of one block");
};

__device__ __forceinline__ void cp_async16(void* dst, const void* src, bool there) {
  const int n = there ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(dst)), "l"(src), "r"(n) : "memory");
}
// a += p * v unless p < 0 (NaN is not): a predicate instead of a branch, of which a masked tile would have one per (row, key)
__device__ __forceinline__ void fma2_unless_negative(float2& a, float2 p, float2 v) {
  uint64_t r = *reinterpret_cast<uint64_t*>(&a);
  asm("{\n\t.reg .pred q;\n\tsetp.geu.f32 q, %1, 0f00000000;\n\t@q fma.rn.f32x2 %0, %2, %3, %0;\n\t}\n"
      : "+l"(r) : "f"(p.x), "l"(*reinterpret_cast<uint64_t*>(&p)), "l"(*reinterpret_cast<uint64_t*>(&v)));
  a = *reinterpret_cast<float2*>(&r);
}

template <int DHP, int RT, bool TREE>
__global__ void __launch_bounds__(256, DHP <= 64 ? 2 : 1) k_seq_attn_simt(const SeqParams p) {
  using C = SimtCfg<DHP, RT>;
  constexpr int LD = C::LD, PLD = C::PLD, KT = kSimtKeys, VW = C::VW, DC = C::DC, RI = C::RI;
  extern __shared__ __align__(16) float sm[];
  float* sQ = sm; float* sK = sm + C::OFF_K; float* sV = sm + C::OFF_V; float* sP = sm + C::OFF_P;
  uint32_t* sMask = reinterpret_cast<uint32_t*>(sm + C::OFF_MASK);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  pdl_wait();
  pdl_launch_dependents();
  const int idx = (int)blockIdx.x / p.Hkv, kvh = (int)blockIdx.x % p.Hkv;
  if (idx >= p.plan->n_items) return;
  const SeqItem it = p.items[idx];
  const int G = p.G, rows = it.rows * G, n_tree = TREE ? seq_tree_tiles(p, it) : 0, chunks = p.dh / 4;
  // queries: rows and columns that are not there are zeros
  for (int i = tid; i < RT * (DHP / 4); i += 256) {
    const int r = i / (DHP / 4), c = i % (DHP / 4);
    const bool there = r < rows && c < chunks;
    const float* src = static_cast<const float*>(p.q) + (there ? (int64_t)(it.row0 + r / G) * p.q_stride + (kvh * G + r % G) * p.dh + c * 4 : 0);
    cp_async16(sQ + r * LD + c * 4, src, there);
  }
  // cached rows of the keys that this thread copies of a tile (-1: none): looked up a tile ahead of their copy
  constexpr int PER = KT * (DHP / 4) / 256;
  int64_t row_of[PER];
  auto look_up = [&](int t) {
    if (!TREE || t >= it.t1) return;
    const SeqTile s = seq_tile<TREE>(p, it, n_tree, t);
    if (s.kind != 1) return;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int j = s.j0 + (tid + u * 256) / (DHP / 4);
      row_of[u] = -1;
      if (j < s.n) {
        const int64_t pg = seq_page(p, it.a, j);
        if (pg < p.n_pages) row_of[u] = (pg * p.page_rows + (j & (p.page_rows - 1))) * p.Hkv + kvh;
      }
    }
  };
  auto fetch = [&](int t, int buf) {
    const SeqTile s = seq_tile<TREE>(p, it, n_tree, t);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int i = tid + u * 256, j = i / (DHP / 4), c = i % (DHP / 4);
      bool there = s.j0 + j < s.n && c < chunks;
      const float *kp = static_cast<const float*>(TREE ? p.q : p.k), *vp = kp;
      if (there) {
        if (!TREE || s.kind == 2) {
          const int64_t row = (int64_t)(TREE ? it.row0 - it.c : it.a) + s.j0 + j;
          kp = static_cast<const float*>(p.k) + row * p.k_stride + kvh * p.dh + c * 4;
          vp = static_cast<const float*>(p.v) + row * p.v_stride + kvh * p.dh + c * 4;
        } else {
          there = row_of[u] >= 0;
          if (there) {
            kp = static_cast<const float*>(p.ck) + row_of[u] * p.dh + c * 4;
            vp = static_cast<const float*>(p.cv) + row_of[u] * p.dh + c * 4;
          }
        }
      }
      cp_async16(sK + (buf * KT + j) * LD + c * 4, kp, there);
      cp_async16(sV + (buf * KT + j) * LD + c * 4, vp, there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float m[RI], l[RI], acc[RI][DC * VW];
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < DC * VW; ++c) acc[i][c] = 0.f;
  }
  // the row whose mask this thread keeps: its token, and how far up its chain of ancestors it has come
  const int mtok = tid < rows ? tid / G : 0;
  int anc = it.c + mtok;
  if (it.t0 < it.t1) {
    look_up(it.t0);
    fetch(it.t0, 0);
    look_up(it.t0 + 1);
  }
  for (int t = it.t0; t < it.t1; ++t) {
    const int buf = (t - it.t0) & 1;
    const SeqTile s = seq_tile<TREE>(p, it, n_tree, t);
    const bool masked = s.kind == 2 || (s.kind == 0 ? s.j0 + KT > it.c : s.j0 + KT > s.n);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    uint32_t* mask = sMask + buf * 2 * RT;           // a slower warp may still read the previous tile's
    if (masked && tid < RT) {
      uint32_t w0 = 0, w1 = 0;
      if (TREE && s.kind == 2) {
        while (anc >= s.j0) {
          const int bit = anc - s.j0;
          if (bit < 32) w0 |= 1u << bit; else if (bit < 64) w1 |= 1u << (bit - 32);
          anc = seq_parent(p, it.row0 - it.c, anc);
        }
      } else {
        const int n = (s.kind == 0 ? it.c + mtok : s.n) - s.j0;               // of the tile's keys
        w0 = n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1u : 0u;
        w1 = n >= 64 ? 0xffffffffu : n > 32 ? (1u << (n - 32)) - 1u : 0u;
      }
      mask[2 * tid] = w0; mask[2 * tid + 1] = w1;
    }
    __syncthreads();
    if (t + 1 < it.t1) fetch(t + 1, buf ^ 1);
    look_up(t + 2);
    const float *kb = sK + buf * KT * LD, *vb = sV + buf * KT * LD;
    float2 sc2[RI][4];                               // sums over even and odd features
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sc2[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < DHP; c += 4) {
      float4 kf[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kf[j] = *reinterpret_cast<const float4*>(kb + (tx + 16 * j) * LD + c);
#pragma unroll
      for (int i = 0; i < RI; ++i) {
        const float4 qf = *reinterpret_cast<const float4*>(sQ + (ty + 16 * i) * LD + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc2[i][j] = __ffma2_rn(make_float2(qf.x, qf.y), make_float2(kf[j].x, kf[j].y), sc2[i][j]);
          sc2[i][j] = __ffma2_rn(make_float2(qf.z, qf.w), make_float2(kf[j].z, kf[j].w), sc2[i][j]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < RI; ++i) {
      const int r = ty + 16 * i;
      bool sees[4];
      float mx = -INFINITY, sc[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sees[j] = !masked || ((mask[2 * r + (j >> 1)] >> (tx + 16 * (j & 1))) & 1u) != 0;
        sc[j] = sees[j] ? (sc2[i][j].x + sc2[i][j].y) * p.scale_log2 : -INFINITY;
        mx = fmaxf(mx, sc[j]);
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m[i], mx), ref = m_new == -INFINITY ? 0.f : m_new;
      const float factor = exp2f(m[i] - ref);
      m[i] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = exp2f(sc[j] - ref);
        if (sees[j]) sum += e;
        sP[r * PLD + tx + 16 * j] = sees[j] ? e : -1.f;
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      l[i] = l[i] * factor + sum;
#pragma unroll
      for (int c = 0; c < DC * VW; ++c) acc[i][c] *= factor;
    }
    __syncwarp();                                    // a row's probabilities come from the half warp that reads them
    auto values = [&](auto skip) {
#pragma unroll 2
      for (int j = 0; j < KT; j += 4) {
        float pf[RI][4];
#pragma unroll
        for (int i = 0; i < RI; ++i) *reinterpret_cast<float4*>(pf[i]) = *reinterpret_cast<const float4*>(sP + (ty + 16 * i) * PLD + j);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float vf[DC * VW];
#pragma unroll
          for (int c = 0; c < DC; ++c) {
            const float* src = vb + (j + jj) * LD + c * 16 * VW + tx * VW;
            if constexpr (VW == 4) *reinterpret_cast<float4*>(vf + c * VW) = *reinterpret_cast<const float4*>(src);
            else *reinterpret_cast<float2*>(vf + c * VW) = *reinterpret_cast<const float2*>(src);
          }
#pragma unroll
          for (int i = 0; i < RI; ++i) {
#pragma unroll
            for (int c = 0; c < DC * VW; c += 2) {
              float2& a = *reinterpret_cast<float2*>(&acc[i][c]);
              const float2 pp = make_float2(pf[i][jj], pf[i][jj]), vv = make_float2(vf[c], vf[c + 1]);
              if constexpr (decltype(skip)::value) fma2_unless_negative(a, pp, vv);
              else a = __ffma2_rn(pp, vv, a);
            }
          }
        }
      }
    };
    if (masked) values(std::true_type()); else values(std::false_type());
    __syncwarp();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  // the first row that sees a key
  const int seeing = TREE ? (it.b > 0 || p.k != nullptr ? 0 : RT) : min(max(1 - it.c, 0), RT) * G;
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int r = ty + 16 * i;
    if (r >= rows) continue;
    if (it.part < 0) {
      const float inv = seq_inverse(l[i], r >= seeing);
      float* o = static_cast<float*>(p.out) + (int64_t)(it.row0 + r / G) * p.out_stride + (kvh * G + r % G) * p.dh;
#pragma unroll
      for (int c = 0; c < DC; ++c)
        if (c * 16 * VW + tx * VW < p.dh)
#pragma unroll
          for (int e = 0; e < VW; ++e) o[c * 16 * VW + tx * VW + e] = acc[i][c * VW + e] * inv;
    } else {
      const int R = p.part_rows;
      const int64_t at = (int64_t)it.part * p.Hkv + kvh;
      if (tx == 0) { p.part_ml[at * 2 * R + r] = m[i]; p.part_ml[(at * 2 + 1) * R + r] = l[i]; }
      float* o = p.part_acc + (at * R + r) * p.dh;
#pragma unroll
      for (int c = 0; c < DC; ++c)
        if (c * 16 * VW + tx * VW < p.dh)
#pragma unroll
          for (int e = 0; e < VW; ++e) o[c * 16 * VW + tx * VW + e] = acc[i][c * VW + e];
    }
  }
}

template <int DHP, int RT, bool TREE>
static lime_status launch_simt(const SeqParams& p, cudaStream_t st) {
  static bool set[kMaxDeviceOrdinals] = {};
  constexpr int smem = SimtCfg<DHP, RT>::SMEM;
  const lime_status s = ensure_dynamic_smem((const void*)k_seq_attn_simt<DHP, RT, TREE>, smem, set);
  if (s != LIME_OK) return s;
  ProfScope _p("k_seq_attn_simt", st);
  launch_pdl(k_seq_attn_simt<DHP, RT, TREE>, dim3((unsigned)p.items_upper * p.Hkv), dim3(256), smem, st, p);
  LIME_LAUNCH_CHECK("k_seq_attn_simt");
  return LIME_OK;
}
template <int DHP>
static lime_status pick_simt(const SeqParams& p, bool tree, bool few, cudaStream_t st) {
  if (few) return tree ? launch_simt<DHP, 16, true>(p, st) : launch_simt<DHP, 16, false>(p, st);
  return tree ? launch_simt<DHP, 64, true>(p, st) : launch_simt<DHP, 64, false>(p, st);
}
lime_status launch_seq_attn_simt(const SeqParams& p, bool tree, bool few, cudaStream_t st) {
  return p.dh <= 32 ? pick_simt<32>(p, tree, few, st) : p.dh <= 64 ? pick_simt<64>(p, tree, few, st) : pick_simt<128>(p, tree, few, st);
}

}  // namespace lime

// What the tensor-core kernels of the sequence path's attention share (k_seq_attn_tc.cu, k_seq_attn_d64_tc.cu).
//
// Where a bounded wait gave up (lime_device_status): the barrier, by who waits.
//   d_h > 64: loads 111 kv_empty, 123 q_empty; scores 112 q_full, 113 kv_full, 114 s_free; values 115 kv_full, 116 mend_done, 117 p_ready,
//     124 o_free, 125 x_free; mending 118 kv_full, 119 mend_ask; softmax 120 s_full, 121 pv_done before a rescale, 122 pv_done at the end,
//     126 ml_full, 127 ml_free; 110: shared memory not aligned
//   d_h <= 64: loads 141 q_empty, 142 kv_empty; products 143 kv_full (keys), 144 q_full, 145 kv_full (values), 146 o_free, 147 p_ready, 151
//     s_free; softmax 148 s_full, 149 pv_done of the tile before, 150 pv_done at the end; 140: shared memory not aligned
#pragma once
#include "seq_common.cuh"
#include "tc_common.cuh"

namespace lime {

constexpr float kSeqRescale = 8.0f;                                // log2 units
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

// 4 x 4 transpose of 16-byte pieces inside each group of four lanes: lane 4j + i then holds piece i of rows 4j .. 4j + 3, so that every
// store instruction writes whole 64-byte parts of rows.
__device__ __forceinline__ void seq_xchg(uint4& keep_lo, uint4& keep_hi, bool upper, int dist) {
  // lanes with `upper` clear give away keep_hi and receive into it; lanes with it set give away keep_lo
  uint4 send = upper ? keep_lo : keep_hi, recv;
  recv.x = __shfl_xor_sync(0xffffffffu, send.x, dist); recv.y = __shfl_xor_sync(0xffffffffu, send.y, dist);
  recv.z = __shfl_xor_sync(0xffffffffu, send.z, dist); recv.w = __shfl_xor_sync(0xffffffffu, send.w, dist);
  if (upper) keep_lo = recv; else keep_hi = recv;
}
__device__ __forceinline__ void seq_transpose4(uint4 (&t)[4], int lane) {
  seq_xchg(t[0], t[1], (lane & 1) != 0, 1);
  seq_xchg(t[2], t[3], (lane & 1) != 0, 1);
  seq_xchg(t[0], t[2], (lane & 2) != 0, 2);
  seq_xchg(t[1], t[3], (lane & 2) != 0, 2);
}
// 32 columns of a warp's 32 rows, from column `col`, to the output (bf16) or to the partial results (fp32); `to`: where this lane's row
// begins there (elements), -1: nowhere; `dh`: columns a row has.
__device__ __forceinline__ void seq_store32(const SeqParams& p, bool whole, const float (&a)[32], int64_t to, int col, int lane) {
  if (whole) {
    uint4 t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      t[i] = make_uint4(seq_pack(a[8 * i], a[8 * i + 1]), seq_pack(a[8 * i + 2], a[8 * i + 3]), seq_pack(a[8 * i + 4], a[8 * i + 5]), seq_pack(a[8 * i + 6], a[8 * i + 7]));
    seq_transpose4(t, lane);
    const int at = col + (lane & 3) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = __shfl_sync(0xffffffffu, to, (lane & ~3) + i);
      if (row >= 0 && at < p.dh) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + row + at) = t[i];
    }
  } else {
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      uint4 t[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        t[i] = make_uint4(__float_as_uint(a[h + 4 * i]), __float_as_uint(a[h + 4 * i + 1]), __float_as_uint(a[h + 4 * i + 2]), __float_as_uint(a[h + 4 * i + 3]));
      seq_transpose4(t, lane);
      const int at = col + h + (lane & 3) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t row = __shfl_sync(0xffffffffu, to, (lane & ~3) + i);
        if (row >= 0 && at < p.dh) *reinterpret_cast<uint4*>(p.part_acc + row + at) = t[i];
      }
    }
  }
}
// 16 bytes of a value tile with what is not finite set to zero
__device__ __forceinline__ uint4 seq_finite8(uint4 x) {
  uint32_t* u = reinterpret_cast<uint32_t*>(&x);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if ((u[e] & 0x7f80u) == 0x7f80u) u[e] &= 0xffff0000u;
    if ((u[e] & 0x7f800000u) == 0x7f800000u) u[e] &= 0xffffu;
  }
  return x;
}
// Whether a row of the item does not see all keys of a tile of `keys`.
__device__ __forceinline__ bool seq_masked(const SeqItem& it, const SeqTile& k, int keys) {
  return k.kind == 2 || (k.kind == 0 ? k.j0 + keys > it.c : k.j0 + keys > k.n);
}
// Adds to a[0..31] (columns c0.. of the result of the item's token `token`) the values that are not finite of the keys that it sees in
// those tiles of lo .. hi that mask anything.
template <bool TREE>
__device__ __noinline__ void seq_add_not_finite(const SeqParams& p, int work, int token, int lo, int hi, int c0, float (&a)[32]) {
  const SeqItem it = p.items[work / p.Hkv];
  const int kvh = work % p.Hkv, n_tree = TREE ? seq_tree_tiles(p, it) : 0;
  const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v);
  auto add = [&](const __nv_bfloat16* row) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c0 + u * 8 >= p.dh) break;
      const uint4 x = *reinterpret_cast<const uint4*>(row + c0 + u * 8);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xffff0000u);
        if (!(fabsf(lo) < INFINITY)) a[u * 8 + 2 * e] += lo;
        if (!(fabsf(hi) < INFINITY)) a[u * 8 + 2 * e + 1] += hi;
      }
    }
  };
  int anc = it.c + token;                                  // the chain of ancestors is walked once, as its tiles come from the last one back
  for (int t = lo; t < hi; ++t) {
    const SeqTile k = seq_tile<TREE>(p, it, n_tree, t);
    if (!seq_masked(it, k, p.kt)) continue;
    if (TREE && k.kind == 2) {
      for (; anc >= k.j0; anc = seq_parent(p, it.row0 - it.c, anc))
        if (anc < k.j0 + p.kt) add(v + (int64_t)(it.row0 - it.c + anc) * p.v_stride + kvh * p.dh);
    } else {
      const int end = min(k.j0 + p.kt, TREE ? k.n : it.c + token);
      for (int j = k.j0; j < end; ++j) {
        if (!TREE) {
          add(v + (int64_t)(it.a + j) * p.v_stride + kvh * p.dh);
        } else {
          const int64_t pg = seq_page(p, it.a, j);
          if (pg < p.n_pages) add(static_cast<const __nv_bfloat16*>(p.cv) + ((pg * p.page_rows + (j & (p.page_rows - 1))) * p.Hkv + kvh) * p.dh);
        }
      }
    }
  }
}

__device__ __forceinline__ SeqItem seq_item(const SeqParams& p, int work) {
  const int4* src = reinterpret_cast<const int4*>(p.items + work / p.Hkv);
  const int4 x = src[0], y = src[1];
  return {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
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

// The tensor maps of a call: queries in boxes of q_rows tokens x G heads, keys and values in boxes of `keys` rows (pages: of at most a
// page).  Maps of tensors that are not there stand on the queries and are not read inside.
struct SeqMaps { CUtensorMap q, k, v, ck, cv; };
inline bool seq_make_maps(SeqMaps& m, const SeqParams& p, bool tree, int q_rows, int keys) {
  const bool fresh = p.k != nullptr && (tree || p.kv_rows > 0), pages = tree && p.n_pages > 0;
  const uint64_t rows = fresh ? (uint64_t)(tree ? p.q_rows : p.kv_rows) : 1, crows = pages ? (uint64_t)(p.n_pages * p.page_rows) : 1;
  const uint32_t box = (uint32_t)(tree && p.page_rows < keys ? p.page_rows : keys);
  return make_tmap_bf16_heads(&m.q, p.q, p.Hq, p.dh, (uint64_t)p.q_rows, p.q_stride, p.G, q_rows) &&
         make_tmap_bf16_heads(&m.k, fresh ? p.k : p.q, p.Hkv, p.dh, rows, fresh ? p.k_stride : p.q_stride, 1, keys) &&
         make_tmap_bf16_heads(&m.v, fresh ? p.v : p.q, p.Hkv, p.dh, rows, fresh ? p.v_stride : p.q_stride, 1, keys) &&
         make_tmap_bf16_heads(&m.ck, pages ? p.ck : p.q, p.Hkv, p.dh, crows, (uint64_t)p.Hkv * p.dh, 1, box) &&
         make_tmap_bf16_heads(&m.cv, pages ? p.cv : p.q, p.Hkv, p.dh, crows, (uint64_t)p.Hkv * p.dh, 1, box);
}

}  // namespace lime

// Attention of the sequence path for a few rows over the cache alone (bf16): new events whose keys are in the cache already, up to 8
// stacked rows (tokens x the query heads of one head of keys) an item, all of which see all of its keys.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(scale log2(e) (<q_i, k_j> - m_i))
//
// Bound: HBM, every key and value is read once for 8 rows or fewer.  So nothing is staged: a warp takes 16 keys at a time straight into
// registers in the layout of mma.sync m16n8k16 (tcgen05 has 128 rows a tile and a chain of hand-overs behind it, which is what bounds it
// here).  Both contractions are free in the order of their inner index, so a lane's 16 bytes of a key row are its share of two steps, and
// its values of 2 x 2 keys are paired by byte permutes:
//   S [16 (8 used) x 8 keys] += Q [16 x 16 features] . K^T       lane (g, t): key g, features 8t .. 8t+7 of every 32
//   O^T [16 features x 8]    += V^T [16 x 16 keys] . P^T         lane (g, t): keys 2t, 2t+1, 8+2t, 9+2t, features 8g .. 8g+7 of every 64
// where S, rounded, is P^T as it lies.  (O = P . V would keep rows 8..15 in registers for nothing: spills, 209 us for the events below.)
// The next keys are requested when the scores are formed, the next values when the products are.  A page has at least 16 rows, so 16
// aligned keys lie in one; the lanes look up the pages of 32 steps at once.  Four warps share an item's keys and are joined in shared
// memory; items are those of k_seq_schedule, dealt back and forth.
// Measured: 64 events of 16 heads over 16..16384 rows of 4 heads of 128 (1.07 GB) 180 us, 5.98 TB/s, 0.91 of the copy rate (221 on
// tcgen05); 256 over 512 rows of 4 heads of 32 24.5 us (53); 32 over 500..5000 rows of 8 heads of 64 44.6 us; one over 1000 rows of 2
// heads of 64 11.6 us (17), nearly all of it the latency of three launches.
// Online softmax, the reference raised when exceeded by 2^8; probabilities are rounded to bf16 for the value product (the operands of an
// mma have one type) and summed unrounded in fp32.
#include <type_traits>

#include "seq_tc.cuh"

namespace lime {

constexpr int kFewWarps = 4;

// 16 or 8 bytes, or zeros
__device__ __forceinline__ void few_load(uint4& x, const __nv_bfloat16* p, bool there) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\tmov.u32 %2, 0;\n\tmov.u32 %3, 0;\n\t"
               "@q ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "=&r"(x.x), "=&r"(x.y), "=&r"(x.z), "=&r"(x.w) : "l"(p), "r"((int)there));
}
__device__ __forceinline__ void few_load(uint2& x, const __nv_bfloat16* p, bool there) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %3, 0;\n\tmov.u32 %0, 0;\n\tmov.u32 %1, 0;\n\t"
               "@q ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];\n\t}"
               : "=&r"(x.x), "=&r"(x.y) : "l"(p), "r"((int)there));
}
// d [16 x 8] += a [16 x 16] . b [16 x 8]
__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int DHP>
__global__ void __launch_bounds__(32 * kFewWarps, seq_few_blocks(DHP)) k_seq_attn_few(const __grid_constant__ SeqParams p) {
  constexpr int KC = DHP / 32, VC = DHP >= 64 ? DHP / 64 : 1, VF = DHP >= 64 ? 8 : 4;       // chunks of a key row; of a value row, and their features
  __shared__ __align__(16) float s_o[kFewWarps][8][DHP];
  __shared__ float s_m[kFewWarps][8], s_l[kFewWarps][8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  pdl_wait();
  pdl_launch_dependents();
  const __nv_bfloat16 *q = static_cast<const __nv_bfloat16*>(p.q), *ck = static_cast<const __nv_bfloat16*>(p.ck), *cv = static_cast<const __nv_bfloat16*>(p.cv);
  const int n_work = p.plan->n_items * p.Hkv, G = p.G, R = p.part_rows;
  const int64_t step = (int64_t)p.Hkv * p.dh;
  int turn = 0;
  auto next_work = [&]() {                         // back and forth; -1: the end
    for (;;) {
      const int64_t first = (int64_t)turn * gridDim.x;
      if (first >= n_work) return -1;
      const int w = (int)first + ((turn & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x);
      ++turn;
      if (w < n_work) return w;
    }
  };
  int work = next_work();
  if (work < 0) return;
  SeqItem it = seq_item(p, work);
  uint4 qf[KC], kf[2][KC];
  typename std::conditional<DHP == 32, uint2, uint4>::type vf[4][VC];
  int kvh, end, rows, j, my_row;
  // first row in the cache of every step's keys, 32 steps of the warp at a time; -1: a page that is not there
  auto look_up = [&](int j) {
    j += lane * (16 * kFewWarps);
    my_row = -1;
    if (j < end) {
      const int64_t pg = seq_page(p, it.a, j);
      if (pg < p.n_pages) my_row = (int)(pg * p.page_rows + (j & (p.page_rows - 1)));
    }
  };
  auto load_k = [&](int j, int row) {
    const __nv_bfloat16* src = ck + (int64_t)max(row, 0) * step + kvh * p.dh + t * 8;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int c = 0; c < KC; ++c) few_load(kf[n][c], src + (n * 8 + g) * step + c * 32, row >= 0 && j + n * 8 + g < end && c * 32 + t * 8 < p.dh);
  };
  auto load_v = [&](int j, int row) {
    const __nv_bfloat16* src = cv + (int64_t)max(row, 0) * step + kvh * p.dh + g * VF;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = (u >> 1) * 8 + t * 2 + (u & 1);
      const bool there = row >= 0 && j + at < end;
#pragma unroll
      for (int c = 0; c < VC; ++c) few_load(vf[u][c], src + at * step + c * 64, there && c * 64 + g * VF < p.dh);
    }
  };
  auto begin = [&]() {
    kvh = work % p.Hkv;
    end = min(it.t1 * p.kt, it.b);
    rows = it.rows * G;
    j = it.t0 * p.kt + warp * 16;
    const __nv_bfloat16* src = q + (int64_t)(it.row0 + g / G) * p.q_stride + (kvh * G + g % G) * p.dh + t * 8;
#pragma unroll
    for (int c = 0; c < KC; ++c) few_load(qf[c], src + c * 32, g < rows && c * 32 + t * 8 < p.dh);
    look_up(j);
  };
  begin();
#pragma unroll 1
  for (;;) {
    int row = __shfl_sync(0xffffffffu, my_row, 0);
    load_k(j, row);
    load_v(j, row);
    float o[VC][VF / 2][4], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int f = 0; f < VF / 2; ++f) o[c][f][0] = o[c][f][1] = o[c][f][2] = o[c][f][3] = 0.f;
#pragma unroll 1
    for (int n = 1; j < end; ++n) {
      float s[2][4];                               // rows 8..15 are zeros
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          few_mma(s[h], qf[c].x, 0, qf[c].y, 0, kf[h][c].x, kf[h][c].y);
          few_mma(s[h], qf[c].z, 0, qf[c].w, 0, kf[h][c].z, kf[h][c].w);
        }
      }
      const int next = j + 16 * kFewWarps;
      if ((n & 31) == 0) look_up(next);
      row = __shfl_sync(0xffffffffu, my_row, n & 31);
      load_k(next, row);
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          s[h][e] = j + h * 8 + t * 2 + e < end ? s[h][e] * p.scale_log2 : -INFINITY;
          top = fmaxf(top, s[h][e]);
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      if (__any_sync(0xffffffffu, top > m + 8.f)) {
        const float to = fmaxf(top, m), w = to == -INFINITY ? 1.f : seq_ex2(m - to);
        m = to;
        l *= w;
        const float w0 = __shfl_sync(0xffffffffu, w, t * 8), w1 = __shfl_sync(0xffffffffu, w, t * 8 + 4);
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int f = 0; f < VF / 2; ++f) { o[c][f][0] *= w0; o[c][f][1] *= w1; o[c][f][2] *= w0; o[c][f][3] *= w1; }
      }
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) { s[h][e] = seq_ex2(s[h][e] - ref); l += s[h][e]; }
      const uint32_t p0 = seq_pack(s[0][0], s[0][1]), p1 = seq_pack(s[1][0], s[1][1]);
#pragma unroll
      for (int c = 0; c < VC; ++c)
#pragma unroll
        for (int f = 0; f < VF / 2; ++f) {
          const uint32_t a = (&vf[0][c].x)[f], b = (&vf[1][c].x)[f], d = (&vf[2][c].x)[f], e = (&vf[3][c].x)[f];
          few_mma(o[c][f], __byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(d, e, 0x5410), __byte_perm(d, e, 0x7632), p0, p1);
        }
      load_v(next, row);
      j = next;
    }
    // the next item is looked up while this one is joined
    const int row0 = it.row0, part = it.part, was_rows = rows, was_kvh = kvh;
    const bool any = it.t0 < it.t1;
    work = next_work();
    if (work >= 0) it = seq_item(p, work);
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
    for (int c = 0; c < VC; ++c)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int f = 0; f < VF / 2; f += 2)
          *reinterpret_cast<float4*>(&s_o[warp][t * 2 + e][c * 64 + g * VF + f * 2]) = make_float4(o[c][f][e], o[c][f][2 + e], o[c][f + 1][e], o[c][f + 1][2 + e]);
    if (t == 0) { s_m[warp][g] = m; s_l[warp][g] = l; }
    __syncthreads();
    if (work >= 0) begin();
#pragma unroll 1
    for (int i = tid; i < was_rows * (DHP / 4); i += 32 * kFewWarps) {
      const int r = i / (DHP / 4), at = i % (DHP / 4) * 4;
      float top = s_m[0][r], sum = 0.f;
#pragma unroll
      for (int w = 1; w < kFewWarps; ++w) top = fmaxf(top, s_m[w][r]);
      const float ref = top == -INFINITY ? 0.f : top;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        const float f = seq_ex2(s_m[w][r] - ref);
        const float4 x = *reinterpret_cast<const float4*>(&s_o[w][r][at]);
        sum = fmaf(f, s_l[w][r], sum);
        acc.x = fmaf(f, x.x, acc.x); acc.y = fmaf(f, x.y, acc.y); acc.z = fmaf(f, x.z, acc.z); acc.w = fmaf(f, x.w, acc.w);
      }
      if (at >= p.dh) continue;
      if (part < 0) {
        const float inv = seq_inverse(sum, any);
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.out) + (int64_t)(row0 + r / G) * p.out_stride + (was_kvh * G + r % G) * p.dh + at;
        *reinterpret_cast<uint2*>(to) = make_uint2(seq_pack(acc.x * inv, acc.y * inv), seq_pack(acc.z * inv, acc.w * inv));
      } else {
        const int64_t at_part = (int64_t)part * p.Hkv + was_kvh;
        if (at == 0) { p.part_ml[at_part * 2 * R + r] = top; p.part_ml[(at_part * 2 + 1) * R + r] = sum; }
        *reinterpret_cast<float4*>(p.part_acc + (at_part * R + r) * p.dh + at) = acc;
      }
    }
    if (work < 0) return;
    __syncthreads();
  }
}

lime_status launch_seq_attn_few(const SeqParams& p, cudaStream_t st) {
  const int64_t work = (int64_t)p.items_upper * p.Hkv;
  const dim3 grid((unsigned)(work < p.ctas ? work : p.ctas));
  ProfScope _p("k_seq_attn_few", st);
  if (p.dh <= 32) launch_pdl(k_seq_attn_few<32>, grid, dim3(32 * kFewWarps), 0, st, p);
  else if (p.dh <= 64) launch_pdl(k_seq_attn_few<64>, grid, dim3(32 * kFewWarps), 0, st, p);
  else launch_pdl(k_seq_attn_few<128>, grid, dim3(32 * kFewWarps), 0, st, p);
  LIME_LAUNCH_CHECK("k_seq_attn_few");
  return LIME_OK;
}

}  // namespace lime

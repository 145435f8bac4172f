// Norm of every head and rotation by position in one pass, keys and values on to the cache (lime_norm_rotate):
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma,   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * base^(-2i / rot_dim)
//
// Bound: HBM; every row is read once and written once per place it goes to.  What it costs besides is instructions, so they are shared: a
// group of lanes takes several heads of one token, a head's row at a time, 8 features a lane (16 bytes of bf16, a warp reads and writes
// whole lines).  The token's cosines and sines, formed once per block, and the gains are multiplied once per thread, out = (r x) A +
// (r x') B with x' the other half of the pair: from the lane itself (neighbours), by shuffle as stored (halves of whole lanes), or else
// through shared memory; arithmetic on pairs of fp32.  Values are copied without any.
// Measured: 30011 rows of 16 + 4 + 4 heads of 128 (bf16, keys to the cache as well) 83 us, 4.8 TB/s, 0.74 of the copy rate; 131072
// rows of 4 + 4 + 4 heads of 32 56.0 us; 10007 rows of 8 + 2 heads of 64 (fp32) 14.5 us.  Three blocks an SM (80 registers) issue in 0.59, 0.44
// and 0.48 of the cycles: what is left is latency.  Before: a row per group at a time, gains and angles per row, 198, 166 and 24.8 us; four
// heads a thread instead of eight 110.8 us, no prefetch 91.2 us, four blocks an SM 90.7 us.
// Angles: a position times a frequency in turns, as an integer fraction of 2^64, wraps by itself and keeps all of its bits: the product is
// exact to 2^-33 of a turn for any 32-bit position, where one in fp32 would have lost it beyond some thousand.  Rounded to fp32 for the
// sine, within half a turn of 0, it is off by 2^-26 of a turn at most (9.4e-8 radians, 1.6 roundings of 1).
#include "seq_common.cuh"

namespace lime {

struct NormRotateParams {
  const void *q, *k, *v, *gamma_q, *gamma_k;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, cache_rows;
  const int32_t *positions, *slots;
  void *q_out, *k_out, *cache_k, *cache_v;
  int32_t* dev_flag;
  int64_t rows;
  int Hq, Hkv, dh, rot, interleaved, share, tokens;
  float eps;
  uint64_t freq[64];
};

// 8 features of a head as stored
template <typename T> struct Row8;
template <> struct Row8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = a; *reinterpret_cast<float4*>(p + 4) = b; }
  __device__ __forceinline__ void get(float2 (&f)[4]) const { f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w); }
  __device__ __forceinline__ void put(const float2 (&f)[4]) { a = make_float4(f[0].x, f[0].y, f[1].x, f[1].y); b = make_float4(f[2].x, f[2].y, f[3].x, f[3].y); }
  __device__ __forceinline__ Row8 from(int lane) const {
    Row8 r;
    r.a.x = __shfl_sync(0xffffffffu, a.x, lane); r.a.y = __shfl_sync(0xffffffffu, a.y, lane); r.a.z = __shfl_sync(0xffffffffu, a.z, lane); r.a.w = __shfl_sync(0xffffffffu, a.w, lane);
    r.b.x = __shfl_sync(0xffffffffu, b.x, lane); r.b.y = __shfl_sync(0xffffffffu, b.y, lane); r.b.z = __shfl_sync(0xffffffffu, b.z, lane); r.b.w = __shfl_sync(0xffffffffu, b.w, lane);
    return r;
  }
};
template <> struct Row8<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void get(float2 (&f)[4]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xffff0000u));
  }
  __device__ __forceinline__ void put(const float2 (&f)[4]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[i].x, f[i].y);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
  __device__ __forceinline__ Row8 from(int lane) const {
    Row8 r;
    r.w.x = __shfl_sync(0xffffffffu, w.x, lane); r.w.y = __shfl_sync(0xffffffffu, w.y, lane); r.w.z = __shfl_sync(0xffffffffu, w.z, lane); r.w.w = __shfl_sync(0xffffffffu, w.w, lane);
    return r;
  }
};

constexpr int kRotThreads = 256, kRotTurns = 1024;
template <typename T> constexpr int kRotFlight = 8 / sizeof(T);          // rows of a thread in flight: 4 of bf16, 2 of fp32
enum { ROT_NEIGHBOURS = 0, ROT_LANES = 1, ROT_ANY = 2 };

// LANES lanes per head row (a power of two, 8 features each; those past dh / 8 idle); `share` groups of lanes work on one token, `tokens`
// tokens per block.
template <typename T, int LANES, int MODE>
__global__ void __launch_bounds__(kRotThreads, 3) k_norm_rotate(const __grid_constant__ NormRotateParams p) {
  __shared__ __align__(16) float s_turn[2 * kRotTurns];
  __shared__ __align__(16) float s_row[MODE == ROT_ANY ? kRotThreads / LANES : 1][LANES * 8];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
  const int n = (int)min((int64_t)p.tokens, p.rows - t0), half = p.rot / 2;
  const int grp = threadIdx.x / LANES, lane = threadIdx.x % LANES, sub = grp % p.share, tt = grp / p.share;
  const bool mine = tt < n && lane * 8 < p.dh;
  const int64_t row = t0 + (tt < n ? tt : 0);
  int slot = -1;
  if (p.cache_k != nullptr && tt < n) {
    slot = __ldg(p.slots + row);
    if (slot < -1 || slot >= p.cache_rows) {
      if (sub == 0 && lane == 0 && p.dev_flag != nullptr) atomicMin(p.dev_flag, (int32_t)row);
      slot = -1;
    }
  }
  // the rows are on their way into L2 while the angles are formed
  if (mine && (lane * 8 * sizeof(T)) % 128 == 0) {
    for (int h = sub; h < p.Hq; h += p.share) prefetch_l2(static_cast<const T*>(p.q) + row * p.q_stride + h * p.dh + lane * 8);
    for (int h = sub; h < p.Hkv; h += p.share) {
      prefetch_l2(static_cast<const T*>(p.k) + row * p.k_stride + h * p.dh + lane * 8);
      if (p.v != nullptr) prefetch_l2(static_cast<const T*>(p.v) + row * p.v_stride + h * p.dh + lane * 8);
    }
  }
  // cosines of all tokens, then the sines; a thread keeps its frequency
  float *s_cos = s_turn, *s_sin = s_turn + kRotTurns;
  if (half > 0) {
    const int per = kRotThreads / half, f = threadIdx.x % half;
    const uint64_t freq = p.freq[f];
    for (int t = threadIdx.x / half; t < n && threadIdx.x < per * half; t += per) {
      const uint64_t turn = (uint64_t)(int64_t)__ldg(p.positions + t0 + t) * freq;          // modulo one turn
      sincospif((float)(int32_t)(turn >> 32) * (1.f / 2147483648.f), s_sin + t * half + f, s_cos + t * half + f);
    }
  }
  __syncthreads();
  const bool turned = mine && lane * 8 < p.rot;
  // the lane that holds the other halves of the lane's pairs (the group's first lane of a warp is a multiple of LANES)
  const int partner = (threadIdx.x & 31) + (MODE != ROT_LANES || !turned ? 0 : lane * 8 < half ? half / 8 : -(half / 8));
  float2 cs[4], sn[4];                                 // of the lane's features, the sine with the sign that the partner gets
#pragma unroll
  for (int i = 0; i < 4; ++i) { cs[i] = make_float2(1.f, 1.f); sn[i] = make_float2(0.f, 0.f); }
  if (turned) {
    if (MODE == ROT_NEIGHBOURS) {
      const float4 c = *reinterpret_cast<const float4*>(s_cos + tt * half + lane * 4), w = *reinterpret_cast<const float4*>(s_sin + tt * half + lane * 4);
      cs[0] = make_float2(c.x, c.x); cs[1] = make_float2(c.y, c.y); cs[2] = make_float2(c.z, c.z); cs[3] = make_float2(c.w, c.w);
      sn[0] = make_float2(-w.x, w.x); sn[1] = make_float2(-w.y, w.y); sn[2] = make_float2(-w.z, w.z); sn[3] = make_float2(-w.w, w.w);
    } else if (MODE == ROT_LANES) {
      const bool second = lane * 8 >= half;
      const int at = tt * half + lane * 8 - (second ? half : 0);
      const float2 sign = second ? make_float2(1.f, 1.f) : make_float2(-1.f, -1.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cs[i] = *reinterpret_cast<const float2*>(s_cos + at + 2 * i);
        sn[i] = __fmul2_rn(*reinterpret_cast<const float2*>(s_sin + at + 2 * i), sign);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = lane * 8 + e;
        if (at >= p.rot) break;
        const bool second = p.interleaved ? (at & 1) != 0 : at >= half;
        const int i = tt * half + (p.interleaved ? at >> 1 : second ? at - half : at);
        reinterpret_cast<float*>(cs)[e] = s_cos[i];
        reinterpret_cast<float*>(sn)[e] = second ? s_sin[i] : -s_sin[i];
      }
    }
  }
  const int64_t at_cache = (int64_t)slot * p.Hkv * p.dh + lane * 8;
  const float inv_dh = 1.f / (float)p.dh;
  constexpr int FLIGHT = kRotFlight<T>;

  auto heads_of = [&](const T* src, const T* gamma, int heads, T* dst, T* dst2) {
    float2 A[4], B[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { A[i] = cs[i]; B[i] = sn[i]; }
    if (gamma != nullptr) {
      float2 g[4], o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = make_float2(1.f, 1.f);
      Row8<T> w;
      w.put(g);
      if (lane * 8 < p.dh) w.load(gamma + lane * 8);
      w.get(g);
      if (MODE == ROT_NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = make_float2(g[i].y, g[i].x);
      } else if (MODE == ROT_LANES) {
        w.from(partner).get(o);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int at = lane * 8 + e;
          reinterpret_cast<float*>(o)[e] = at >= p.rot ? 1.f : Store<T>::ld(gamma + (p.interleaved ? at ^ 1 : at < half ? at + half : at - half));
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) { A[i] = __fmul2_rn(A[i], g[i]); B[i] = __fmul2_rn(B[i], o[i]); }
    }
    src += lane * 8;
    for (int h0 = 0; h0 < heads; h0 += FLIGHT * p.share) {
      Row8<T> x[FLIGHT];
#pragma unroll
      for (int u = 0; u < FLIGHT; ++u) {
        const int h = h0 + u * p.share + sub;
        if (mine && h < heads) x[u].load(src + h * p.dh);
      }
#pragma unroll
      for (int u = 0; u < FLIGHT; ++u) {
        if (h0 + u * p.share >= heads) break;
        const int h = h0 + u * p.share + sub;
        const bool live = mine && h < heads;
        float2 f[4], o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = make_float2(0.f, 0.f);
        if (live) x[u].get(f);
        float2 s2 = __fmul2_rn(f[0], f[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) s2 = __ffma2_rn(f[i], f[i], s2);
        float ss = s2.x + s2.y;
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float r = rsqrtf(fmaf(ss, inv_dh, p.eps));
        const float2 r2 = make_float2(r, r);
        if (MODE == ROT_NEIGHBOURS) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = turned ? make_float2(f[i].y, f[i].x) : f[i];
        } else if (MODE == ROT_LANES) {
          x[u].from(partner).get(o);
        } else {
          float* buf = s_row[grp];
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(buf + lane * 8 + 2 * i) = f[i];
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int at = lane * 8 + e;
            reinterpret_cast<float*>(o)[e] = buf[at >= p.rot ? at : p.interleaved ? at ^ 1 : at < half ? at + half : at - half];
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __ffma2_rn(__fmul2_rn(f[i], r2), A[i], __fmul2_rn(__fmul2_rn(o[i], r2), B[i]));
        if (live) {
          x[u].put(f);
          if (dst != nullptr) x[u].store(dst + h * p.dh);
          if (dst2 != nullptr) x[u].store(dst2 + h * p.dh);
        }
      }
    }
  };
  heads_of(static_cast<const T*>(p.q) + row * p.q_stride, static_cast<const T*>(p.gamma_q), p.Hq, static_cast<T*>(p.q_out) + row * p.q_out_stride + lane * 8, nullptr);
  heads_of(static_cast<const T*>(p.k) + row * p.k_stride, static_cast<const T*>(p.gamma_k), p.Hkv,
           p.k_out != nullptr ? static_cast<T*>(p.k_out) + row * p.k_out_stride + lane * 8 : nullptr, slot >= 0 ? static_cast<T*>(p.cache_k) + at_cache : nullptr);
  if (p.v != nullptr && slot >= 0 && mine)
    for (int h = sub; h < p.Hkv; h += p.share) {
      Row8<T> x;
      x.load(static_cast<const T*>(p.v) + row * p.v_stride + h * p.dh + lane * 8);
      x.store(static_cast<T*>(p.cache_v) + at_cache + h * p.dh);
    }
}

template <typename T, int LANES>
static void launch_lanes(NormRotateParams& p, cudaStream_t st) {
  // Groups per token: up to eight query heads each where there are many rows, one each where a call is short.
  const int groups = kRotThreads / LANES;
  const int64_t each = p.rows * p.Hq * LANES / (8ll * kSMs * kRotThreads);
  const int per = each < 1 ? 1 : each > 8 ? 8 : (int)each;
  p.share = (p.Hq + per - 1) / per;
  if (p.share > groups) p.share = groups;
  p.tokens = groups / p.share;
  if (p.rot > 0 && p.tokens > kRotTurns / (p.rot / 2)) p.tokens = kRotTurns / (p.rot / 2);
  const dim3 grid((unsigned)((p.rows + p.tokens - 1) / p.tokens)), block(kRotThreads);
  if (p.rot == 0 || (p.interleaved && p.rot % 8 == 0)) launch_pdl(k_norm_rotate<T, LANES, ROT_NEIGHBOURS>, grid, block, 0, st, p);
  else if (!p.interleaved && p.rot % 16 == 0) launch_pdl(k_norm_rotate<T, LANES, ROT_LANES>, grid, block, 0, st, p);
  else launch_pdl(k_norm_rotate<T, LANES, ROT_ANY>, grid, block, 0, st, p);
}
template <typename T>
static void launch_dtype(NormRotateParams& p, cudaStream_t st) {
  if (p.dh <= 8) launch_lanes<T, 1>(p, st);
  else if (p.dh <= 16) launch_lanes<T, 2>(p, st);
  else if (p.dh <= 32) launch_lanes<T, 4>(p, st);
  else if (p.dh <= 64) launch_lanes<T, 8>(p, st);
  else launch_lanes<T, 16>(p, st);
}

lime_status launch_norm_rotate(const NormRotateArgs& a, cudaStream_t st) {
  NormRotateParams p;
  p.q = a.q; p.k = a.k; p.v = a.v; p.gamma_q = a.gamma_q; p.gamma_k = a.gamma_k;
  p.q_stride = a.q_stride; p.k_stride = a.k_stride; p.v_stride = a.v_stride; p.q_out_stride = a.q_out_stride; p.k_out_stride = a.k_out_stride;
  p.cache_rows = a.cache_rows; p.positions = a.positions; p.slots = a.slots; p.q_out = a.q_out; p.k_out = a.k_out;
  p.cache_k = a.cache_k; p.cache_v = a.cache_v; p.dev_flag = a.dev_flag; p.rows = a.rows;
  p.Hq = a.seq->Hq; p.Hkv = a.seq->Hkv; p.dh = a.seq->d_h; p.rot = a.seq->rot_dim; p.interleaved = a.seq->rot_interleaved; p.eps = a.seq->norm_eps;
  for (int i = 0; i < 64; ++i) p.freq[i] = a.rot_freq[i];
  ProfScope _p("k_norm_rotate", st);
  if (a.dtype == LIME_BF16) launch_dtype<__nv_bfloat16>(p, st);
  else launch_dtype<float>(p, st);
  LIME_LAUNCH_CHECK("k_norm_rotate");
  return LIME_OK;
}

}  // namespace lime

// Norm of every head and rotation by position in one pass, keys and values on to the cache (lime_norm_rotate):
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma,   (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * base^(-2i / rot_dim)
//
// Bound: HBM; every row is read once and written once per place it goes to.  A block takes kTokens rows of all heads: it forms the
// cosines and sines of these rows once (they serve every head), then a group of lanes takes a head's row, 8 features a lane (16 bytes of
// bf16, so a warp reads and writes whole lines), sums the squares by shuffles and exchanges the pairs through shared memory.
// Angles: a position times a frequency in turns, as an integer fraction of 2^64, wraps by itself and keeps all of its bits: what is left
// of the turn is exact to 2^-33 for any 32-bit position, where a product in fp32 would have lost it beyond some thousand.
#include "seq_common.cuh"

namespace lime {

struct NormRotateParams {
  const void *q, *k, *v, *gamma_q, *gamma_k;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride, cache_rows;
  const int32_t *positions, *slots;
  void *q_out, *k_out, *cache_k, *cache_v;
  int32_t* dev_flag;
  int64_t rows;
  int Hq, Hkv, dh, rot, interleaved;
  float eps;
  uint64_t freq[64];
};

template <typename T> struct Row8;
template <> struct Row8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = a; *reinterpret_cast<float4*>(p + 4) = b; }
  __device__ __forceinline__ void get(float (&f)[8]) const { f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w; }
  __device__ __forceinline__ void put(const float (&f)[8]) { a = make_float4(f[0], f[1], f[2], f[3]); b = make_float4(f[4], f[5], f[6], f[7]); }
};
template <> struct Row8<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ void put(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
};

constexpr int kRotThreads = 256;

// LANES lanes per head row (a power of two, 8 features each; those past dh / 8 idle), TOKENS rows per block
template <typename T, int LANES, int TOKENS>
__global__ void __launch_bounds__(kRotThreads) k_norm_rotate(const __grid_constant__ NormRotateParams p) {
  __shared__ float2 s_turn[TOKENS][64];
  __shared__ __align__(16) float s_row[kRotThreads / LANES][LANES * 8];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
  const int n = (int)min((int64_t)TOKENS, p.rows - t0), half = p.rot / 2;
  for (int i = threadIdx.x; i < n * half; i += kRotThreads) {
    const int t = i / half, f = i % half;
    const uint64_t turn = (uint64_t)(int64_t)__ldg(p.positions + t0 + t) * p.freq[f];          // modulo one turn
    float sn, cs;
    sincospif((float)(int32_t)(turn >> 32) * (1.f / 2147483648.f), &sn, &cs);
    s_turn[t][f] = make_float2(cs, sn);
  }
  __syncthreads();
  const int grp = threadIdx.x / LANES, lane = threadIdx.x % LANES, heads = p.Hq + p.Hkv + (p.v != nullptr ? p.Hkv : 0);
  const bool mine = lane * 8 < p.dh;
  for (int i0 = 0; i0 < n * heads; i0 += kRotThreads / LANES) {
    const int i = i0 + grp;
    const bool live = i < n * heads;
    const int t = live ? i / heads : 0, h = live ? i % heads : 0;
    const int64_t row = t0 + t;
    const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
    const int hk = is_q ? h : is_v ? h - p.Hq - p.Hkv : h - p.Hq;
    const T* src = is_q ? static_cast<const T*>(p.q) + row * p.q_stride : is_v ? static_cast<const T*>(p.v) + row * p.v_stride : static_cast<const T*>(p.k) + row * p.k_stride;
    src += hk * p.dh + lane * 8;
    Row8<T> x;
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (live && mine) { x.load(src); x.get(f); }
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (!is_v) {
      const float r = rsqrtf(ss / (float)p.dh + p.eps);
      const void* gamma = is_q ? p.gamma_q : p.gamma_k;
      float g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (gamma != nullptr && mine) { Row8<T> w; w.load(static_cast<const T*>(gamma) + lane * 8); w.get(g); }
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = f[e] * r * g[e];
    }
    float* buf = s_row[grp];
    *reinterpret_cast<float4*>(buf + lane * 8) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(buf + lane * 8 + 4) = make_float4(f[4], f[5], f[6], f[7]);
    __syncwarp();
    if (!is_v && lane * 8 < p.rot) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = lane * 8 + e;
        if (at >= p.rot) break;
        const bool second = p.interleaved ? (e & 1) != 0 : at >= half;
        const int pair = p.interleaved ? at >> 1 : second ? at - half : at;
        const float other = buf[p.interleaved ? at ^ 1 : second ? at - half : at + half];
        const float2 w = s_turn[t][pair];
        f[e] = second ? fmaf(f[e], w.x, other * w.y) : fmaf(f[e], w.x, -(other * w.y));
      }
    }
    __syncwarp();
    if (!live || !mine) continue;
    if (!is_v) x.put(f);
    if (is_q) {
      x.store(static_cast<T*>(p.q_out) + row * p.q_out_stride + hk * p.dh + lane * 8);
      continue;
    }
    if (!is_v && p.k_out != nullptr) x.store(static_cast<T*>(p.k_out) + row * p.k_out_stride + hk * p.dh + lane * 8);
    if (p.cache_k != nullptr) {
      const int slot = __ldg(p.slots + row);
      if (slot >= 0 && slot < p.cache_rows)
        x.store(static_cast<T*>(is_v ? p.cache_v : p.cache_k) + ((int64_t)slot * p.Hkv + hk) * p.dh + lane * 8);
      else if (slot != -1 && p.dev_flag != nullptr)
        atomicMin(p.dev_flag, (int32_t)row);
    }
  }
}

template <typename T, int LANES>
static void launch_lanes(const NormRotateParams& p, cudaStream_t st) {
  constexpr int tokens = 4;
  launch_pdl(k_norm_rotate<T, LANES, tokens>, dim3((unsigned)((p.rows + tokens - 1) / tokens)), dim3(kRotThreads), 0, st, p);
}
template <typename T>
static void launch_dtype(const NormRotateParams& p, cudaStream_t st) {
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

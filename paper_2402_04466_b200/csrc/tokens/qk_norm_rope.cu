// Queries' and keys' RMS norm per head and position rotation, one pass (tt_qk_norm_rope).
//
//   y = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> s * (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq[i]
//
// Bound by memory: every row is read and written once.  A row of D elements belongs to D / 8 lanes with eight elements each, so a row's
// sum of squares is a butterfly over at most 16 lanes and both elements of a pair sit in one lane: with the halves layout a
// lane below rot / 8 holds elements 4l..4l+3 and their partners rot / 2 further on, with the interleaved layout 8l..8l+7.
// All heads of a token share its angles: a block works them out once for its tokens, before the rows arrive, and
// keeps cosine and sine in shared memory.  The angle is reduced in 64 bits (turns = position * inv_freq / 2 pi, less the
// nearest whole number): at position 5e6 a product of 32 bits would be off by 0.3 radians.
#include "tokens.h"

#include "../tc_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int THREADS = 256;
constexpr int ROWS_PER_THREAD = 2;     // in flight together

template <typename T>
struct Four;     // four neighbouring elements
template <>
struct Four<float> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float* f) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  static __device__ __forceinline__ void store(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
};
template <>
struct Four<__nv_bfloat16> {
  uint2 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
    *reinterpret_cast<uint2*>(p) = make_uint2(tc::pack_bf16(f[0], f[1]), tc::pack_bf16(f[2], f[3]));
  }
};

template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS) qk_norm_rope_kernel(const __grid_constant__ RopeParams p, int tokens_per_block) {
  constexpr int LANES = D / 8;                      // to a row
  constexpr int GROUPS = THREADS / LANES;           // rows at a time
  extern __shared__ float2 angle[];                 // [tokens_per_block][rot / 2]: cosine and sine, with rot_scale
  const int b = blockIdx.y;
  const int n = clamp_length(p.lengths, b, p.tokens);
  const int t0 = (int)blockIdx.x * tokens_per_block;
  if (t0 >= n) return;
  const int nt = min(tokens_per_block, n - t0);
  const int half = p.rot >> 1;
  for (int i = threadIdx.x; i < nt * half; i += THREADS) {
    const int t = i / half, c = i - t * half;
    const double turns = (double)p.positions[(int64_t)b * p.pos_stride + t0 + t] * (p.inv_freq[c] * 0.15915494309189533577);
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    angle[i] = make_float2(cs * p.rot_scale, sn * p.rot_scale);
  }
  __syncthreads();
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int heads = p.heads[0] + p.heads[1], rows = nt * heads;
  const bool turned = lane * 8 < p.rot;
  // the two runs of four elements of this lane
  const int e0 = !INTERLEAVED && turned ? lane * 4 : lane * 8;
  const int e1 = !INTERLEAVED && turned ? lane * 4 + half : lane * 8 + 4;
  float w[2][8];
  for (int s = 0; s < 2; ++s)
    for (int j = 0; j < 8; ++j) w[s][j] = p.weight[s] ? p.weight[s][(j < 4 ? e0 : e1 - 4) + j] : 1.f;

  for (int r0 = 0; r0 < rows; r0 += GROUPS * ROWS_PER_THREAD) {
    Four<T> a[ROWS_PER_THREAD][2];
    T* dst[ROWS_PER_THREAD];
    int tok[ROWS_PER_THREAD], side[ROWS_PER_THREAD];
#pragma unroll
    for (int u = 0; u < ROWS_PER_THREAD; ++u) {
      const int r = r0 + u * GROUPS + group;
      const int t = r / heads, hh = r - t * heads;
      side[u] = hh >= p.heads[0];
      const int h = side[u] ? hh - p.heads[0] : hh;
      tok[u] = r < rows ? t : -1;
      const View& x = p.x[side[u]];
      const View& y = p.y[side[u]];
      const T* src = reinterpret_cast<const T*>(x.p) + b * x.b + (int64_t)(t0 + t) * x.t + h * x.h;
      dst[u] = reinterpret_cast<T*>(y.p) + b * y.b + (int64_t)(t0 + t) * y.t + h * y.h;
      if (tok[u] >= 0) {
        a[u][0].load(src + e0);
        a[u][1].load(src + e1);
      }
    }
#pragma unroll
    for (int u = 0; u < ROWS_PER_THREAD; ++u) {
      float f[8];
      a[u][0].get(f);
      a[u][1].get(f + 4);
      if (p.norm) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(f[j], f[j], q);
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
        const float inv = 1.f / sqrtf(q * (1.f / D) + p.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = f[j] * inv * (side[u] ? w[1][j] : w[0][j]);
      }
      if (tok[u] < 0) continue;
      if (turned) {
        const float2* ang = angle + tok[u] * half + lane * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 cs = ang[j];
          float& lo = INTERLEAVED ? f[2 * j] : f[j];
          float& hi = INTERLEAVED ? f[2 * j + 1] : f[j + 4];
          const float x0 = lo, x1 = hi;
          lo = x0 * cs.x - x1 * cs.y;
          hi = x1 * cs.x + x0 * cs.y;
        }
      }
      Four<T>::store(dst[u] + e0, f);
      Four<T>::store(dst[u] + e1, f + 4);
    }
  }
}

template <typename T, int D>
cudaError_t launch(const RopeParams& p, bool interleaved, cudaStream_t s) {
  const int heads = p.heads[0] + p.heads[1];
  // a block's rows: two rounds of all its threads where the tokens fill the device, at least one token
  const int rows = THREADS / (D / 8) * ROWS_PER_THREAD * 2;
  int per_block = rows / heads < 1 ? 1 : rows / heads;
  while (per_block > 1 && (int64_t)((p.tokens + per_block - 1) / per_block) * p.batch < 2 * PLAN_SMS) per_block >>= 1;
  const dim3 grid((unsigned)((p.tokens + per_block - 1) / per_block), (unsigned)p.batch);
  const size_t smem = (size_t)per_block * (size_t)(p.rot / 2) * sizeof(float2);
  if (interleaved) qk_norm_rope_kernel<T, D, true><<<grid, THREADS, smem, s>>>(p, per_block);
  else qk_norm_rope_kernel<T, D, false><<<grid, THREADS, smem, s>>>(p, per_block);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_qk_norm_rope(const RopeParams& p, bool bf16, int D, bool interleaved, cudaStream_t s) {
  if (bf16) return D == 32 ? launch<__nv_bfloat16, 32>(p, interleaved, s) : D == 64 ? launch<__nv_bfloat16, 64>(p, interleaved, s) : launch<__nv_bfloat16, 128>(p, interleaved, s);
  return D == 32 ? launch<float, 32>(p, interleaved, s) : D == 64 ? launch<float, 64>(p, interleaved, s) : launch<float, 128>(p, interleaved, s);
}

}  // namespace tok
}  // namespace tt

// Queries' and keys' RMS norm per head and position rotation, one pass (tt_qk_norm_rope).
//
//   y = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> s * (a cos t - b sin t, b cos t + a sin t),  t = position * inv_freq[i]
//
// Bound by memory: every row is read and written once.  A row of D elements belongs to D / 8 lanes with eight elements each, so a row's
// sum of squares is a butterfly over at most 16 lanes and both elements of a pair sit in one lane: with the halves layout a
// lane below rot / 8 holds elements 4l..4l+3 and their partners rot / 2 further on, with the interleaved layout 8l..8l+7.
// A token's lanes go through its heads, queries then keys: the four angles of a lane are worked out once and stay in registers, as do
// the weights of a side; a few rows are in flight together, and nothing is shared between lanes but the sums.
// (Rows of all heads spread over the lanes, with the angles of a step shared through shared memory, took three times the
// instructions, most of them for addresses, and 43 to 57 us for eight maps of 14400 tokens.)
// Eight maps of 14400 tokens of 4 + 4 heads of 64: 35.3 us, 5.2 TB/s, 80 % of a plain copy's rate; eight tokens: 3.1 us, a launch.
// The angle is reduced in 64 bits (turns = position * inv_freq / 2 pi, less the nearest whole number): at position 5e6 a
// product of 32 bits would be off by 0.3 radians.
#include "tokens.h"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int THREADS = 128;

// Eight elements of a row as they lie in memory, and as pairs: lo[j] is turned with hi[j].  Runs: one of eight elements where pairs are
// neighbours, else one of lo's and one of hi's.
template <typename T, bool INTERLEAVED>
struct Eight;
template <bool INTERLEAVED>
struct Eight<float, INTERLEAVED> {
  float4 v[2];
  __device__ __forceinline__ void load(const float* p, int gap) {
    v[0] = *reinterpret_cast<const float4*>(p);
    v[1] = *reinterpret_cast<const float4*>(p + gap);
  }
  __device__ __forceinline__ void get(Two (&lo)[2], Two (&hi)[2]) const {
    if (INTERLEAVED) {
      lo[0] = pack2(v[0].x, v[0].z); lo[1] = pack2(v[1].x, v[1].z);
      hi[0] = pack2(v[0].y, v[0].w); hi[1] = pack2(v[1].y, v[1].w);
    } else {
      lo[0] = pack2(v[0].x, v[0].y); lo[1] = pack2(v[0].z, v[0].w);
      hi[0] = pack2(v[1].x, v[1].y); hi[1] = pack2(v[1].z, v[1].w);
    }
  }
  static __device__ __forceinline__ void store(float* p, int gap, const Two (&lo)[2], const Two (&hi)[2]) {
    float a[4], e[4];
    unpack2(lo[0], a[0], a[1]); unpack2(lo[1], a[2], a[3]); unpack2(hi[0], e[0], e[1]); unpack2(hi[1], e[2], e[3]);
    *reinterpret_cast<float4*>(p) = INTERLEAVED ? make_float4(a[0], e[0], a[1], e[1]) : make_float4(a[0], a[1], a[2], a[3]);
    *reinterpret_cast<float4*>(p + gap) = INTERLEAVED ? make_float4(a[2], e[2], a[3], e[3]) : make_float4(e[0], e[1], e[2], e[3]);
  }
};
__device__ __forceinline__ float low_of(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_of(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
template <bool INTERLEAVED>
struct Eight<__nv_bfloat16, INTERLEAVED> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int gap) {
    if (INTERLEAVED) {
      v = *reinterpret_cast<const uint4*>(p);
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(p), e = *reinterpret_cast<const uint2*>(p + gap);
      v = make_uint4(a.x, a.y, e.x, e.y);
    }
  }
  __device__ __forceinline__ void get(Two (&lo)[2], Two (&hi)[2]) const {
    if (INTERLEAVED) {
      lo[0] = pack2(low_of(v.x), low_of(v.y)); lo[1] = pack2(low_of(v.z), low_of(v.w));
      hi[0] = pack2(high_of(v.x), high_of(v.y)); hi[1] = pack2(high_of(v.z), high_of(v.w));
    } else {
      lo[0] = pack2(low_of(v.x), high_of(v.x)); lo[1] = pack2(low_of(v.y), high_of(v.y));
      hi[0] = pack2(low_of(v.z), high_of(v.z)); hi[1] = pack2(low_of(v.w), high_of(v.w));
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, int gap, const Two (&lo)[2], const Two (&hi)[2]) {
    float a[4], e[4];
    unpack2(lo[0], a[0], a[1]); unpack2(lo[1], a[2], a[3]); unpack2(hi[0], e[0], e[1]); unpack2(hi[1], e[2], e[3]);
    if (INTERLEAVED) {
      *reinterpret_cast<uint4*>(p) = make_uint4(tc::pack_bf16(a[0], e[0]), tc::pack_bf16(a[1], e[1]), tc::pack_bf16(a[2], e[2]), tc::pack_bf16(a[3], e[3]));
    } else {
      *reinterpret_cast<uint2*>(p) = make_uint2(tc::pack_bf16(a[0], a[1]), tc::pack_bf16(a[2], a[3]));
      *reinterpret_cast<uint2*>(p + gap) = make_uint2(tc::pack_bf16(e[0], e[1]), tc::pack_bf16(e[2], e[3]));
    }
  }
};

// Cosine and sine of a turn (|turns| <= 1/2).  For bf16 results the special-function unit's are far inside the result's rounding (2^-20
// against 2^-9); fp32 results take the full-precision functions.
template <typename T>
__device__ __forceinline__ void turn(float turns, float& cs, float& sn) {
  if constexpr (sizeof(T) == 2) {
    const float x = turns * 6.283185307179586f;
    cs = __cosf(x);
    sn = __sinf(x);
  } else {
    sincospif(2.f * turns, &sn, &cs);
  }
}

// U: rows of a lane and side in flight; split: heads of either side to a block (grid z: the runs of heads)
template <typename T, int D, bool INTERLEAVED, int U>
__global__ void __launch_bounds__(THREADS) qk_norm_rope_kernel(const __grid_constant__ RopeParams p, int split) {
  constexpr int LANES = D / 8;                      // to a token
  const int b = blockIdx.y;
  const int n = clamp_length(p.lengths, b, p.tokens);
  const int token = (int)blockIdx.x * (THREADS / LANES) + (int)threadIdx.x / LANES, lane = threadIdx.x % LANES;
  if ((int)blockIdx.x * (THREADS / LANES) + ((int)threadIdx.x & ~31) / LANES >= n) return;      // the whole warp
  const bool here = token < n;
  const int half = p.rot >> 1;
  const bool turned = lane * 8 < p.rot, norm = p.norm != 0;
  // this lane's elements: 4 at `from` and 4 at `from + gap`; pairs 4 lane .. 4 lane + 3
  const int from = !INTERLEAVED && turned ? lane * 4 : lane * 8, gap = !INTERLEAVED && turned ? half : 4;
  // the first rows of both sides are on their way while the angles are worked out
  Eight<T, INTERLEAVED> next[2][U];
  const T* src[2];
  auto load = [&](int side, int h, int h1) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h + u < h1) {
        if (here) next[side][u].load(src[side], gap);
        src[side] += p.x[side].h;
      }
  };
  const int h0 = (int)blockIdx.z * split;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    src[side] = reinterpret_cast<const T*>(p.x[side].p) + b * p.x[side].b + token * p.x[side].t + h0 * p.x[side].h + from;
    load(side, h0, min(p.heads[side], h0 + split));
  }
  Two c2[2], s2[2];
  if (turned) {
    const double pos = here ? (double)p.positions[b * p.pos_stride + token] * 0.15915494309189533577 : 0.0;
    float cs[4], sn[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double turns = pos * p.inv_freq[4 * lane + j];
      turn<T>((float)(turns - rint(turns)), cs[j], sn[j]);
    }
    const float g = p.rot_scale;
    c2[0] = pack2(cs[0] * g, cs[1] * g); c2[1] = pack2(cs[2] * g, cs[3] * g);
    s2[0] = pack2(sn[0] * g, sn[1] * g); s2[1] = pack2(sn[2] * g, sn[3] * g);
  }
  const float eps = p.eps;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const int h1 = min(p.heads[side], h0 + split);
    if (h0 >= h1) continue;
    const int64_t y_head = p.y[side].h;
    T* dst = reinterpret_cast<T*>(p.y[side].p) + b * p.y[side].b + token * p.y[side].t + h0 * y_head + from;
    Two wl[2], wh[2];
    if (norm) {
      const float* w = p.weight[side];
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = w ? __ldg(w + from + (j < 4 ? j : gap + j - 4)) : 1.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        wl[j] = INTERLEAVED ? pack2(f[4 * j], f[4 * j + 2]) : pack2(f[2 * j], f[2 * j + 1]);
        wh[j] = INTERLEAVED ? pack2(f[4 * j + 1], f[4 * j + 3]) : pack2(f[4 + 2 * j], f[4 + 2 * j + 1]);
      }
    }
    for (int h = h0; h < h1; h += U) {
      Eight<T, INTERLEAVED> a[U];
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] = next[side][u];
      load(side, h + U, h1);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u >= h1) break;
        Two lo[2], hi[2];
        a[u].get(lo, hi);
        if (norm) {
          const Two sq = fma2_of(lo[0], lo[0], fma2_of(lo[1], lo[1], fma2_of(hi[0], hi[0], mul2_of(hi[1], hi[1]))));
          float q, q1;
          unpack2(sq, q, q1);
          q += q1;
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, o);
          const float inv = rsqrtf(fmaf(q, 1.f / D, eps));
          const Two inv2 = pack2(inv, inv);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            lo[j] = mul2_of(mul2_of(lo[j], inv2), wl[j]);
            hi[j] = mul2_of(mul2_of(hi[j], inv2), wh[j]);
          }
        }
        if (turned) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const Two x = lo[j];
            lo[j] = sub2_of(mul2_of(x, c2[j]), mul2_of(hi[j], s2[j]));
            hi[j] = fma2_of(x, s2[j], mul2_of(hi[j], c2[j]));
          }
        }
        if (here) Eight<T, INTERLEAVED>::store(dst, gap, lo, hi);
        dst += y_head;
      }
    }
  }
}

template <typename T, int D, bool INTERLEAVED>
cudaError_t launch(const RopeParams& p, cudaStream_t s) {
  const int heads = p.heads[0] > p.heads[1] ? p.heads[0] : p.heads[1];
  const int64_t blocks = ((int64_t)p.tokens + THREADS / (D / 8) - 1) / (THREADS / (D / 8));
  // One row a side in flight where there is but one, or where all heads side by side do not fill the device (eight tokens of 4 + 4 heads:
  // 3.1 us, with two 3.6); else two (eight maps of 14400 tokens of 4 + 4 heads: 34.8 us, with one 42.8, with four 39.1).
  if (heads == 1 || blocks * p.batch * heads < 4 * PLAN_SMS) {
    qk_norm_rope_kernel<T, D, INTERLEAVED, 1><<<dim3((unsigned)blocks, (unsigned)p.batch, (unsigned)heads), THREADS, 0, s>>>(p, 1);
  } else {
    // a token's heads over several blocks where the tokens alone do not fill the device
    int split = heads;
    while (split > 2 && blocks * p.batch * ((heads + split - 1) / split) < 4 * PLAN_SMS) split = (split + 1) / 2;
    qk_norm_rope_kernel<T, D, INTERLEAVED, 2><<<dim3((unsigned)blocks, (unsigned)p.batch, (unsigned)((heads + split - 1) / split)), THREADS, 0, s>>>(p, split);
  }
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const RopeParams& p, bool interleaved, cudaStream_t s) {
  return interleaved ? launch<T, D, true>(p, s) : launch<T, D, false>(p, s);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const RopeParams& p, bool bf16, int D, bool interleaved, cudaStream_t s) {
  if (bf16) return D == 32 ? launch<__nv_bfloat16, 32>(p, interleaved, s) : D == 64 ? launch<__nv_bfloat16, 64>(p, interleaved, s) : launch<__nv_bfloat16, 128>(p, interleaved, s);
  return D == 32 ? launch<float, 32>(p, interleaved, s) : D == 64 ? launch<float, 64>(p, interleaved, s) : launch<float, 128>(p, interleaved, s);
}

}  // namespace tok
}  // namespace tt

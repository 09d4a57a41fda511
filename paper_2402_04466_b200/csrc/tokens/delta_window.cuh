// What depends on no state of a window of the gated delta rule.
//
// With G_i the sum of log_decay up to and including token i of the window, a window's corrections u_i solve (1 + A) U = R, A_ij = beta_i e^(G_i - G_j) (k_i . k_j) for j < i, and
// out reads them with the weights P_ij = scale e^(G_i - G_j) (q_i . k_j), j <= i.  Four warps take a window: A and P by products of 16 rows to a warp, the
// inverses of both diagonal blocks of 16 by substitution, a column to a lane, and the block below them as -T_11 A_10 T_00, by products again.  All of it counts with
// fp32's bits: operands that are not bf16 to begin with are cut into three bf16 terms.  (P of bf16 calls: 16 bits.)
#pragma once

#include "delta_common.cuh"

namespace tt {
namespace tok {

// 2^x for x of 0 and below, as pair: to half a step of the result and little more, where exp2f is off by two.  By a Taylor polynomial of e^(y ln 2), |y| <= 1/2.
__device__ __forceinline__ float exp2_pair(float hi, float lo) {
  if (!(hi > -150.f)) return hi == hi ? 0.f : hi;
  const float whole = rintf(hi), y = ((hi - whole) + lo) * 0.693147181f;
  float f = 1.f / 5040.f;
  f = fmaf(f, y, 1.f / 720.f);
  f = fmaf(f, y, 1.f / 120.f);
  f = fmaf(f, y, 1.f / 24.f);
  f = fmaf(f, y, 1.f / 6.f);
  f = fmaf(f, y, 0.5f);
  f = fmaf(f, y, 1.f);
  f = fmaf(f, y, 1.f);
  return scalbnf(f, (int)whole);
}
// an 8 x 8 block of pairs' terms, rows for columns
__device__ __forceinline__ uint32_t transposed(uint32_t u) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(u));
  return r;
}
__device__ __forceinline__ float fade_of(float2 to, float2 from) { return exp2_fast((to.x - from.x) + (to.y - from.y)); }

template <typename T, int D>
struct DeltaWindow {
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3, SEEN = sizeof(T) == 2 ? 2 : 3;
  static constexpr int C = DELTA_C, TT = DELTA_TT, TK = DELTA_TK, KS = D / 16, KP = D + 8, AP = C + 4, TILE = C * KP;
  struct Room {
    float A[C * AP];             // A, then its inverse
    float2 sums[C];              // log2(e) G as a pair of floats: what counts are differences of far larger sums
    float betas[C];
  };
  // ks and qs: [term][C][KP], there behind ready(), where the four warps meet as in meet(); decay and beta: of the first warp's lanes' tokens, 0 behind the last
  template <typename Ready, typename Meet>
  static __device__ __forceinline__ void prepare(DeltaRecord<SEEN>& record, Room& room, const __nv_bfloat16* ks, const __nv_bfloat16* qs, float decay, float beta, float scale, int warp, int lane,
                                                 Ready ready, Meet meet);
};

template <typename T, int D>
template <typename Ready, typename Meet>
__device__ __forceinline__ void DeltaWindow<T, D>::prepare(DeltaRecord<SEEN>& record, Room& room, const __nv_bfloat16* ks, const __nv_bfloat16* qs, float decay, float beta, float scale, int warp,
                                                           int lane, Ready ready, Meet meet) {
  const int g = lane >> 2, t = lane & 3;
  float* A = room.A;
  float2* sums = room.sums;
  float* betas = room.betas;
  if (warp == 0) {
    // -infinity: all of it, like -10^5
    const float mine = decay < -1e5f ? -1e5f : decay;
    float hi = mine * 1.44269504f, lo = fmaf(mine, 1.44269504f, -hi) + mine * 1.92596299e-8f;      // log2(e) to 48 bits
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const float x = __shfl_up_sync(0xffffffffu, hi, d), y = __shfl_up_sync(0xffffffffu, lo, d);
      // the sum of two pairs: that of the first floats, and what it lost (Knuth's two-sum)
      const float sum = hi + x, back = sum - hi, lost = (hi - (sum - back)) + (x - back), rest = lost + (lo + y);
      const float first = sum + rest;
      if (lane >= d) {
        lo = rest - (first - sum);
        hi = first;
      }
    }
    const float2 all = make_float2(__shfl_sync(0xffffffffu, hi, 31), __shfl_sync(0xffffffffu, lo, 31));
    sums[lane] = make_float2(hi, lo);
    betas[lane] = beta;
    record.beta[lane] = beta;
    record.up[lane] = exp2f(hi + lo);
    record.down[lane] = exp2f((all.x - hi) + (all.y - lo));
    // the one factor that a state meets again and again: its error would add up
    if (lane == 31) record.whole = exp2_pair(hi, lo);
  }
  ready();
  // 16 rows to a warp: the first two take A, the others P, in columns up to the diagonal
  {
    const int strip = 1 - (warp & 1);
    const bool keys = warp < 2;
    const __nv_bfloat16* left = keys ? ks : qs;
    float acc[TT][4];
#pragma unroll
    for (int i = 0; i < TT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll 2
    for (int x = 0; x < KS; ++x) {
      uint32_t a[TERMS][4];
#pragma unroll
      for (int i = 0; i < TERMS; ++i) ldmatrix4<false>(a[i], smem_u32(left + i * TILE + (16 * strip + (lane & 15)) * KP + x * 16 + (lane >> 4) * 8));
#pragma unroll
      for (int c = 0; c < TT; c += 2)
        if (c <= 2 * strip) {
          uint32_t one[TERMS][2], two[TERMS][2];
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            uint32_t f[4];
            ldmatrix4<false>(f, smem_u32(ks + e * TILE + (8 * c + (lane & 7) + 8 * (lane >> 4)) * KP + x * 16 + ((lane >> 3) & 1) * 8));
            one[e][0] = f[0]; one[e][1] = f[1]; two[e][0] = f[2]; two[e][1] = f[3];
          }
          product(acc[c], a, one);
          product(acc[c + 1], a, two);
        }
    }
    const int i0 = 16 * strip + g;
    const float2 to[2] = {sums[i0], sums[i0 + 8]};
    const float gains[2] = {keys ? betas[i0] : scale, keys ? betas[i0 + 8] : scale};
    // the weights' registers: rows i0 of an accumulator are columns of the second operand
    uint32_t terms[2][TT][3];
    float odd = 0.f;
#pragma unroll
    for (int c = 0; c < TT; ++c)
      if (c < 2 * strip + 2) {
        const int j = 8 * c + 2 * t;
        const float2 from[2] = {sums[j], sums[j + 1]};
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = i0 + 8 * r;
          float f[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            f[x] = gains[r] * fade_of(to[r], from[x]) * acc[c][2 * r + x];
            if (keys ? j + x >= i : j + x > i) f[x] = 0.f;
          }
          if (keys) *reinterpret_cast<float2*>(A + i * AP + j) = make_float2(f[0], f[1]);
          else {
            cut(f[0], f[1], terms[r][c]);
            odd = fmaf(f[0], 0.f, fmaf(f[1], 0.f, odd));
          }
        }
      }
    if (!keys) {
      // q_i . k_j may pass what 32 bits hold where u_j or the decay between is 0 and out sees nothing of it.  A NaN in place of a beta makes the chain take the window token by token.
      if (__any_sync(0xffffffffu, odd != 0.f) && lane == 0) record.beta[16 * strip] = NAN;
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int x = 0; x < TK; ++x)
          if (x <= strip)
#pragma unroll
            for (int e = 0; e < SEEN; ++e)
              *reinterpret_cast<uint2*>(record.weights[delta_place(2 * strip + r, x)][e][lane]) = make_uint2(terms[r][2 * x][e], terms[r][2 * x + 1][e]);
    }
  }
  meet();
  auto put = [&](int tile, int x, int e, uint32_t b0, uint32_t b1) { *reinterpret_cast<uint2*>(record.inverse[delta_place(tile, x)][e][lane]) = make_uint2(b0, b1); };
  // the two blocks of 16 on the diagonal, a column to a lane
  float* block = A + (warp & 1) * 16 * (AP + 1);
  if (warp < 2) {
    const int j = lane & 15;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float a[16];
#pragma unroll
      for (int m = 0; m < i; m += 4) {
        const float4 f = *reinterpret_cast<const float4*>(block + i * AP + m);
        a[m] = f.x; a[m + 1] = f.y; a[m + 2] = f.z; a[m + 3] = f.w;
      }
      float sum = i == j ? 1.f : 0.f, other = 0.f;      // two chains
#pragma unroll
      for (int m = 0; m < i; ++m)
        if (m & 1) other = fmaf(-a[m], x[m], other);
        else sum = fmaf(-a[m], x[m], sum);
      x[i] = sum + other;
    }
    __syncwarp();
    if (lane < 16)
#pragma unroll
      for (int i = 0; i < 16; ++i) block[i * AP + j] = x[i];
  }
  meet();
  if (warp < 2) {
    // as the second operand's registers of U's product
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t terms[2][3];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 f = *reinterpret_cast<const float2*>(block + (8 * i + g) * AP + 8 * e + 2 * t);
        cut(f.x, f.y, terms[e]);
      }
#pragma unroll
      for (int e = 0; e < 3; ++e) put(2 * warp + i, warp, e, terms[0][e], terms[1][e]);
    }
  } else {
    // the block below, -T_11 A_10 T_00, transposed as the chain is: (T_00^T A_10^T) T_11^T, of which either warp takes eight rows of T
    uint32_t a[3][4], f[2][3][2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t terms[3];
      const float* from = A + (2 * t + 8 * (e >> 1)) * AP + g + 8 * (e & 1);
      cut(from[0], from[AP], terms);
#pragma unroll
      for (int c = 0; c < 3; ++c) a[c][e] = terms[c];
    }
    auto second = [&](uint32_t (&to)[3][2], const float* rows) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint32_t terms[3];
        const float2 x = *reinterpret_cast<const float2*>(rows + g * AP + 8 * e + 2 * t);
        cut(x.x, x.y, terms);
#pragma unroll
        for (int c = 0; c < 3; ++c) to[c][e] = terms[c];
      }
    };
    float sums[2][3][4] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      second(f[i], A + (16 + 8 * i) * AP);
      product_apart(sums[i], a, f[i]);
    }
    second(f[0], A + (16 + 8 * (warp - 2)) * AP + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float (&x)[3][4] = sums[e >> 1];
      const int c = 2 * (e & 1);
      uint32_t terms[3];
      cut(-(x[0][c] + (x[1][c] + x[2][c])), -(x[0][c + 1] + (x[1][c + 1] + x[2][c + 1])), terms);
#pragma unroll
      for (int z = 0; z < 3; ++z) a[z][e] = terms[z];
    }
    float last[3][4] = {};
    product_apart(last, a, f[0]);
    uint32_t low[3], high[3];
    cut(last[0][0] + (last[1][0] + last[2][0]), last[0][1] + (last[1][1] + last[2][1]), low);
    cut(last[0][2] + (last[1][2] + last[2][2]), last[0][3] + (last[1][3] + last[2][3]), high);
#pragma unroll
    for (int e = 0; e < 3; ++e) put(warp, 0, e, transposed(low[e]), transposed(high[e]));
  }
}

}  // namespace tok
}  // namespace tt

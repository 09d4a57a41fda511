// Cross attention of few bf16 queries, and of masked ones (tt_cross_attention): keys and values straight from memory into registers.
//
// With a handful of rows per key and value head (seven tools, times the heads of a group) the operator is bound by reading K and V once,
// 4 D bytes a key for 4 D operations a row.  A warp takes 16 rows x 16 keys at a time with m16n8k16 products.  Nothing goes through
// shared memory: the order of a product's inner index is free as long as both operands agree, and so is the order of its columns.
//   scores:  lane (g, t) = (lane / 4, lane % 4) supplies key g's elements t D/4 .. (t+1) D/4, one run of 16-byte loads, and the
//            queries' fragments are laid out in the same order;
//   sums:    it supplies elements g D/8 .. (g+1) D/8 of keys 2t, 2t+1, 2t+8, 2t+9, again 16-byte loads; column n of product i is
//            element n D/8 + i, and two keys' elements are paired by byte permutes.
// Weights are split into two bf16 terms, so that they count with 16 bits and more: the second product is not what the time goes to.
// Every warp runs through its own keys with its own maximum, which only moves when a weight would pass 2^8; warps join through shared
// memory, blocks of split keys through cross_join_kernel.
#include "tokens.h"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

template <int D>
struct Few {
  static constexpr int WARPS = D == 128 ? 4 : 8;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int KS = D / 16;          // steps of the scores' inner index
  static constexpr int NT = D / 8;           // column products of the sums
  static constexpr int KQ = D / 32;          // 16-byte loads of a key's quarter
  static constexpr int OP = D + 4;           // pitch of the joint sums
};

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What a warp holds of 16 keys.
template <int D>
struct Keys {
  uint4 k[2][Few<D>::KQ];        // keys g and 8 + g, elements t D/4 ..
  uint32_t v[4][D / 16];         // keys 2t, 2t+1, 2t+8, 2t+9, elements g D/8 ..
};

template <int D>
__device__ __forceinline__ void fetch(Keys<D>& r, const __nv_bfloat16* k, const __nv_bfloat16* v, int64_t kt, int64_t vt, int j, int j1, int g, int t) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int key = j + 8 * i + g;
#pragma unroll
    for (int c = 0; c < Few<D>::KQ; ++c)
      r.k[i][c] = key < j1 ? __ldg(reinterpret_cast<const uint4*>(k + key * kt + t * (D / 4)) + c) : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = j + 2 * t + (i & 1) + (i >> 1) * 8;
    const __nv_bfloat16* at = v + key * vt + g * (D / 8);
    if constexpr (D == 32) {
      const uint2 u = key < j1 ? __ldg(reinterpret_cast<const uint2*>(at)) : make_uint2(0u, 0u);
      r.v[i][0] = u.x; r.v[i][1] = u.y;
    } else {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const uint4 u = key < j1 ? __ldg(reinterpret_cast<const uint4*>(at) + c) : make_uint4(0u, 0u, 0u, 0u);
        r.v[i][4 * c] = u.x; r.v[i][4 * c + 1] = u.y; r.v[i][4 * c + 2] = u.z; r.v[i][4 * c + 3] = u.w;
      }
    }
  }
}

template <int D, bool MASK>
__global__ void __launch_bounds__(Few<D>::THREADS, 2) cross_few_kernel(const __grid_constant__ CrossParams p) {
  using F = Few<D>;
  __shared__ float s_o[F::WARPS][16][F::OP];
  __shared__ float2 s_ml[F::WARPS][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x % p.splits, row0 = (int)(blockIdx.x / p.splits) * 16, hk = blockIdx.y, b = blockIdx.z;
  const int rows = clamp_length(p.q_lengths, b, p.q_tokens) * p.group;
  const int keys = clamp_length(p.kv_lengths, b, p.kv_tokens);
  const int j0 = split * p.split_keys, j1 = min(keys, j0 + p.split_keys);
  if (row0 >= rows || (split > 0 && j0 >= keys)) return;
  const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v.p) + b * p.v.b + hk * p.v.h;

  Keys<D> cur, next;
  int j = j0 + warp * 16;
  fetch<D>(cur, k, v, p.k.t, p.v.t, j, j1, g, t);

  // queries: rows g and g + 8, elements t D/4 ..; step s of the inner index takes elements 4s .. 4s+3 of each lane's run
  uint32_t q[F::KS][4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row0 + g + 8 * i;
    const uint4* src = reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.q.p) + b * p.q.b + (int64_t)(row / p.group) * p.q.t +
                                                      ((int64_t)hk * p.group + row % p.group) * p.q.h + t * (D / 4));
#pragma unroll
    for (int c = 0; c < F::KQ; ++c) {
      const uint4 u = row < rows ? __ldg(src + c) : make_uint4(0u, 0u, 0u, 0u);
      q[2 * c][i] = u.x; q[2 * c][2 + i] = u.y;
      q[2 * c + 1][i] = u.z; q[2 * c + 1][2 + i] = u.w;
    }
  }
  const uint8_t* mask[2];
  if (MASK) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + g + 8 * i;
      mask[i] = p.mask + b * p.mask_b + (int64_t)((row < rows ? row : row0) / p.group) * p.mask_q;
    }
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float o[F::NT][4];
#pragma unroll
  for (int i = 0; i < F::NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  const float c = p.scale_log2;

  for (; j < j1; j += 16 * F::WARPS) {
    fetch<D>(next, k, v, p.k.t, p.v.t, j + 16 * F::WARPS, j1, g, t);
    float s[2][4];                             // keys 2t, 2t+1 (+ 8 x first index) for rows g, g + 8
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
      for (int x = 0; x < F::KQ; ++x) {
        mma16816(s[i], q[2 * x], cur.k[i][x].x, cur.k[i][x].y);
        mma16816(s[i], q[2 * x + 1], cur.k[i][x].z, cur.k[i][x].w);
      }
    }
    bool seen[2][4];
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int key = j + 8 * i + 2 * t + (x & 1);
        seen[i][x] = key < j1;
        if (MASK) seen[i][x] = seen[i][x] && mask[x >> 1][key];
        s[i][x] *= c;
        if (seen[i][x]) top[x >> 1] = fmaxf(top[x >> 1], s[i][x]);
      }
    if (__any_sync(0xffffffffu, top[0] > m[0] + 8.f || top[1] > m[1] + 8.f)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float now = top[r];
        now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 1));
        now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 2));
        now = fmaxf(now, m[r]);
        const float fade = now == -INFINITY ? 1.f : exp2_fast(m[r] - now);
        m[r] = now;
        l[r] *= fade;
#pragma unroll
        for (int i = 0; i < F::NT; ++i) { o[i][2 * r] *= fade; o[i][2 * r + 1] *= fade; }
      }
    }
    const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
    float w[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        w[i][x] = seen[i][x] ? exp2_fast(s[i][x] - base[x >> 1]) : -0.f;      // the sign marks what is not seen
        l[x >> 1] += w[i][x];
      }
    bool careful = false;
    if (MASK) {
      // an infinity or NaN among the values: bf16 with all exponent bits set
      uint32_t odd = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int x = 0; x < D / 16; ++x) odd |= __vcmpeq2(cur.v[i][x] & 0x7F807F80u, 0x7F807F80u);
      careful = __any_sync(0xffffffffu, odd != 0u);
    }
    if (!MASK || !careful) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float a = w[i][2 * r], e = w[i][2 * r + 1];
          const uint32_t u = pack_bf16(a, e);
          hi[2 * i + r] = u;
          lo[2 * i + r] = pack_bf16(a - __uint_as_float(u << 16), e - __uint_as_float(u & 0xFFFF0000u));
        }
#pragma unroll
      for (int x = 0; x < D / 16; ++x) {
        // elements 2x and 2x + 1 of the lane's run: one column product each
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t sel = e ? 0x7632u : 0x5410u;
          const uint32_t b0 = __byte_perm(cur.v[0][x], cur.v[1][x], sel), b1 = __byte_perm(cur.v[2][x], cur.v[3][x], sel);
          mma16816(o[2 * x + e], hi, b0, b1);
          mma16816(o[2 * x + e], lo, b0, b1);
        }
      }
    } else {
      // one key at a time, left out of the rows that do not see it
      for (int kk = 0; kk < 16 && j + kk < j1; ++kk) {
        const int from = (lane & ~3) | ((kk & 7) >> 1);
        float mine[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float pick = kk < 8 ? (kk & 1 ? w[0][2 * r + 1] : w[0][2 * r]) : (kk & 1 ? w[1][2 * r + 1] : w[1][2 * r]);
          mine[r] = __shfl_sync(0xffffffffu, pick, from);
        }
#pragma unroll
        for (int i = 0; i < F::NT; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float val = __bfloat162float(v[(int64_t)(j + kk) * p.v.t + (2 * t + x) * (D / 8) + i]);
            if (!signbit(mine[0])) o[i][x] = fmaf(mine[0], val, o[i][x]);
            if (!signbit(mine[1])) o[i][2 + x] = fmaf(mine[1], val, o[i][2 + x]);
          }
      }
    }
    cur = next;
  }

  // join the warps: row r of the tile, element d
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    if (t == 0) s_ml[warp][g + 8 * r] = make_float2(m[r], l[r]);
#pragma unroll
    for (int i = 0; i < F::NT; ++i) {
      s_o[warp][g + 8 * r][(2 * t) * (D / 8) + i] = o[i][2 * r];
      s_o[warp][g + 8 * r][(2 * t + 1) * (D / 8) + i] = o[i][2 * r + 1];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (D / 2); i += F::THREADS) {
    const int r = i / (D / 2), d = i % (D / 2) * 2, row = row0 + r;
    if (row >= rows) break;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) top = fmaxf(top, s_ml[x][r].x);
    const float base = top == -INFINITY ? 0.f : top;
    float a = 0.f, e = 0.f, total = 0.f;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) {
      const float2 ml = s_ml[x][r];
      const float f = exp2_fast(ml.x - base);
      total = fmaf(f, ml.y, total);
      a = fmaf(f, s_o[x][r][d], a);
      e = fmaf(f, s_o[x][r][d + 1], e);
    }
    if (p.splits > 1) {
      const Part to = part_of(p, D, b, hk, row);
      if (d == 0) to.stat[split] = make_float2(top, total);
      *reinterpret_cast<float2*>(to.sum + (int64_t)split * D + d) = make_float2(a, e);
    } else {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + ((int64_t)hk * p.group + row % p.group) * p.o.h;
      *reinterpret_cast<uint32_t*>(dst + d) = pack_bf16(a * inv, e * inv);
    }
  }
}

template <int D, bool MASK>
cudaError_t launch(const CrossParams& p, cudaStream_t s) {
  const int64_t tiles = ((int64_t)p.q_tokens * p.group + 15) / 16;
  cross_few_kernel<D, MASK><<<dim3((unsigned)(tiles * p.splits), (unsigned)(p.heads / p.group), (unsigned)p.batch), Few<D>::THREADS, 0, s>>>(p);
  return cudaGetLastError();
}
template <int D>
cudaError_t launch(const CrossParams& p, cudaStream_t s) {
  return p.mask ? launch<D, true>(p, s) : launch<D, false>(p, s);
}

}  // namespace

cudaError_t launch_cross_few(const CrossParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<32>(p, s) : D == 64 ? launch<64>(p, s) : launch<128>(p, s);
}

}  // namespace tok
}  // namespace tt

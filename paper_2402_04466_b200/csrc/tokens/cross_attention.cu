// Cross attention of fp32 operands, on the fp32 units (tt_cross_attention), the join of split keys, and the choice between the kernels.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = 2^(s_ij - m_i),  s_ij = scale * log2(e) * q_i k_j,  m_i the running maximum.
//
// One pass over the keys in tiles of 64.  The rows of a block's tile are queries x heads of one key and value head (row r: query
// r / group, head r % group), so that shared heads read K and V once.  Where the row tiles alone do not fill the device the keys
// are split over blocks, each leaves its sum, maximum and total, and cross_join_kernel joins them in order.
//
// Bound by what the fp32 units read from shared memory, a load of 16 bytes for four packed multiply-adds at most: 1023 queries of 2 heads of 32
// over one of keys and values on 4096 keys take 46.6 us, 1.1 GFLOP of products (15 us of the units alone) and 2 us of exponentials.  (Weights kept
// twice, as the pairs that the multiply-adds take: fewer instructions, more loads, 55 us.)
//
// Differential attention (MAPS = 2): scores of either half of a head's columns, weights of both maps side by side, every value read once for both: the same sizes 67.7 us (as two passes 90).
//
// A masked weight is kept as -0: it adds nothing to a finite value, and where a tile of V holds an infinity or NaN its sign
// tells the slow loop to leave it out.
#include "token_ptx.cuh"
#include "tokens.h"

namespace tt {
namespace tok {
namespace {

constexpr int THREADS = 256;           // 16 x 16
constexpr int BN = 64;                 // keys of a tile

template <int D, int BM, int MAPS>
struct Shape {
  static constexpr int A = BM / 16;                     // rows to a thread
  static constexpr int N = BN / 16;                     // keys to a thread
  static constexpr int E = D / 16;                      // columns to a thread
  static constexpr int QP = D + 4, PP = MAPS * BN + 4;   // weights of two maps lie side by side
  static constexpr int KV = BN * (QP + D);              // a tile's keys and values, of which two are in shared memory
  static constexpr size_t smem = sizeof(float) * (BM * QP + 2 * KV + BM * PP);
};

// 16 bytes to shared memory without waiting for them, or zeros
__device__ __forceinline__ void copy16(float* dst, const float* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ bool all_finite(float4 f) {
  return isfinite(f.x) && isfinite(f.y) && isfinite(f.z) && isfinite(f.w);
}

template <int D, int BM, int MAPS>
__global__ void __launch_bounds__(THREADS, MAPS == 2 && D == 32 && BM == 64 ? 2 : 0) cross_kernel(const __grid_constant__ ParamsOf<MAPS> p) {
  using S = Shape<D, BM, MAPS>;
  constexpr int A = S::A, N = S::N, E = S::E, QP = S::QP, PP = S::PP;
  extern __shared__ float4 raw[];
  float* qs = reinterpret_cast<float*>(raw);
  float* kv = qs + BM * QP;
  float* ps = kv + 2 * S::KV;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int split = blockIdx.x % p.splits, row0 = (int)(blockIdx.x / p.splits) * BM, hk = blockIdx.y, b = blockIdx.z;
  const int rows = clamp_length(p.q_lengths, b, p.q_tokens) * p.group;
  const int keys = clamp_length(p.kv_lengths, b, p.kv_tokens);
  const int j0 = split * p.split_keys, j1 = min(keys, j0 + p.split_keys);
  if (row0 >= rows || (split > 0 && j0 >= keys)) return;
  const float* q = reinterpret_cast<const float*>(p.q.p) + b * p.q.b + (int64_t)hk * p.group * p.q.h;
  const float* k = reinterpret_cast<const float*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const float* v = reinterpret_cast<const float*>(p.v.p) + b * p.v.b + hk * p.v.h;
  for (int i = threadIdx.x; i < BM * (D / 4); i += THREADS) {
    const int r = i / (D / 4), c = i % (D / 4) * 4;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row0 + r < rows) f = *reinterpret_cast<const float4*>(q + (int64_t)((row0 + r) / p.group) * p.q.t + (row0 + r) % p.group * p.q.h + c);
    *reinterpret_cast<float4*>(qs + r * QP + c) = f;
  }
  float m[MAPS][A], l[MAPS][A];
  Two o[MAPS][A][E / 2];               // pairs of neighbouring columns
#pragma unroll
  for (int w = 0; w < MAPS; ++w)
#pragma unroll
    for (int a = 0; a < A; ++a) {
      m[w][a] = -INFINITY;
      l[w][a] = 0.f;
#pragma unroll
      for (int c = 0; c < E / 2; ++c) o[w][a][c] = pack2(0.f, 0.f);
    }
  Two both[MAPS == 2 ? A : 1][MAPS == 2 ? E : 1];      // of two maps: a column's sums of either
  if (MAPS == 2)
#pragma unroll
    for (int a = 0; a < (MAPS == 2 ? A : 1); ++a)
#pragma unroll
      for (int c = 0; c < (MAPS == 2 ? E : 1); ++c) both[a][c] = pack2(0.f, 0.f);
  auto fetch = [&](int j, float* dst) {
    for (int i = threadIdx.x; i < BN * (D / 4); i += THREADS) {
      const int r = i / (D / 4), c = i % (D / 4) * 4;
      const bool there = j + r < j1;
      const int64_t at = there ? j + r : 0;
      copy16(dst + r * QP + c, k + at * p.k.t + c, there);
      copy16(dst + BN * QP + r * D + c, v + at * p.v.t + c, there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (j0 < j1) fetch(j0, kv);
  for (int j = j0; j < j1; j += BN) {
    const float* ks = kv + ((j - j0) / BN & 1) * S::KV;
    const float* vs = ks + BN * QP;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    bool odd = false;
    if (p.mask)
      for (int i = threadIdx.x; i < BN * (D / 4); i += THREADS) odd |= !all_finite(*reinterpret_cast<const float4*>(vs + i * 4));      // its own copies
    const bool careful = __syncthreads_or(odd) && p.mask;      // the tile is there, and the one before has been read: the next one takes its place
    if (j + BN < j1) fetch(j + BN, kv + ((j - j0) / BN + 1 & 1) * S::KV);
    float s[MAPS][A][N];
#pragma unroll
    for (int w = 0; w < MAPS; ++w) {
      Two acc[A][N];                   // even and odd elements
#pragma unroll
      for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < N; ++c) acc[a][c] = pack2(0.f, 0.f);
#pragma unroll 4
      for (int e = w * (D / MAPS); e < (w + 1) * (D / MAPS); e += 4) {
        ulonglong2 x[A], y[N];
#pragma unroll
        for (int a = 0; a < A; ++a) x[a] = *reinterpret_cast<const ulonglong2*>(qs + (ty + 16 * a) * QP + e);
#pragma unroll
        for (int c = 0; c < N; ++c) y[c] = *reinterpret_cast<const ulonglong2*>(ks + (tx + 16 * c) * QP + e);
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
          for (int c = 0; c < N; ++c) acc[a][c] = fma2_of(x[a].y, y[c].y, fma2_of(x[a].x, y[c].x, acc[a][c]));
      }
#pragma unroll
      for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < N; ++c) {
          float lo, hi;
          unpack2(acc[a][c], lo, hi);
          s[w][a][c] = lo + hi;
        }
    }
    const bool whole = !p.mask && j + BN <= j1;      // every key of the tile is seen by every row
#pragma unroll
    for (int a = 0; a < A; ++a) {
      bool seen[N];
#pragma unroll
      for (int c = 0; c < N; ++c) seen[c] = true;
      if (!whole) {
        const int row = row0 + ty + 16 * a;
        const uint8_t* mask = p.mask && row < rows ? p.mask + b * p.mask_b + (int64_t)(row / p.group) * p.mask_q + j : nullptr;
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const int at = tx + 16 * c;
          seen[c] = j + at < j1 && (!mask || mask[at]);
          if (!seen[c])
#pragma unroll
            for (int w = 0; w < MAPS; ++w) s[w][a][c] = -INFINITY;
        }
      }
      if constexpr (MAPS == 1) {
        float top = s[0][a][0];
#pragma unroll
        for (int c = 1; c < N; ++c) top = fmaxf(top, s[0][a][c]);
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
        top *= p.scale_log2;
        const float now = fmaxf(m[0][a], top), base = now == -INFINITY ? 0.f : now;
        const float fade = exp2_fast(m[0][a] - base);
        m[0][a] = now;
        float add = 0.f;
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const float weight = seen[c] ? exp2_fast(fmaf(s[0][a][c], p.scale_log2, -base)) : -0.f;
          add += weight;
          ps[(ty + 16 * a) * PP + tx + 16 * c] = weight;
        }
        l[0][a] = fmaf(l[0][a], fade, add);    // this thread's share of the keys
        const Two f2 = pack2(fade, fade);
#pragma unroll
        for (int c = 0; c < E / 2; ++c) o[0][a][c] = mul2_of(o[0][a][c], f2);
      } else {
        // The maxima only move when a weight would pass 2^8: sixteen threads to a row agree on them by four shuffles each.
        float top[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          top[w] = s[w][a][0];
#pragma unroll
          for (int c = 1; c < N; ++c) top[w] = fmaxf(top[w], s[w][a][c]);
          top[w] *= p.scale_log2;
        }
        if (__any_sync(0xFFFFFFFFu, top[0] > m[0][a] + 8.f || top[1] > m[1][a] + 8.f)) {
          float fade[2];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) top[w] = fmaxf(top[w], __shfl_xor_sync(0xFFFFFFFFu, top[w], x));
            const float now = fmaxf(m[w][a], top[w]);
            fade[w] = now == -INFINITY ? 1.f : exp2_fast(m[w][a] - now);
            m[w][a] = now;
            l[w][a] *= fade[w];
          }
          const Two f2 = pack2(fade[0], fade[1]);
#pragma unroll
          for (int c = 0; c < E; ++c) both[a][c] = mul2_of(both[a][c], f2);
        }
        const float base[2] = {m[0][a] == -INFINITY ? 0.f : m[0][a], m[1][a] == -INFINITY ? 0.f : m[1][a]};
#pragma unroll
        for (int c = 0; c < N; ++c) {
          float weight[2];
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            weight[w] = seen[c] ? exp2_fast(fmaf(s[w][a][c], p.scale_log2, -base[w])) : -0.f;
            l[w][a] += weight[w];
          }
          *reinterpret_cast<float2*>(ps + (ty + 16 * a) * PP + 2 * (tx + 16 * c)) = make_float2(weight[0], weight[1]);
        }
      }
    }
    __syncwarp();                      // a row's 16 threads are half a warp
    if constexpr (MAPS == 2) {
      // both maps' weights of two keys in one load, as the pairs that the multiply-adds take
      auto add_up = [&](auto some) {           // some: not every key of every row
#pragma unroll 2
        for (int i = 0; i < BN; i += 2) {
          Two y[2][E / 2], column[2][E];
          load_pairs<D>(vs + i * D, tx, y[0]);
          load_pairs<D>(vs + (i + 1) * D, tx, y[1]);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < E / 2; ++c) {
              float lo, hi;
              unpack2(y[k][c], lo, hi);
              column[k][2 * c] = pack2(lo, lo);
              column[k][2 * c + 1] = pack2(hi, hi);
            }
#pragma unroll
          for (int a = 0; a < A; ++a) {
            const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(ps + (ty + 16 * a) * PP + 2 * i);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const Two w2 = k == 0 ? x.x : x.y;
              if (!decltype(some)::value || (w2 >> 31 & 1) == 0)      // a weight of -0 is of a key that the row does not see
#pragma unroll
                for (int c = 0; c < E; ++c) both[a][c] = fma2_of(w2, column[k][c], both[a][c]);
            }
          }
        }
      };
      if (careful) add_up(std::true_type{});
      else add_up(std::false_type{});
    } else if (!careful) {
#pragma unroll 2
      for (int i = 0; i < BN; i += 4) {  // four keys: a row's weights in one load
        float4 row4[A];
#pragma unroll
        for (int a = 0; a < A; ++a) row4[a] = *reinterpret_cast<const float4*>(ps + (ty + 16 * a) * PP + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          Two y[E / 2];
          load_pairs<D>(vs + (i + k) * D, tx, y);
#pragma unroll
          for (int a = 0; a < A; ++a) {
            const float x = k == 0 ? row4[a].x : k == 1 ? row4[a].y : k == 2 ? row4[a].z : row4[a].w;
            const Two x2 = pack2(x, x);
#pragma unroll
            for (int c = 0; c < E / 2; ++c) o[0][a][c] = fma2_of(x2, y[c], o[0][a][c]);
          }
        }
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < BN; ++i) {
        Two y[E / 2];
        load_pairs<D>(vs + i * D, tx, y);
#pragma unroll
        for (int a = 0; a < A; ++a) {
          const float x = ps[(ty + 16 * a) * PP + i];
          if (!signbit(x))
#pragma unroll
            for (int c = 0; c < E / 2; ++c) o[0][a][c] = fma2_of(pack2(x, x), y[c], o[0][a][c]);
        }
      }
    }
  }
  if constexpr (MAPS == 2) {
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int c = 0; c < E / 2; ++c) {
        float x[2][2];
        unpack2(both[a][2 * c], x[0][0], x[1][0]);
        unpack2(both[a][2 * c + 1], x[0][1], x[1][1]);
        o[0][a][c] = pack2(x[0][0], x[0][1]);
        o[1][a][c] = pack2(x[1][0], x[1][1]);
      }
  }
  if (MAPS == 1 || p.splits > 1) {
#pragma unroll
    for (int w = 0; w < MAPS; ++w)
#pragma unroll
      for (int a = 0; a < A; ++a) {
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) l[w][a] += __shfl_xor_sync(0xFFFFFFFFu, l[w][a], x);
        const int row = row0 + ty + 16 * a;
        if (row >= rows) continue;
        const float inv = p.splits > 1 ? 1.f : l[w][a] == 0.f ? 0.f : 1.f / l[w][a];
        const Part to = part_of<MAPS>(p, D, b, hk, row, w);
        if (p.splits > 1 && tx == 0) to.stat[split] = make_float2(m[w][a], l[w][a]);
        float* dst = p.splits > 1 ? to.sum + (int64_t)split * D
                                  : reinterpret_cast<float*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + ((int64_t)hk * p.group + row % p.group) * p.o.h;
        const Two i2 = pack2(inv, inv);
#pragma unroll
        for (int c = 0; c < E / 2; ++c) *reinterpret_cast<Two*>(dst + (D == 32 ? 2 * tx : 4 * tx + (c & 1) * 2 + (c >> 1) * 64)) = mul2_of(o[w][a][c], i2);
      }
  }
  if constexpr (MAPS == 2) {
    if (p.splits == 1)
#pragma unroll
      for (int a = 0; a < A; ++a) {
        const int row = row0 + ty + 16 * a;      // the other half of the warp has another one
        const int head = hk * p.group + row % p.group;
        // both halves' heads, one behind the other: a whole warp works out either
        const float low = lambda_of(p.end, D / 2, __shfl_sync(0xFFFFFFFFu, head, 0)), high = lambda_of(p.end, D / 2, __shfl_sync(0xFFFFFFFFu, head, 16));
        const float lambda = threadIdx.x % 32 < 16 ? low : high;
        float inv[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
#pragma unroll
          for (int x = 8; x > 0; x >>= 1) l[w][a] += __shfl_xor_sync(0xFFFFFFFFu, l[w][a], x);
          inv[w] = l[w][a] == 0.f ? 0.f : 1.f / l[w][a];
        }
        const Two one = pack2(inv[0], inv[0]), two = pack2(-lambda * inv[1], -lambda * inv[1]);
        Two y[E / 2], sq = pack2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < E / 2; ++c) {
          y[c] = fma2_of(o[1][a][c], two, mul2_of(o[0][a][c], one));
          sq = fma2_of(y[c], y[c], sq);
        }
        float s0, s1;
        unpack2(sq, s0, s1);
        s0 += s1;
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) s0 += __shfl_xor_sync(0xFFFFFFFFu, s0, x);
        const float gain = row_gain<D>(p.end, s0);
        if (row >= rows) continue;
        float* dst = reinterpret_cast<float*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + (int64_t)head * p.o.h;
#pragma unroll
        for (int c = 0; c < E / 2; ++c) {
          const int d = D == 32 ? 2 * tx : 4 * tx + (c & 1) * 2 + (c >> 1) * 64;
          *reinterpret_cast<Two*>(dst + d) = mul2_of(y[c], pack2(gain * norm_weight(p.end, d), gain * norm_weight(p.end, d + 1)));
        }
      }
  }
}

// One warp per row: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
template <typename T, int D, int MAPS>
__global__ void __launch_bounds__(128) cross_join_kernel(const __grid_constant__ ParamsOf<MAPS> p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x % 32, row = (int)blockIdx.x * 4 + (int)threadIdx.x / 32, hk = blockIdx.y, b = blockIdx.z;
  if (row >= clamp_length(p.q_lengths, b, p.q_tokens) * p.group) return;
  const int keys = clamp_length(p.kv_lengths, b, p.kv_tokens);
  const int n = p.split_keys == 0 ? p.splits : keys > p.split_keys ? (keys + p.split_keys - 1) / p.split_keys : 1;
  float y[MAPS][E];
#pragma unroll
  for (int w = 0; w < MAPS; ++w) {
    const Part from = part_of<MAPS>(p, D, b, hk, row, w);
    float top = -INFINITY;
    for (int s = lane; s < n; s += 32) top = fmaxf(top, from.stat[s].x);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    if (top == -INFINITY) top = 0.f;
    float o[E] = {}, l = 0.f;
#pragma unroll 8                       // the loads of eight splits in flight together
    for (int s = 0; s < n; ++s) {
      const float2 st = from.stat[s];
      const float f = exp2f(st.x - top);
      l = fmaf(f, st.y, l);
#pragma unroll
      for (int c = 0; c < E; ++c) o[c] = fmaf(f, from.sum[(int64_t)s * D + lane * E + c], o[c]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int c = 0; c < E; ++c) y[w][c] = o[c] * inv;
  }
  const int head = hk * p.group + row % p.group;
  T* dst = reinterpret_cast<T*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + (int64_t)head * p.o.h;
  if constexpr (MAPS == 2) {
    const float lambda = lambda_of(p.end, D / 2, head);
    float squares = 0.f;
#pragma unroll
    for (int c = 0; c < E; ++c) {
      y[0][c] = fmaf(-lambda, y[1][c], y[0][c]);
      squares = fmaf(y[0][c], y[0][c], squares);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) squares += __shfl_xor_sync(0xFFFFFFFFu, squares, x);
    const float gain = row_gain<D>(p.end, squares);
#pragma unroll
    for (int c = 0; c < E; ++c) y[0][c] *= gain * norm_weight(p.end, lane * E + c);
  }
#pragma unroll
  for (int c = 0; c < E; ++c) dst[lane * E + c] = (T)y[0][c];
}

template <int D, int BM, int MAPS>
cudaError_t launch_scalar(const ParamsOf<MAPS>& p, cudaStream_t s) {
  const size_t smem = Shape<D, BM, MAPS>::smem;
  static OncePerContext once;
  cudaError_t e = once([&] { return cudaFuncSetAttribute(cross_kernel<D, BM, MAPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((int64_t)p.q_tokens * p.group + BM - 1) / BM;
  cross_kernel<D, BM, MAPS><<<dim3((unsigned)(tiles * p.splits), (unsigned)(p.heads / p.group), (unsigned)p.batch), THREADS, smem, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int D, int MAPS>
cudaError_t launch_typed(const ParamsOf<MAPS>& p, const CrossPlan& plan, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if constexpr (sizeof(T) == 2) e = launch_cross_few<MAPS>(p, D, plan.warps, s);
  else e = plan.rows == 16 ? launch_scalar<D, 16, MAPS>(p, s) : launch_scalar<D, 64, MAPS>(p, s);
  if (e != cudaSuccess || p.splits == 1) return e;
  const int64_t rows = (int64_t)p.q_tokens * p.group;
  cross_join_kernel<T, D, MAPS><<<dim3((unsigned)((rows + 3) / 4), (unsigned)(p.heads / p.group), (unsigned)p.batch), 128, 0, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int MAPS>
cudaError_t launch_typed(const ParamsOf<MAPS>& p, const CrossPlan& plan, int D, cudaStream_t s) {
  return D == 32 ? launch_typed<T, 32, MAPS>(p, plan, s) : D == 64 ? launch_typed<T, 64, MAPS>(p, plan, s) : launch_typed<T, 128, MAPS>(p, plan, s);
}

}  // namespace

CrossPlan cross_plan(int batch, int q_tokens, int kv_tokens, int heads, int group, int D, bool bf16, bool mask, int maps) {
  CrossPlan plan{};
  plan.splits = plan.cluster = 1;
  // The kernel for many queries takes work from half a million keys x tiles of 16 rows on.  Both measured around that, us with the one for few and the one for
  // many, heads of 32, 64, 128: 5 x 2 heads on 4800 keys, 128 queries (0.38 million) 18.0 17.2, 24.1 19.5, 41.5 26.6; 192 (0.58) 18.7 17.4, 24.7 21.6, 41.5 31.5;
  // one entry's 256 queries of 2 heads (0.15) 8.8 16.9, 10.5 21.6, 15.4 32.1; 700 (0.42) 18.2 17.5, 24.1 22.1, 40.9 34.8; 8 x 4 heads on 14400 keys, 65 queries
  // (2.3) 55.4 50.6, 81.5 52.6, 158 65.9.  So it is not taken too soon, and up to a third (heads of 64) or a half (128) too late where entries are several and
  // keys fewer than that.  (Masks are the other kernel's whatever the size; up to 64 queries leave three quarters of a tile of 256 rows empty.)
  // Of two maps (differential attention) the sums are twice as many, and a tile of the kernel for many has 128 queries: it takes work from 0.2 million on,
  // and 33 queries.  Measured in the same way: 5 x 2 heads on 4800 keys, 33 queries (0.14 million) 14.6 22.7, 16.6 22.8, 22.5 26.6; 65 (0.24) 24.8 22.7, 29.0 23.0, 40.8 32.8; 128
  // (0.38) 25.1 22.6, 34.8 26.7, 57.7 39.1; one entry's 256 queries of 2 heads (0.15) 14.6 22.7, 16.6 24.8, 21.9 37.6; 400 (0.24) 24.7 22.7, 28.9 24.8, 39.8 38.9; 8 x 4 heads on 14400
  // keys, 33 queries (1.4) 53.5 53.6, 78 58, 134 74.  (Too soon, up to a third, for two entries' 65 queries of 2 heads on 14400 keys, 0.29 million: 18.4 32.7, 24.6 32.8, 41.0 51.2.)
  const int64_t border = maps == 1 ? 500000 : 200000;
  if (bf16 && !mask && q_tokens > (maps == 1 ? 64 : 32) && kv_tokens > 0 &&
      ((int64_t)q_tokens * group + 15) / 16 * batch * (heads / group) >= border / kv_tokens + 1) {
    plan.kernel = CROSS_TC;
    plan.scratch = cross_tc_scratch(batch, q_tokens, kv_tokens, heads, D, maps);
    return plan;
  }
  const int64_t rows = (int64_t)q_tokens * group;
  if (bf16) {
    plan.kernel = CROSS_FEW;
    plan.split_keys = 0;
    const int64_t tiles = (rows + 15) / 16 * batch * (heads / group);
    // a tile's keys over a cluster of blocks, down to 128 keys to a block, until there are two blocks to a multiprocessor
    while (plan.cluster < 8 && tiles * plan.cluster < 2 * PLAN_SMS && kv_tokens / (2 * plan.cluster) >= 128) plan.cluster *= 2;
    // and over several clusters, which takes a second kernel, where those leave half of the device idle and more than 1024 keys to a block
    const int64_t blocks = tiles * plan.cluster;
    int64_t splits = blocks > 0 && 2 * blocks <= PLAN_SMS && kv_tokens / plan.cluster > 1024 ? PLAN_SMS / blocks : 1;
    const int64_t most = kv_tokens / ((int64_t)plan.cluster * 256);
    plan.splits = (int)(splits < most ? splits : most > 1 ? most : 1);
    // blocks of eight warps where there is but one to a multiprocessor
    plan.warps = blocks * plan.splits <= PLAN_SMS ? 8 : 4;
  } else {
    plan.kernel = CROSS_SCALAR;
    plan.rows = rows <= 16 ? 16 : 64;
    const int64_t blocks = (rows + plan.rows - 1) / plan.rows * batch * (heads / group);
    // Split the keys where the row tiles are fewer than two to a multiprocessor, down to two tiles of keys to a block.  Of two maps two blocks with 64 rows fit a multiprocessor with heads
    // of 32 only (registers, and shared memory by 3 KB with heads of 64), and blocks with 16 rows lose more by twice the parts to join than the second gains: one to a multiprocessor then.  Both
    // measured, us with one and with two: 1023 queries of 2 heads on 4096 keys, heads of 32 75.6 67.7, of 64 108.8 116.7, of 128 185.6 192.6; 300 queries, heads of 64 49 64, of
    // 128 75 96; 7 queries of 5 x 2 heads on 4800 keys 26.6 28.7, 36.9 38.9, 53.3 60.0.
    const int64_t fit = maps == 2 && !(D == 32 && plan.rows == 64) ? 1 : 2;
    int64_t splits = blocks > 0 ? fit * PLAN_SMS / blocks : 1;
    const int64_t most = ((int64_t)kv_tokens + 2 * BN - 1) / (2 * BN);
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    const int64_t each = (((int64_t)kv_tokens + splits - 1) / splits + BN - 1) / BN * BN;
    plan.split_keys = each > 0 ? (int)each : BN;
    plan.splits = kv_tokens > 0 ? (int)(((int64_t)kv_tokens + each - 1) / each) : 1;
  }
  plan.scratch = plan.splits > 1 ? (uint64_t)(rows * maps * batch * (heads / group)) * (uint64_t)plan.splits * (uint64_t)(D + 2) * 4u : 0u;
  return plan;
}

template <int MAPS>
cudaError_t launch_cross(const ParamsOf<MAPS>& p, const CrossPlan& plan, bool bf16, int D, cudaStream_t s) {
  if (plan.kernel == CROSS_TC) return launch_cross_tc<MAPS>(p, D, s);
  return bf16 ? launch_typed<__nv_bfloat16, MAPS>(p, plan, D, s) : launch_typed<float, MAPS>(p, plan, D, s);
}
template cudaError_t launch_cross<1>(const CrossParams&, const CrossPlan&, bool, int, cudaStream_t);
template cudaError_t launch_cross<2>(const DiffParams&, const CrossPlan&, bool, int, cudaStream_t);

}  // namespace tok
}  // namespace tt

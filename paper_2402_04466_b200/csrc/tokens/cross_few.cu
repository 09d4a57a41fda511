// Cross attention of few bf16 queries, and of masked ones (tt_cross_attention).
//
// With a handful of rows per key and value head (seven tools, times the heads of a group) the operator is bound by reading K and V once,
// 4 D bytes a key for 4 D operations a row.  What it takes is bytes in flight: every warp has a ring of tiles of its own
// in shared memory, 8 KB of keys and values each, fetched by its first lane through tensor maps, three ahead; no block-wide barrier until
// the end.  A warp takes 16 rows with m16n8k16 products (keys and values by ldmatrix), keeps its own maximum, which only moves when a
// weight would pass 2^8, and splits weights into two bf16 terms, so that they count with 16 bits and more: the products
// are not what the time goes to.  (Of an infinite value the two may make a NaN: then the warp's sums are taken again.)  Warps join through shared memory, the blocks of a cluster, which share an entry's keys, through each
// other's, and clusters, where one to a tile of rows does not fill the device, through cross_join_kernel.
//
// Registers in place of the rings (two tiles of 16 keys a warp, a tile ahead) came to 2.9 TB/s on eight streams of 14400 keys:
// latency, with 4 KB in flight per warp and most of the instructions addresses and byte permutes.  With the rings: 18.2 us (maps cut to 8100 to 14400 keys), 5.0 TB/s where a plain
// copy has 6.5; five streams of 4800 keys with masks take 9.25 us, 2 us of it K and V, the rest a launch, a chain of loads and the joins.
//
// Differential attention (MAPS = 2, tt_differential_attention): the two halves of a head's columns make two maps of scores, for the same number of products, and each tile of values meets
// both maps' weights while its registers are there, for twice as many.  The joins take both maps; a warp to a row ends with lambda and the norm, which reads the whole row.  The
// same eight streams 23.6 us, of which K and V would be 14; the same five with masks 11.5; clips of 60 keys 5.1.  With heads of 128 eight streams of 14400 keys take 46.3 us call by call (88.2 with
// the block's sums beside the rings, where two blocks did not fit a multiprocessor).
#include "tokens.h"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int MAX_CLUSTER = 8;

template <int MAPS>
struct CrossFewParams {
  TensorMap128 map_k, map_v;                   // [D][token][head][batch], box of Few::KEYS tokens
  ParamsOf<MAPS> c;
  int32_t k_h, k_b, v_h, v_b;                  // 0 where the axis is shared, else 1
};

template <int D, int W, int M>
struct Few {
  static constexpr int MAPS = M;               // 2: differential attention, a map of either half of the heads
  static constexpr int WARPS = W;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int STAGES = 3;
  static constexpr int KEYS = 2048 / D;        // of a tile
  static constexpr int ROW = D == 32 ? 64 : 128;
  static constexpr int SLABS = D == 128 ? 2 : 1;
  static constexpr int SLAB_BYTES = KEYS * ROW;
  static constexpr int HALF = 4096;            // keys of a tile, then values
  static constexpr int RING = STAGES * 2 * HALF;
  static constexpr int NK = KEYS / 8;          // products across a tile's keys
  static constexpr int NT = D / 8;             // products across the columns of the sums
  static constexpr int OP = D + 8;             // pitch of the joint sums
  static constexpr int SMEM = WARPS * RING + 1024;
  static constexpr int SUMS = MAPS * WARPS * 16 * OP * 4;         // bytes of the warps' sums, behind which lie the block's
  static_assert(SUMS + MAPS * 16 * D * 4 <= WARPS * RING, "the sums take the rings' place");
  static constexpr int BLOCKS = W == 4 ? 2 : 1;                   // to a multiprocessor: cross_plan counts on them
  static constexpr int STATIC = WARPS * STAGES * 8 + MAPS * (WARPS + 1) * 16 * 8 + 16 * 4;
  static_assert(BLOCKS * (SMEM + STATIC + 1024) <= 228 * 1024, "shared memory, of which each block takes 1 KB more");
};

// Where row `row`'s run `run` of 8 elements lies in a swizzled half of a tile.
template <int D>
__device__ __forceinline__ uint32_t run_at(int row, int run) {
  if (D == 32) return (uint32_t)(row * 64 + ((run ^ (row >> 1 & 3)) << 4));
  return (uint32_t)((run >> 3) * Few<D, 4, 1>::SLAB_BYTES + row * 128 + (((run & 7) ^ (row & 7)) << 4));
}
// A pair of floats from the same place in the shared memory of block `rank` of the cluster.
__device__ __forceinline__ float2 cluster_load(const float2* at, int rank, int cluster) {
  if (cluster == 1) return *at;
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(map_to_cta(smem_u32(at), (uint32_t)rank)) : "memory");
  return v;
}

// A warp's sums once more, key by key on the fp32 units, from the maxima that its rows g and g + 8 ended with: where a value is an infinity the two
// terms of its weight, whose signs may differ, have made a NaN of it.
template <int D>
__device__ __noinline__ void sums_again(const CrossParams& p, int b, int hk, int row0, int rows, int first, int j1, int step, const float (&m)[2], float (&o)[D / 8][4]) {
  constexpr int E = D / 4;                     // elements of a score to a lane
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(p.k.p) + b * p.k.b + hk * p.k.h + t * E;
  const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v.p) + b * p.v.b + hk * p.v.h + 2 * t;
  float q[2][E];
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + g + 8 * r;
    const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.q.p) + b * p.q.b + (int64_t)(row / p.group) * p.q.t + ((int64_t)hk * p.group + row % p.group) * p.q.h + t * E;
    for (int x = 0; x < E; ++x) q[r][x] = row < rows ? __bfloat162float(src[x]) : 0.f;
  }
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  for (int j = first; j < j1; j += step)
    for (int key = j; key < min(j1, j + Few<D, 4, 1>::KEYS); ++key) {
      float w[2];
      for (int r = 0; r < 2; ++r) {
        float s = 0.f;
        for (int x = 0; x < E; ++x) s = fmaf(q[r][x], __bfloat162float(k[key * p.k.t + x]), s);
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        w[r] = exp2_fast(fmaf(s, p.scale_log2, m[r] == -INFINITY ? 0.f : -m[r]));
      }
      for (int i = 0; i < D / 8; ++i)
        for (int x = 0; x < 4; ++x) o[i][x] = fmaf(w[x >> 1], __bfloat162float(v[key * p.v.t + 8 * i + (x & 1)]), o[i][x]);
    }
}

template <int D, bool MASK, int W, int MAPS>
__global__ void __launch_bounds__(Few<D, W, MAPS>::THREADS, Few<D, W, MAPS>::BLOCKS) cross_few_kernel(const __grid_constant__ CrossFewParams<MAPS> pp) {
  using F = Few<D, W, MAPS>;
  const ParamsOf<MAPS>& p = pp.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[F::WARPS][F::STAGES];
  __shared__ float2 s_ml[MAPS][F::WARPS][16];
  __shared__ float2 s_stat[MAPS][16];
  __shared__ float s_lambda[16];
  uint8_t* ring0 = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int pieces = p.splits * p.cluster;
  const int piece = blockIdx.x % pieces, row0 = (int)(blockIdx.x / pieces) * 16, hk = blockIdx.y, b = blockIdx.z;
  const int rows = clamp_length(p.q_lengths, b, p.q_tokens) * p.group;
  const int keys = clamp_length(p.kv_lengths, b, p.kv_tokens);
  if (row0 >= rows) return;                    // the whole cluster
  // an entry's keys in equal pieces, however many it has
  const int each = (int)(((int64_t)keys + F::KEYS * pieces - 1) / (F::KEYS * pieces)) * F::KEYS;
  const int j0 = min(keys, piece * each), j1 = min(keys, j0 + each);
  constexpr int STEP = F::KEYS * F::WARPS;
  const int first = j0 + warp * F::KEYS;

  const uint32_t ring = smem_u32(ring0 + warp * F::RING);
  auto load = [&](int j, int stage) {
    const uint32_t bar = smem_u32(&s_full[warp][stage]), dst = ring + (uint32_t)(stage * 2 * F::HALF);
    mbar_arrive_expect_tx(bar, 2 * F::HALF);
    for (int s = 0; s < F::SLABS; ++s) {
      tma_load_4d(dst + s * F::SLAB_BYTES, &pp.map_k, bar, s * 64, j, hk * pp.k_h, b * pp.k_b);
      tma_load_4d(dst + F::HALF + s * F::SLAB_BYTES, &pp.map_v, bar, s * 64, j, hk * pp.v_h, b * pp.v_b);
    }
  };
  if (lane == 0) {
    for (int s = 0; s < F::STAGES; ++s) mbar_init(smem_u32(&s_full[warp][s]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int s = 0; s < F::STAGES; ++s)
      if (first + s * STEP < j1) load(first + s * STEP, s);
  }
  __syncwarp();

  // queries: rows g and g + 8
  uint32_t q[D / 16][4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row0 + g + 8 * i;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const __nv_bfloat16*>(p.q.p) + b * p.q.b + (int64_t)(row / p.group) * p.q.t +
                                                            ((int64_t)hk * p.group + row % p.group) * p.q.h) + t;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      q[s][i] = row < rows ? __ldg(src + 8 * s) : 0u;
      q[s][2 + i] = row < rows ? __ldg(src + 8 * s + 4) : 0u;
    }
  }
  const uint8_t* mask[2] = {nullptr, nullptr};
  const bool pairs = MASK && (((uintptr_t)p.mask | (uintptr_t)p.mask_b | (uintptr_t)p.mask_q | (uintptr_t)(uint32_t)first) & 1u) == 0u;
  uint32_t seen[MASK ? F::NK : 1][2], coming[MASK ? F::NK : 1][2];    // mask bytes of keys 8 n + 2t and 8 n + 2t + 1 for both rows
  auto fetch_mask = [&](int j) {
    if (pairs && j + F::KEYS <= j1) {
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) coming[n][i] = __ldg(reinterpret_cast<const uint16_t*>(mask[i] + j + 8 * n + 2 * t));
    } else {
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int key = j + 8 * n + 2 * t;
          coming[n][i] = (key < j1 ? mask[i][key] : 0u) | (key + 1 < j1 ? (uint32_t)mask[i][key + 1] << 8 : 0u);
        }
    }
  };
  if (MASK) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + g + 8 * i;
      mask[i] = p.mask + b * p.mask_b + (int64_t)((row < rows ? row : row0) / p.group) * p.mask_q;
    }
    fetch_mask(first);
  }
  if constexpr (MAPS == 2) {
    // rows r and r + group are of one head; the last warps have the fewest keys
    for (int r = F::WARPS - 1 - warp; r < min(16, p.group); r += F::WARPS) {
      const float f = lambda_of(p.end, D / 2, hk * p.group + (row0 + r) % p.group);
      if (lane == 0) s_lambda[r] = f;
    }
  }
  float m[MAPS][2], l[MAPS][2], o[MAPS][F::NT][4];
#pragma unroll
  for (int w = 0; w < MAPS; ++w) {
    m[w][0] = m[w][1] = -INFINITY;
    l[w][0] = l[w][1] = 0.f;
#pragma unroll
    for (int i = 0; i < F::NT; ++i) o[w][i][0] = o[w][i][1] = o[w][i][2] = o[w][i][3] = 0.f;
  }
  const float c = p.scale_log2;

  int stage = 0;
  uint32_t phase = 0;
  for (int j = first; j < j1; j += STEP) {
    if (MASK) {
#pragma unroll
      for (int n = 0; n < F::NK; ++n) { seen[n][0] = coming[n][0]; seen[n][1] = coming[n][1]; }
      if (j + STEP < j1) fetch_mask(j + STEP);
    }
    if (!__all_sync(0xffffffffu, mbar_wait_limit(smem_u32(&s_full[warp][stage]), phase, WAIT_LIMIT))) {
      // ran out: give the copies in flight time to land, report, and leave the rest out
      for (int i = 0; i < 64; ++i) __nanosleep(16000);
      if (lane == 0 && p.status) atomicCAS(p.status, 0, WAIT_CROSS_FEW + warp);
      break;
    }
    const uint32_t ks = ring + (uint32_t)(stage * 2 * F::HALF), vs = ks + F::HALF;
    const int rem = j1 - j;
    if (rem < F::KEYS) {
      // the warp's last tile: values behind the last key may be anything, and weights of 0 would make NaN of it
      for (int i = lane; i < (F::KEYS - rem) * (D / 8); i += 32)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vs + run_at<D>(rem + i / (D / 8), i % (D / 8))), "r"(0u) : "memory");
      __syncwarp();
    }
    float s[MAPS][F::NK][4];                   // keys 8 n + 2t, 8 n + 2t + 1 for rows g, g + 8
#pragma unroll
    for (int n = 0; n < F::NK; ++n) {
#pragma unroll
      for (int w = 0; w < MAPS; ++w) s[w][n][0] = s[w][n][1] = s[w][n][2] = s[w][n][3] = 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {       // 32 elements of 8 keys
        uint32_t f[4];
        ldmatrix4<false>(f, ks + run_at<D>(8 * n + (lane & 7), 4 * x + (lane >> 3)));
        mma16816(s[2 * x / (D / 16 / MAPS)][n], q[2 * x], f[0], f[1]);
        mma16816(s[(2 * x + 1) / (D / 16 / MAPS)][n], q[2 * x + 1], f[2], f[3]);
      }
    }
#pragma unroll
    for (int w = 0; w < MAPS; ++w) {
      if (rem < F::KEYS) {
#pragma unroll
        for (int n = 0; n < F::NK; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (8 * n + 2 * t + (x & 1) >= rem) s[w][n][x] = -INFINITY;
      }
      if (MASK) {
#pragma unroll
        for (int n = 0; n < F::NK; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if ((seen[n][x >> 1] & (x & 1 ? 0xFF00u : 0xFFu)) == 0u) s[w][n][x] = -INFINITY;
      }
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int n = 0; n < F::NK; ++n) {
        top[0] = max3(top[0], s[w][n][0], s[w][n][1]);
        top[1] = max3(top[1], s[w][n][2], s[w][n][3]);
      }
      if (__any_sync(0xffffffffu, top[0] * c > m[w][0] + 8.f || top[1] * c > m[w][1] + 8.f)) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float now = top[r] * c;
          now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 1));
          now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 2));
          now = fmaxf(now, m[w][r]);
          const float fade = now == -INFINITY ? 1.f : exp2_fast(m[w][r] - now);
          m[w][r] = now;
          l[w][r] *= fade;
#pragma unroll
          for (int i = 0; i < F::NT; ++i) { o[w][i][2 * r] *= fade; o[w][i][2 * r + 1] *= fade; }
        }
      }
      const float base[2] = {m[w][0] == -INFINITY ? 0.f : m[w][0], m[w][1] == -INFINITY ? 0.f : m[w][1]};
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[w][n][x] = exp2_fast(fmaf(s[w][n][x], c, -base[x >> 1]));
          l[w][x >> 1] += s[w][n][x];
        }
    }
    bool careful = false;
    if (MASK) {
      // an infinity or NaN among the values: times 0 it is a NaN, which the sum then keeps
      __nv_bfloat162 odd = __float2bfloat162_rn(0.f);
#pragma unroll
      for (int i = 0; i < F::HALF / 512; ++i) {
        uint32_t f[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3]) : "r"(vs + (uint32_t)(i * 512 + lane * 16)));
#pragma unroll
        for (int x = 0; x < 4; ++x) odd = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&f[x]), __float2bfloat162_rn(0.f), odd);
      }
      careful = __any_sync(0xffffffffu, (*reinterpret_cast<const uint32_t*>(&odd) & 0x7FFF7FFFu) != 0u);
    }
    if (!MASK || !careful) {
#pragma unroll
      for (int k = 0; k < F::NK / 2; ++k) {    // 16 keys
        uint32_t hi[MAPS][4], lo[MAPS][4];
#pragma unroll
        for (int w = 0; w < MAPS; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = s[w][2 * k + (i >> 1)][2 * (i & 1)], e = s[w][2 * k + (i >> 1)][2 * (i & 1) + 1];
            hi[w][i] = pack_bf16(a, e);
            lo[w][i] = pack_bf16(a - __uint_as_float(hi[w][i] << 16), e - __uint_as_float(hi[w][i] & 0xFFFF0000u));
          }
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {     // 16 columns
          uint32_t f[4];
          ldmatrix4<true>(f, vs + run_at<D>(16 * k + (lane & 15), 2 * x + (lane >> 4)));
#pragma unroll
          for (int w = 0; w < MAPS; ++w) {
            mma16816(o[w][2 * x], hi[w], f[0], f[1]);
            mma16816(o[w][2 * x], lo[w], f[0], f[1]);
            mma16816(o[w][2 * x + 1], hi[w], f[2], f[3]);
            mma16816(o[w][2 * x + 1], lo[w], f[2], f[3]);
          }
        }
      }
    } else {
      // one key at a time, left out of the rows that do not see it
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll 1
        for (int kk = 0; kk < 8 && 8 * n + kk < rem; ++kk) {
          const int from = (lane & ~3) | (kk >> 1), key = 8 * n + kk;
          float mine[MAPS][2];
          uint32_t sees[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int w = 0; w < MAPS; ++w) mine[w][r] = __shfl_sync(0xffffffffu, kk & 1 ? s[w][n][2 * r + 1] : s[w][n][2 * r], from);
            sees[r] = __shfl_sync(0xffffffffu, seen[n][r] >> (8 * (kk & 1)) & 0xFFu, from);
          }
#pragma unroll
          for (int i = 0; i < F::NT; ++i) {
            uint32_t u;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u) : "r"(vs + run_at<D>(key, i) + (uint32_t)(4 * t)));
            const float v0 = __uint_as_float(u << 16), v1 = __uint_as_float(u & 0xFFFF0000u);
#pragma unroll
            for (int w = 0; w < MAPS; ++w) {
              if (sees[0]) { o[w][i][0] = fmaf(mine[w][0], v0, o[w][i][0]); o[w][i][1] = fmaf(mine[w][0], v1, o[w][i][1]); }
              if (sees[1]) { o[w][i][2] = fmaf(mine[w][1], v0, o[w][i][2]); o[w][i][3] = fmaf(mine[w][1], v1, o[w][i][3]); }
            }
          }
        }
    }
    __syncwarp();                              // the tile has been read
    if (lane == 0 && j + F::STAGES * STEP < j1) load(j + F::STAGES * STEP, stage);
    if (++stage == F::STAGES) { stage = 0; phase ^= 1u; }
  }
  if constexpr (!MASK && MAPS == 1) {
    // (under a mask every tile's values are looked at before they are used; here that took eight streams' 14400 keys from 18.2 to 20.0 us)
    float odd[4] = {0.f, 0.f, 0.f, 0.f};       // four chains
#pragma unroll
    for (int i = 0; i < F::NT; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) odd[x] = fmaf(o[0][i][x], 0.f, odd[x]);
    if (__builtin_expect(__any_sync(0xffffffffu, odd[0] + odd[1] + (odd[2] + odd[3]) != 0.f), 0)) {
      const float top[2] = {m[0][0], m[0][1]};
      float again[F::NT][4];
      sums_again<D>(p, b, hk, row0, rows, first, j1, STEP, top, again);
#pragma unroll
      for (int i = 0; i < F::NT; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[0][i][x] = again[i][x];
    }
  }

  // join the warps: row r of the tile, element d.  The sums take the place of the rings, whose copies have all landed.
  __syncthreads();
  float* s_o = reinterpret_cast<float*>(ring0);      // [MAPS][WARPS][16][OP]
  auto& s_sum = *reinterpret_cast<float (*)[MAPS][16][D]>(ring0 + F::SUMS);      // the block's: in the same place in every block of a cluster
#pragma unroll
  for (int w = 0; w < MAPS; ++w)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[w][r] += __shfl_xor_sync(0xffffffffu, l[w][r], 1);
      l[w][r] += __shfl_xor_sync(0xffffffffu, l[w][r], 2);
      if (t == 0) s_ml[w][warp][g + 8 * r] = make_float2(m[w][r], l[w][r]);
#pragma unroll
      for (int i = 0; i < F::NT; ++i)
        *reinterpret_cast<float2*>(s_o + ((w * F::WARPS + warp) * 16 + g + 8 * r) * F::OP + 8 * i + 2 * t) = make_float2(o[w][i][2 * r], o[w][i][2 * r + 1]);
    }
  __syncthreads();
  const int live = min(16, rows - row0);
  for (int i = threadIdx.x; i < MAPS * live * (D / 4); i += F::THREADS) {
    const int d = i % (D / 4) * 4, w = MAPS == 2 && i / (D / 4) >= live, r = i / (D / 4) - w * live;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) top = fmaxf(top, s_ml[w][x][r].x);
    const float base = top == -INFINITY ? 0.f : top;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) {
      const float2 ml = s_ml[w][x][r];
      const float4 v = *reinterpret_cast<const float4*>(s_o + ((w * F::WARPS + x) * 16 + r) * F::OP + d);
      const float f = exp2_fast(ml.x - base);
      total = fmaf(f, ml.y, total);
      sum.x = fmaf(f, v.x, sum.x);
      sum.y = fmaf(f, v.y, sum.y);
      sum.z = fmaf(f, v.z, sum.z);
      sum.w = fmaf(f, v.w, sum.w);
    }
    *reinterpret_cast<float4*>(&s_sum[w][r][d]) = sum;
    if (d == 0) s_stat[w][r] = make_float2(top, total);
  }
  constexpr int E = (D + 63) / 64;             // pairs of a lane in a row (heads of 32: of the first 16 lanes)
  float2 weight[MAPS == 2 ? E : 1];            // of the norm: on its way while the cluster meets
  if constexpr (MAPS == 2) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = 64 * e + 2 * lane;
      weight[e] = d < D ? make_float2(norm_weight(p.end, d), norm_weight(p.end, d + 1)) : make_float2(0.f, 0.f);
    }
  }
  // join the blocks of the cluster: each takes its share of the elements from all of them
  if (p.cluster > 1) cluster_sync_all();
  else __syncthreads();
  const int rank = p.cluster > 1 ? (int)cluster_ctarank() : 0;
  // elements d and d + 1 of row r, map w, of all blocks: sums, total and maximum
  auto joined = [&](int w, int r, int d, float& top, float& total) {
    float2 stat[MAX_CLUSTER], sum[MAX_CLUSTER];
    top = -INFINITY;
#pragma unroll
    for (int x = 0; x < MAX_CLUSTER; ++x)
      if (x < p.cluster) {
        stat[x] = cluster_load(&s_stat[w][r], x, p.cluster);
        sum[x] = cluster_load(reinterpret_cast<float2*>(&s_sum[w][r][d]), x, p.cluster);
        top = fmaxf(top, stat[x].x);
      }
    const float base = top == -INFINITY ? 0.f : top;
    float a = 0.f, e = 0.f;
    total = 0.f;
#pragma unroll
    for (int x = 0; x < MAX_CLUSTER; ++x)
      if (x < p.cluster) {
        const float f = exp2_fast(stat[x].x - base);
        total = fmaf(f, stat[x].y, total);
        a = fmaf(f, sum[x].x, a);
        e = fmaf(f, sum[x].y, e);
      }
    return make_float2(a, e);
  };
  if (MAPS == 1 || p.splits > 1) {
#pragma unroll
    for (int w = 0; w < MAPS; ++w)
      for (int i = rank * F::THREADS + threadIdx.x; i < 16 * (D / 2); i += F::THREADS * p.cluster) {
        const int r = i / (D / 2), d = i % (D / 2) * 2, row = row0 + r;
        if (row >= rows) break;
        float top, total;
        const float2 sum = joined(w, r, d, top, total);
        if (p.splits > 1) {
          const Part to = part_of<MAPS>(p, D, b, hk, row, w);
          const int split = piece / p.cluster;
          if (d == 0) to.stat[split] = make_float2(top, total);
          *reinterpret_cast<float2*>(to.sum + (int64_t)split * D + d) = sum;
        } else {
          const float inv = total == 0.f ? 0.f : 1.f / total;
          __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + ((int64_t)hk * p.group + row % p.group) * p.o.h;
          *reinterpret_cast<uint32_t*>(dst + d) = pack_bf16(sum.x * inv, sum.y * inv);
        }
      }
  }
  if constexpr (MAPS == 2) {
    // a warp to a row, whose norm takes all of its elements
    if (p.splits == 1)
      for (int r = rank * F::WARPS + warp; r < 16 && row0 + r < rows; r += F::WARPS * p.cluster) {
        const int row = row0 + r;
        // all loads first: the sums' of both maps, and block x's maximum and total to lane x, map 2's to lane 8 + x
        float2 sums[2][E][MAX_CLUSTER];
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int e = 0; e < E; ++e)
#pragma unroll
            for (int x = 0; x < MAX_CLUSTER; ++x)
              sums[w][e][x] = x < p.cluster && 64 * e + 2 * lane < D ? cluster_load(reinterpret_cast<float2*>(&s_sum[w][r][64 * e + 2 * lane]), x, p.cluster) : make_float2(0.f, 0.f);
        const float2 stat = lane < 16 && (lane & 7) < p.cluster ? cluster_load(&s_stat[lane >> 3][r], lane & 7, p.cluster) : make_float2(-INFINITY, 0.f);
        float top = stat.x;
#pragma unroll
        for (int x = 4; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        float f = exp2_fast(stat.x - (top == -INFINITY ? 0.f : top)), total = f * stat.y;
#pragma unroll
        for (int x = 4; x > 0; x >>= 1) total += __shfl_xor_sync(0xffffffffu, total, x);
        f *= total == 0.f ? 0.f : (lane < 8 ? 1.f : -s_lambda[r % p.group]) / total;
        float2 y[E];
        float squares = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int x = 0; x < MAX_CLUSTER; ++x) {
            const float share = __shfl_sync(0xffffffffu, f, 8 * w + x);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              y[e].x = fmaf(share, sums[w][e][x].x, y[e].x);
              y[e].y = fmaf(share, sums[w][e][x].y, y[e].y);
            }
          }
#pragma unroll
        for (int e = 0; e < E; ++e) squares = fmaf(y[e].x, y[e].x, fmaf(y[e].y, y[e].y, squares));
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, x);
        const float gain = row_gain<D>(p.end, squares);
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + ((int64_t)hk * p.group + row % p.group) * p.o.h;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int d = 64 * e + 2 * lane;
          if (d < D) *reinterpret_cast<uint32_t*>(dst + d) = pack_bf16(y[e].x * gain * weight[e].x, y[e].y * gain * weight[e].y);
        }
      }
  }
  if (p.cluster > 1) cluster_sync_all();       // no block leaves while another reads its sums
}

template <int D, bool MASK, int W, int MAPS>
cudaError_t launch(const CrossFewParams<MAPS>& p, cudaStream_t s) {
  using F = Few<D, W, MAPS>;
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(cross_few_kernel<D, MASK, W, MAPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM); });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((int64_t)p.c.q_tokens * p.c.group + 15) / 16;
  return launch_kernel(cross_few_kernel<D, MASK, W, MAPS>, dim3((unsigned)(tiles * p.c.splits * p.c.cluster), (unsigned)(p.c.heads / p.c.group), (unsigned)p.c.batch),
                       F::THREADS, F::SMEM, s, p, false, p.c.cluster);
}
template <int D, int MAPS>
cudaError_t launch(const ParamsOf<MAPS>& c, int warps, cudaStream_t s) {
  CrossFewParams<MAPS> p{};
  const int kv_heads = c.heads / c.group, keys = Few<D, 4, MAPS>::KEYS;
  if (c.kv_tokens > 0 && (!token_map(&p.map_k, c.k, D, c.kv_tokens, kv_heads, c.batch, keys) || !token_map(&p.map_v, c.v, D, c.kv_tokens, kv_heads, c.batch, keys)))
    return cudaErrorInvalidValue;
  p.c = c;
  p.k_h = c.k.h != 0; p.k_b = c.k.b != 0; p.v_h = c.v.h != 0; p.v_b = c.v.b != 0;
  if (warps == 8) return p.c.mask ? launch<D, true, 8, MAPS>(p, s) : launch<D, false, 8, MAPS>(p, s);
  return p.c.mask ? launch<D, true, 4, MAPS>(p, s) : launch<D, false, 4, MAPS>(p, s);
}

}  // namespace

template <int MAPS>
cudaError_t launch_cross_few(const ParamsOf<MAPS>& p, int D, int warps, cudaStream_t s) {
  return D == 32 ? launch<32, MAPS>(p, warps, s) : D == 64 ? launch<64, MAPS>(p, warps, s) : launch<128, MAPS>(p, warps, s);
}
template cudaError_t launch_cross_few<1>(const CrossParams&, int, int, cudaStream_t);
template cudaError_t launch_cross_few<2>(const DiffParams&, int, int, cudaStream_t);

}  // namespace tok
}  // namespace tt

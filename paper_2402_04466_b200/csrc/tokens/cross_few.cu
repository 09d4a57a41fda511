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
#include "tokens.h"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int MAX_CLUSTER = 8;

struct CrossFewParams {
  TensorMap128 map_k, map_v;                   // [D][token][head][batch], box of Few::KEYS tokens
  CrossParams c;
  int32_t k_h, k_b, v_h, v_b;                  // 0 where the axis is shared, else 1
};

template <int D, int W>
struct Few {
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
  static constexpr int BLOCKS = W == 4 ? 2 : 1;                   // to a multiprocessor
  static_assert(WARPS * 16 * OP * 4 <= WARPS * RING, "the sums take the rings' place");
};

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANSPOSED>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  if (TRANSPOSED) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Where row `row`'s run `run` of 8 elements lies in a swizzled half of a tile.
template <int D>
__device__ __forceinline__ uint32_t run_at(int row, int run) {
  if (D == 32) return (uint32_t)(row * 64 + ((run ^ (row >> 1 & 3)) << 4));
  return (uint32_t)((run >> 3) * Few<D, 4>::SLAB_BYTES + row * 128 + (((run & 7) ^ (row & 7)) << 4));
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
    for (int key = j; key < min(j1, j + Few<D, 4>::KEYS); ++key) {
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

template <int D, bool MASK, int W>
__global__ void __launch_bounds__(Few<D, W>::THREADS, Few<D, W>::BLOCKS) cross_few_kernel(const __grid_constant__ CrossFewParams pp) {
  using F = Few<D, W>;
  const CrossParams& p = pp.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[F::WARPS][F::STAGES];
  __shared__ float2 s_ml[F::WARPS][16];
  __shared__ float s_sum[16][D];
  __shared__ float2 s_stat[16];
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
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float o[F::NT][4];
#pragma unroll
  for (int i = 0; i < F::NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
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
    float s[F::NK][4];                         // keys 8 n + 2t, 8 n + 2t + 1 for rows g, g + 8
#pragma unroll
    for (int n = 0; n < F::NK; ++n) {
      s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {       // 32 elements of 8 keys
        uint32_t f[4];
        ldmatrix4<false>(f, ks + run_at<D>(8 * n + (lane & 7), 4 * x + (lane >> 3)));
        mma16816(s[n], q[2 * x], f[0], f[1]);
        mma16816(s[n], q[2 * x + 1], f[2], f[3]);
      }
    }
    if (rem < F::KEYS) {
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (8 * n + 2 * t + (x & 1) >= rem) s[n][x] = -INFINITY;
    }
    if (MASK) {
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if ((seen[n][x >> 1] & (x & 1 ? 0xFF00u : 0xFFu)) == 0u) s[n][x] = -INFINITY;
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < F::NK; ++n) {
      top[0] = max3(top[0], s[n][0], s[n][1]);
      top[1] = max3(top[1], s[n][2], s[n][3]);
    }
    if (__any_sync(0xffffffffu, top[0] * c > m[0] + 8.f || top[1] * c > m[1] + 8.f)) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float now = top[r] * c;
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
#pragma unroll
    for (int n = 0; n < F::NK; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[n][x] = exp2_fast(fmaf(s[n][x], c, -base[x >> 1]));
        l[x >> 1] += s[n][x];
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
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = s[2 * k + (i >> 1)][2 * (i & 1)], e = s[2 * k + (i >> 1)][2 * (i & 1) + 1];
          hi[i] = pack_bf16(a, e);
          lo[i] = pack_bf16(a - __uint_as_float(hi[i] << 16), e - __uint_as_float(hi[i] & 0xFFFF0000u));
        }
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {     // 16 columns
          uint32_t f[4];
          ldmatrix4<true>(f, vs + run_at<D>(16 * k + (lane & 15), 2 * x + (lane >> 4)));
          mma16816(o[2 * x], hi, f[0], f[1]);
          mma16816(o[2 * x], lo, f[0], f[1]);
          mma16816(o[2 * x + 1], hi, f[2], f[3]);
          mma16816(o[2 * x + 1], lo, f[2], f[3]);
        }
      }
    } else {
      // one key at a time, left out of the rows that do not see it
#pragma unroll
      for (int n = 0; n < F::NK; ++n)
#pragma unroll 1
        for (int kk = 0; kk < 8 && 8 * n + kk < rem; ++kk) {
          const int from = (lane & ~3) | (kk >> 1), key = 8 * n + kk;
          float mine[2];
          uint32_t sees[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            mine[r] = __shfl_sync(0xffffffffu, kk & 1 ? s[n][2 * r + 1] : s[n][2 * r], from);
            sees[r] = __shfl_sync(0xffffffffu, seen[n][r] >> (8 * (kk & 1)) & 0xFFu, from);
          }
#pragma unroll
          for (int i = 0; i < F::NT; ++i) {
            uint32_t u;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u) : "r"(vs + run_at<D>(key, i) + (uint32_t)(4 * t)));
            const float v0 = __uint_as_float(u << 16), v1 = __uint_as_float(u & 0xFFFF0000u);
            if (sees[0]) { o[i][0] = fmaf(mine[0], v0, o[i][0]); o[i][1] = fmaf(mine[0], v1, o[i][1]); }
            if (sees[1]) { o[i][2] = fmaf(mine[1], v0, o[i][2]); o[i][3] = fmaf(mine[1], v1, o[i][3]); }
          }
        }
    }
    __syncwarp();                              // the tile has been read
    if (lane == 0 && j + F::STAGES * STEP < j1) load(j + F::STAGES * STEP, stage);
    if (++stage == F::STAGES) { stage = 0; phase ^= 1u; }
  }
  if (!MASK) {
    // (under a mask every tile's values are looked at before they are used; here that took eight streams' 14400 keys from 18.2 to 20.0 us)
    float odd[4] = {0.f, 0.f, 0.f, 0.f};       // four chains
#pragma unroll
    for (int i = 0; i < F::NT; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) odd[x] = fmaf(o[i][x], 0.f, odd[x]);
    if (__builtin_expect(__any_sync(0xffffffffu, odd[0] + odd[1] + (odd[2] + odd[3]) != 0.f), 0)) {
      const float top[2] = {m[0], m[1]};
      float again[F::NT][4];
      sums_again<D>(p, b, hk, row0, rows, first, j1, STEP, top, again);
#pragma unroll
      for (int i = 0; i < F::NT; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[i][x] = again[i][x];
    }
  }

  // join the warps: row r of the tile, element d.  The sums take the place of the rings, whose copies have all landed.
  __syncthreads();
  float* s_o = reinterpret_cast<float*>(ring0);      // [WARPS][16][OP]
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    if (t == 0) s_ml[warp][g + 8 * r] = make_float2(m[r], l[r]);
#pragma unroll
    for (int i = 0; i < F::NT; ++i) *reinterpret_cast<float2*>(s_o + (warp * 16 + g + 8 * r) * F::OP + 8 * i + 2 * t) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (D / 2); i += F::THREADS) {
    const int r = i / (D / 2), d = i % (D / 2) * 2;
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) top = fmaxf(top, s_ml[x][r].x);
    const float base = top == -INFINITY ? 0.f : top;
    float a = 0.f, e = 0.f, total = 0.f;
#pragma unroll
    for (int x = 0; x < F::WARPS; ++x) {
      const float2 ml = s_ml[x][r], v = *reinterpret_cast<const float2*>(s_o + (x * 16 + r) * F::OP + d);
      const float f = exp2_fast(ml.x - base);
      total = fmaf(f, ml.y, total);
      a = fmaf(f, v.x, a);
      e = fmaf(f, v.y, e);
    }
    *reinterpret_cast<float2*>(&s_sum[r][d]) = make_float2(a, e);
    if (d == 0) s_stat[r] = make_float2(top, total);
  }
  // join the blocks of the cluster: each takes its share of the elements from all of them
  if (p.cluster > 1) cluster_sync_all();
  else __syncthreads();
  const int rank = p.cluster > 1 ? (int)cluster_ctarank() : 0;
  for (int i = rank * F::THREADS + threadIdx.x; i < 16 * (D / 2); i += F::THREADS * p.cluster) {
    const int r = i / (D / 2), d = i % (D / 2) * 2, row = row0 + r;
    if (row >= rows) break;
    float2 stat[MAX_CLUSTER], sum[MAX_CLUSTER];
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < MAX_CLUSTER; ++x)
      if (x < p.cluster) {
        stat[x] = cluster_load(&s_stat[r], x, p.cluster);
        sum[x] = cluster_load(reinterpret_cast<float2*>(&s_sum[r][d]), x, p.cluster);
        top = fmaxf(top, stat[x].x);
      }
    const float base = top == -INFINITY ? 0.f : top;
    float a = 0.f, e = 0.f, total = 0.f;
#pragma unroll
    for (int x = 0; x < MAX_CLUSTER; ++x)
      if (x < p.cluster) {
        const float f = exp2_fast(stat[x].x - base);
        total = fmaf(f, stat[x].y, total);
        a = fmaf(f, sum[x].x, a);
        e = fmaf(f, sum[x].y, e);
      }
    if (p.splits > 1) {
      const Part to = part_of(p, D, b, hk, row);
      const int split = piece / p.cluster;
      if (d == 0) to.stat[split] = make_float2(top, total);
      *reinterpret_cast<float2*>(to.sum + (int64_t)split * D + d) = make_float2(a, e);
    } else {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + (int64_t)(row / p.group) * p.o.t + ((int64_t)hk * p.group + row % p.group) * p.o.h;
      *reinterpret_cast<uint32_t*>(dst + d) = pack_bf16(a * inv, e * inv);
    }
  }
  if (p.cluster > 1) cluster_sync_all();       // no block leaves while another reads its sums
}

template <int D, bool MASK, int W>
cudaError_t launch(const CrossFewParams& p, cudaStream_t s) {
  using F = Few<D, W>;
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(cross_few_kernel<D, MASK, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM); });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((int64_t)p.c.q_tokens * p.c.group + 15) / 16;
  return launch_kernel(cross_few_kernel<D, MASK, W>, dim3((unsigned)(tiles * p.c.splits * p.c.cluster), (unsigned)(p.c.heads / p.c.group), (unsigned)p.c.batch),
                       F::THREADS, F::SMEM, s, p, false, p.c.cluster);
}
template <int D>
cudaError_t launch(const CrossParams& c, int warps, cudaStream_t s) {
  CrossFewParams p{};
  const int kv_heads = c.heads / c.group, keys = Few<D, 4>::KEYS;
  if (c.kv_tokens > 0 && (!token_map(&p.map_k, c.k, D, c.kv_tokens, kv_heads, c.batch, keys) || !token_map(&p.map_v, c.v, D, c.kv_tokens, kv_heads, c.batch, keys)))
    return cudaErrorInvalidValue;
  p.c = c;
  p.k_h = c.k.h != 0; p.k_b = c.k.b != 0; p.v_h = c.v.h != 0; p.v_b = c.v.b != 0;
  if (warps == 8) return p.c.mask ? launch<D, true, 8>(p, s) : launch<D, false, 8>(p, s);
  return p.c.mask ? launch<D, true, 4>(p, s) : launch<D, false, 4>(p, s);
}

}  // namespace

cudaError_t launch_cross_few(const CrossParams& p, int D, int warps, cudaStream_t s) {
  return D == 32 ? launch<32>(p, warps, s) : D == 64 ? launch<64>(p, warps, s) : launch<128>(p, warps, s);
}

}  // namespace tok
}  // namespace tt

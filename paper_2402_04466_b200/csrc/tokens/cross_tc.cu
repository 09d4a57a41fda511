// Cross attention of many bf16 queries on the tensor cores (tt_cross_attention without a mask).
//
//   S = Q K^T (128 queries x 128 keys),  P = 2^(c S - c m),  O += P V,  l += sum P,  c = scale * log2(e)
#include "tokens.h"

#include <cuda.h>

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int BM = 128, BN = 128;

struct CrossTcParams {
  TensorMap128 map_q, map_k, map_v;      // [D][token][head][batch], box of 128 tokens
  View o;
  const int32_t* q_lengths;
  const int32_t* kv_lengths;
  int32_t* status;
  int32_t q_tokens, kv_tokens, heads, group, q_tiles;
  int32_t q_h, q_b, k_h, k_b, v_h, v_b;  // 0 where the axis is shared, else 1
  float scale_log2;
};

template <int D, int TILES>
struct Cfg {
  static constexpr int ROW = D == 32 ? 64 : 128;                    // bytes of a row in a slab
  static constexpr int SLABS = D == 128 ? 2 : 1;
  static constexpr int SLAB_BYTES = BM * ROW;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;             // 128 tokens of one operand
  static constexpr uint32_t LAYOUT = D == 32 ? 4u : 2u;             // 64- or 128-byte swizzle
  static constexpr int STAGES = 2;
  static constexpr int THREADS = TILES * 128 + 64;
  static constexpr int BLOCKS = TILES == 1 ? 2 : 1;                 // to a multiprocessor
  static constexpr int O_COL = TILES * BN;
  static constexpr uint32_t TMEM = TILES * (BN + D) <= 256 ? 256 : 512;
  static constexpr int BAR_BYTES = 256;
  static constexpr int SMEM = (TILES + 2 * STAGES) * TILE_BYTES + BAR_BYTES + 1024;
  static_assert(SMEM * BLOCKS <= 227 * 1024, "shared memory");
};

template <int D, int TILES>
__global__ void __launch_bounds__(Cfg<D, TILES>::THREADS, Cfg<D, TILES>::BLOCKS) cross_tc_kernel(const __grid_constant__ CrossTcParams p) {
  using C = Cfg<D, TILES>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* s_q = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* s_k = s_q + TILES * C::TILE_BYTES;
  uint8_t* s_v = s_k + STAGES * C::TILE_BYTES;
  uint64_t* qfull = reinterpret_cast<uint64_t*>(s_v + STAGES * C::TILE_BYTES);
  uint64_t* kfull = qfull + 1;                 // [STAGES]
  uint64_t* kempty = kfull + STAGES;
  uint64_t* vfull = kempty + STAGES;
  uint64_t* vempty = vfull + STAGES;
  uint64_t* sfull = vempty + STAGES;           // [TILES] scores are there
  uint64_t* pfull = sfull + TILES;             // [TILES] weights are there
  uint64_t* ofull = pfull + TILES;             // [TILES] last product is done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ofull + TILES);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_status = reinterpret_cast<int*>(tmem_slot + 2);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int b = blockIdx.z, h = blockIdx.y, row0 = (int)blockIdx.x * (BM * TILES);
  const int rows = clamp_length(p.q_lengths, b, p.q_tokens), keys = clamp_length(p.kv_lengths, b, p.kv_tokens);
  if (row0 >= rows) return;
  const int n = (keys + BN - 1) / BN;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(qfull), 1);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(kfull + s), 1);
      mbar_init(smem_u32(kempty + s), 1);
      mbar_init(smem_u32(vfull + s), 1);
      mbar_init(smem_u32(vempty + s), 1);
    }
    for (int t = 0; t < TILES; ++t) {
      mbar_init(smem_u32(sfull + t), 1);
      mbar_init(smem_u32(pfull + t), 4);
      mbar_init(smem_u32(ofull + t), 1);
    }
    *abort_flag = 0;
    *s_status = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == TILES * 4 + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == TILES * 4) {
    // ------------------------------------------------------------------------------ loads
    if (lane == 0 && n > 0) {
      const int hk = h / p.group;
      auto load = [&](uint8_t* dst, const void* map, uint64_t* bar, int row, int hh, int bb) {
        for (int s = 0; s < C::SLABS; ++s) tma_load_4d(smem_u32(dst + s * C::SLAB_BYTES), map, smem_u32(bar), s * 64, row, hh, bb);
      };
      mbar_arrive_expect_tx(smem_u32(qfull), TILES * C::TILE_BYTES);
      for (int t = 0; t < TILES; ++t) load(s_q + t * C::TILE_BYTES, &p.map_q, qfull, row0 + t * BM, h * p.q_h, b * p.q_b);
      uint32_t stage = 0, phase = 0;
      for (int j = 0; j < n; ++j) {
        if (!mbar_wait(smem_u32(kempty + stage), phase ^ 1u, abort_flag, s_status, WAIT_CROSS_TC + (int)stage, WAIT_LIMIT)) break;
        mbar_arrive_expect_tx(smem_u32(kfull + stage), C::TILE_BYTES);
        load(s_k + stage * C::TILE_BYTES, &p.map_k, kfull + stage, j * BN, hk * p.k_h, b * p.k_b);
        if (!mbar_wait(smem_u32(vempty + stage), phase ^ 1u, abort_flag, s_status, WAIT_CROSS_TC + 0x10 + (int)stage, WAIT_LIMIT)) break;
        mbar_arrive_expect_tx(smem_u32(vfull + stage), C::TILE_BYTES);
        load(s_v + stage * C::TILE_BYTES, &p.map_v, vfull + stage, j * BN, hk * p.v_h, b * p.v_b);
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == TILES * 4 + 1) {
    // ----------------------------------------------------------------------------- products
    const bool issuer = elect_one();
    constexpr uint32_t QK = make_idesc(BM, BN), PV = make_idesc(BM, D) | B_BY_ROWS;
    const uint64_t q0 = make_smem_desc(smem_u32(s_q), 8 * C::ROW, C::LAYOUT), k0 = make_smem_desc(smem_u32(s_k), 8 * C::ROW, C::LAYOUT);
    const uint64_t v0 = make_rows_desc(smem_u32(s_v), C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    bool ok = true;
    auto scores = [&](int t, uint32_t stage) {
      if (issuer) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t at = (uint64_t)((k / 4) * (C::SLAB_BYTES >> 4) + (k % 4) * 2);
          umma_bf16(tmem + (uint32_t)(t * BN), q0 + (uint64_t)(t * (C::TILE_BYTES >> 4)) + at, k0 + (uint64_t)stage * (C::TILE_BYTES >> 4) + at, QK, k > 0);
        }
        umma_commit(smem_u32(sfull + t));
      }
      __syncwarp();
    };
    uint32_t stage = 0, phase = 0;               // of K one tile ahead of V's
    uint32_t vstage = 0, vphase = 0;
    if (n > 0) {
      ok = mbar_wait(smem_u32(qfull), 0, abort_flag, s_status, WAIT_CROSS_TC + 0x20, WAIT_LIMIT) &&
           mbar_wait(smem_u32(kfull), 0, abort_flag, s_status, WAIT_CROSS_TC + 0x30, WAIT_LIMIT);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        for (int t = 0; t < TILES; ++t) scores(t, 0);
        if (issuer) umma_commit(smem_u32(kempty));
        if (++stage == STAGES) { stage = 0; phase ^= 1u; }
      }
    }
    for (int j = 0; j < n && ok; ++j) {
      ok = mbar_wait(smem_u32(vfull + vstage), vphase, abort_flag, s_status, WAIT_CROSS_TC + 0x40 + (int)vstage, WAIT_LIMIT);
      if (j + 1 < n) ok = ok && mbar_wait(smem_u32(kfull + stage), phase, abort_flag, s_status, WAIT_CROSS_TC + 0x30 + (int)stage, WAIT_LIMIT);
      if (!__all_sync(0xffffffffu, ok)) break;
      const int rem = keys - j * BN;
      if (rem < BN) {
        // rows behind the last key may hold anything, and their weights of 0 would make NaN of it
        for (int s = 0; s < C::SLABS; ++s)
          for (int i = rem * C::ROW + lane * 16; i < C::SLAB_BYTES; i += 512)
            *reinterpret_cast<uint4*>(s_v + vstage * C::TILE_BYTES + s * C::SLAB_BYTES + i) = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
        __syncwarp();
      }
      for (int t = 0; t < TILES; ++t) {
        ok = mbar_wait(smem_u32(pfull + t), (uint32_t)(j & 1), abort_flag, s_status, WAIT_CROSS_TC + 0x50 + t, WAIT_LIMIT);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        tc_fence_after();
        if (issuer) {
#pragma unroll
          for (int k = 0; k < BN / 16; ++k)
            umma_bf16_ts(tmem + (uint32_t)(C::O_COL + t * D), tmem + (uint32_t)(t * BN + k * 8),
                         v0 + (uint64_t)vstage * (C::TILE_BYTES >> 4) + (uint64_t)(k * (16 * C::ROW >> 4)), PV, j > 0 || k > 0);
          if (j + 1 == n) umma_commit(smem_u32(ofull + t));
        }
        __syncwarp();
        if (j + 1 < n) scores(t, stage);
      }
      if (!ok) break;
      if (issuer) {
        umma_commit(smem_u32(vempty + vstage));
        if (j + 1 < n) umma_commit(smem_u32(kempty + stage));
      }
      __syncwarp();
      if (++vstage == STAGES) { vstage = 0; vphase ^= 1u; }
      if (++stage == STAGES) { stage = 0; phase ^= 1u; }
    }
  } else {
    // ------------------------------------------------------------------------------ weights
    const int t = warp >> 2, quarter = warp & 3, row = row0 + t * BM + quarter * 32 + lane;
    const uint32_t s_addr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(t * BN);
    const uint32_t o_addr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(C::O_COL + t * D);
    const float c = p.scale_log2;
    const unsigned long long c2 = pack2(c, c);
    float m = -INFINITY;
    unsigned long long l0 = pack2(0.f, 0.f), l1 = l0;
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(sfull + t), (uint32_t)(j & 1), abort_flag, s_status, WAIT_CROSS_TC + 0x60 + t, WAIT_LIMIT));
      if (!ok) break;
      tc_fence_after();
      uint32_t v[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32_async(s_addr + 32 * i, v[i]);
      tmem_wait_ld();
      const int rem = keys - j * BN;
      if (rem < BN) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < 32; ++x)
            if (32 * i + x >= rem) v[i][x] = 0xFF800000u;
      }
      float top[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top[i] = __uint_as_float(v[i][0]);
#pragma unroll
        for (int x = 1; x < 31; x += 2) top[i] = max3(top[i], __uint_as_float(v[i][x]), __uint_as_float(v[i][x + 1]));
        top[i] = fmaxf(top[i], __uint_as_float(v[i][31]));
      }
      const float now = fmaxf(max3(top[0], top[1], top[2]), top[3]);
      // the maximum only moves when a weight would pass 2^8: until then the sums keep their scale, which loses nothing in fp32
      const bool moved = (now - m) * c > 8.f;
      if (__any_sync(0xffffffffu, moved)) {
        if (j > 0) {
          const float fade = moved ? exp2_fast((m - now) * c) : 1.f;
          const unsigned long long f2 = pack2(fade, fade);
          l0 = mul2_of(l0, f2);
          l1 = mul2_of(l1, f2);
#pragma unroll 1
          for (int i = 0; i < D / 8; ++i) {
            uint32_t o[8];
            tmem_ld8(o_addr + 8 * i, o);
#pragma unroll
            for (int x = 0; x < 8; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * fade);
            tmem_st8(o_addr + 8 * i, o);
          }
        }
        if (moved) m = now;
      }
      const float mc = m == -INFINITY ? 0.f : -m * c;
      const unsigned long long mc2 = pack2(mc, mc);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          float lo, hi;
          unpack2(fma2_of(pack2(__uint_as_float(v[i][2 * x]), __uint_as_float(v[i][2 * x + 1])), c2, mc2), lo, hi);
          lo = exp2_fast(lo);
          hi = exp2_fast(hi);
          if (x & 1) l1 = add2_of(l1, pack2(lo, hi));
          else l0 = add2_of(l0, pack2(lo, hi));
          w[x] = pack_bf16(lo, hi);
        }
        tmem_st16(s_addr + 16 * i, w);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(pfull + t));
    }
    if (ok) {
      float inv = 0.f;
      if (n > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(ofull + t), 0, abort_flag, s_status, WAIT_CROSS_TC + 0x70 + t, WAIT_LIMIT));
        tc_fence_after();
        float a0, a1, a2, a3;
        unpack2(l0, a0, a1);
        unpack2(l1, a2, a3);
        inv = 1.f / ((a0 + a1) + (a2 + a3));
      }
      if (ok) {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + (int64_t)row * p.o.t + h * p.o.h;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          uint32_t o[32];
          if (n > 0) tmem_ld32(o_addr + 32 * i, o);
          if (row < rows) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              uint4 u = make_uint4(0u, 0u, 0u, 0u);
              if (n > 0) {
                auto two = [&](int y) { return pack_bf16(__uint_as_float(o[8 * x + y]) * inv, __uint_as_float(o[8 * x + y + 1]) * inv); };
                u = make_uint4(two(0), two(2), two(4), two(6));
              }
              *reinterpret_cast<uint4*>(dst + 32 * i + 8 * x) = u;
            }
          }
        }
      }
    }
  }

  // ------------------------------------------------------------------------------- teardown
  __syncwarp();
  if (*abort_flag) {
    // a wait ran out: give copies and MMAs in flight time to land before their memory is released
    for (int i = 0; i < 64; ++i) __nanosleep(16000);
    if (threadIdx.x == 0 && p.status) atomicCAS(p.status, 0, *(volatile int*)s_status);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == TILES * 4 + 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::TMEM) : "memory");
  }
}

template <int D, int TILES>
cudaError_t launch(const CrossTcParams& p, int batch, cudaStream_t s) {
  using C = Cfg<D, TILES>;
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(cross_tc_kernel<D, TILES>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
  if (e != cudaSuccess) return e;
  cross_tc_kernel<D, TILES><<<dim3((unsigned)((p.q_tokens + BM * TILES - 1) / (BM * TILES)), (unsigned)p.heads, (unsigned)batch), C::THREADS, C::SMEM, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

bool token_map(TensorMap128* map, const View& v, int D, int tokens, int heads, int batch, int box_tokens) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  const Encode fn = reinterpret_cast<Encode>(tensor_map_encoder());
  if (!fn) return false;
  const int64_t stride[3] = {v.t, v.h, v.b};
  const int extent[3] = {tokens, heads, batch};
  cuuint64_t dims[4] = {(cuuint64_t)D, 1, 1, 1}, bytes[3];
  for (int i = 0; i < 3; ++i) {
    const bool one = extent[i] == 1 || stride[i] == 0;
    dims[i + 1] = one ? 1u : (cuuint64_t)extent[i];
    bytes[i] = one ? (cuuint64_t)D * 2u : (cuuint64_t)stride[i] * 2u;
  }
  const cuuint32_t box[4] = {(cuuint32_t)(D == 128 ? 64 : D), (cuuint32_t)box_tokens, 1, 1}, ones[4] = {1, 1, 1, 1};
  return fn(reinterpret_cast<CUtensorMap*>(map), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, v.p, dims, bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            D == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
cudaError_t launch_cross_tc(const CrossParams& c, int D, cudaStream_t s) {
  CrossTcParams p{};
  const int kv_heads = c.heads / c.group;
  if (!token_map(&p.map_q, c.q, D, c.q_tokens, c.heads, c.batch) ||
      (c.kv_tokens > 0 && (!token_map(&p.map_k, c.k, D, c.kv_tokens, kv_heads, c.batch) || !token_map(&p.map_v, c.v, D, c.kv_tokens, kv_heads, c.batch))))
    return cudaErrorInvalidValue;
  p.o = c.o; p.q_lengths = c.q_lengths; p.kv_lengths = c.kv_lengths; p.status = c.status;
  p.q_tokens = c.q_tokens; p.kv_tokens = c.kv_tokens; p.heads = c.heads; p.group = c.group;
  p.q_h = c.q.h != 0; p.q_b = c.q.b != 0; p.k_h = c.k.h != 0; p.k_b = c.k.b != 0; p.v_h = c.v.h != 0; p.v_b = c.v.b != 0;
  p.scale_log2 = c.scale_log2;
  return D == 32 ? launch<32, 1>(p, c.batch, s) : D == 64 ? launch<64, 1>(p, c.batch, s) : launch<128, 2>(p, c.batch, s);
}

}  // namespace tok
}  // namespace tt

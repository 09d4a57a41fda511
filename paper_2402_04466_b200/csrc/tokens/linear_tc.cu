// Linear attention over several bf16 tokens on the tensor cores (tt_linear_attention): chunks of 128 tokens.
//
// With the fp32 state S before a chunk, l the head's decay, tokens i, j counted from 0, m their number:
//   scores  A = Q K^T;   P_ij = l^(i-j) A_ij for i >= j, else 0
//   out_i   = scale * ( l^(i+1) (Q S)_i + (P V)_i )
//   state   S' = l^m S + K'^T V,  K'_j = l^(m-1-j) k_j
// The state stays in tensor memory as the fp32 accumulator of its own product, scaled in place before each chunk's is added.
#include "linear_common.cuh"
#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

typedef unsigned long long Two;        // two floats

constexpr int CT = 128;                // tokens of a chunk
constexpr int WORKERS = 8;             // warps that compute: two to a quarter of the tokens, for half of the columns each
constexpr int THREADS = WORKERS * 32 + 32;   // and one that loads and issues products

struct LinearTcParams {
  TensorMap128 map_q, map_k, map_v;    // [D][token][head][batch], box of 128 tokens
  LinearParams c;
  int32_t q_h, q_b, k_h, k_b, v_h, v_b;   // 0 where the axis is shared, else 1
};

template <int D, bool WITH_OUT>
struct Cfg {
  static constexpr int ROW = D == 32 ? 64 : 128;                    // bytes of a row in a slab
  static constexpr int SLABS = D == 128 ? 2 : 1;
  static constexpr int SLAB_BYTES = CT * ROW;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;             // 128 tokens of one operand
  static constexpr int STATE_SLAB = D * ROW, STATE_BYTES = SLABS * STATE_SLAB;
  static constexpr uint32_t LAYOUT = D == 32 ? 4u : 2u;             // 64- or 128-byte swizzle
  static constexpr int M = D == 128 ? 128 : 64;                     // rows of the state's product
  static constexpr uint32_t O_COL = CT, S_COL = WITH_OUT ? CT + D : 0;
  static constexpr uint32_t COLS = S_COL + D;
  static constexpr uint32_t TMEM = COLS <= 32 ? 32 : COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static constexpr int TABLE_BYTES = (CT + 4) * 4 + 128;
  static constexpr int SMEM = (WITH_OUT ? 5 : 4) * TILE_BYTES + (WITH_OUT ? STATE_BYTES : 0) + TABLE_BYTES + 128 + 1024;
  static constexpr int BLOCKS = D == 128 ? 1 : WITH_OUT ? 2 : 3;
  static_assert(SMEM * BLOCKS <= 227 * 1024, "shared memory");
};

template <int D, bool WITH_OUT>
__global__ void __launch_bounds__(THREADS, Cfg<D, WITH_OUT>::BLOCKS) linear_tc_kernel(const __grid_constant__ LinearTcParams pp) {
  using C = Cfg<D, WITH_OUT>;
  const LinearParams& p = pp.c;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* s_k = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);   // the keys, then K' first term
  uint8_t* s_k1 = s_k + C::TILE_BYTES;                                                           // second and third term
  uint8_t* s_k2 = s_k1 + C::TILE_BYTES;
  uint8_t* s_v = s_k2 + C::TILE_BYTES;
  uint8_t* s_q = s_v + C::TILE_BYTES;                                                            // WITH_OUT only, as the next
  uint8_t* s_s = s_q + (WITH_OUT ? C::TILE_BYTES : 0);                                           // the state as an operand, rows along K
  float* pw = reinterpret_cast<float*>(s_s + (WITH_OUT ? C::STATE_BYTES : 0));                   // decay^0 .. decay^128
  float* pr = pw + CT + 4;                                                                       // decay^31 .. decay^0
  uint64_t* qfull = reinterpret_cast<uint64_t*>(pr + 32);
  uint64_t* kfull = qfull + 1;
  uint64_t* vfull = kfull + 1;
  uint64_t* first = vfull + 1;         // scores and Q S are there
  uint64_t* second = first + 1;        // out and state are there
  uint64_t* pready = second + 1;       // P, K', scaled accumulators
  uint64_t* sready = pready + 1;       // the state is an operand, out has been read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sready + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_status = reinterpret_cast<int*>(tmem_slot + 2);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x;
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;
  const int len = clamp_length(p.lengths, b, p.tokens), t0 = seg * p.seg_tokens, t1 = min(len, t0 + p.seg_tokens);
  if (WITH_OUT ? seg > 0 && t0 >= len : t0 + p.seg_tokens >= len) return;      // what the last segment adds is not needed
  const int chunks = (t1 - t0 + CT - 1) / CT;
  const int64_t at = ((int64_t)slot * p.heads + h) * D * D;
  float* seg_state = p.segments > 1 ? p.seg_state + (((int64_t)b * p.heads + h) * p.segments + seg) * D * D : nullptr;
  const float* from = p.segments > 1 ? seg_state : p.state + at;
  if (chunks == 0) {                   // an entry without tokens: its state as it was
    if (WITH_OUT && p.state_out + at != from)
      for (int i = threadIdx.x; i < D * D; i += THREADS) p.state_out[at + i] = from[i];
    return;
  }
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(qfull), 1);
    mbar_init(smem_u32(kfull), 1);
    mbar_init(smem_u32(vfull), 1);
    mbar_init(smem_u32(first), 1);
    mbar_init(smem_u32(second), 1);
    mbar_init(smem_u32(pready), WORKERS);
    mbar_init(smem_u32(sready), WORKERS);
    *abort_flag = 0;
    *s_status = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == WORKERS) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const float log_decay = p.log_decay[h];
  if (threadIdx.x < CT + 1) pw[threadIdx.x] = decay_power(log_decay, threadIdx.x);
  if (threadIdx.x < 32) pr[threadIdx.x] = decay_power(log_decay, 31 - threadIdx.x);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == WORKERS) {
    // ----------------------------------------------------------------- loads and products
    const bool issuer = elect_one();
    const int hk = h / p.group;
    auto load = [&](uint8_t* dst, const void* map, uint64_t* bar, int t, int hh, int bb) {
      mbar_arrive_expect_tx(smem_u32(bar), C::TILE_BYTES);
      for (int s = 0; s < C::SLABS; ++s) tma_load_4d(smem_u32(dst + s * C::SLAB_BYTES), map, smem_u32(bar), s * 64, t, hh, bb);
    };
    auto load_q = [&](int c) { if (WITH_OUT && issuer) load(s_q, &pp.map_q, qfull, t0 + c * CT, h * pp.q_h, b * pp.q_b); };
    auto load_k = [&](int c) { if (issuer) load(s_k, &pp.map_k, kfull, t0 + c * CT, hk * pp.k_h, b * pp.k_b); };
    auto load_v = [&](int c) { if (issuer) load(s_v, &pp.map_v, vfull, t0 + c * CT, hk * pp.v_h, b * pp.v_b); };
    load_q(0);
    load_k(0);
    load_v(0);
    __syncwarp();
    constexpr uint32_t QK = make_idesc(CT, CT), QS = make_idesc(CT, D) | B_BY_ROWS, PV = QS, KV = make_idesc(C::M, D) | A_BY_ROWS | B_BY_ROWS;
    const uint64_t q0 = make_smem_desc(smem_u32(s_q), 8 * C::ROW, C::LAYOUT), k0 = make_smem_desc(smem_u32(s_k), 8 * C::ROW, C::LAYOUT);
    const uint64_t st0 = make_rows_desc(smem_u32(s_s), C::STATE_SLAB, 8 * C::ROW, C::LAYOUT);
    const uint64_t v0 = make_rows_desc(smem_u32(s_v), C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    const uint64_t kr0 = make_rows_desc(smem_u32(s_k), C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    bool ok = true;
    auto wait = [&](uint64_t* bar, int c, int code) {
      ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(bar), (uint32_t)(c & 1), abort_flag, s_status, WAIT_LINEAR_TC + code, WAIT_LIMIT));
      return ok;
    };
    for (int c = 0; c < chunks; ++c) {
      if (WITH_OUT) {
        if (!wait(qfull, c, 0x00) || !wait(kfull, c, 0x01) || !wait(sready, c, 0x02)) break;
        tc_fence_after();
        if (issuer) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t o = (uint64_t)((k / 4) * (C::SLAB_BYTES >> 4) + (k % 4) * 2);
            umma_bf16(tmem, q0 + o, k0 + o, QK, k > 0);
          }
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t o = (uint64_t)((k / 4) * (C::SLAB_BYTES >> 4) + (k % 4) * 2);
            umma_bf16(tmem + C::O_COL, q0 + o, st0 + (uint64_t)(k * C::ROW), QS, k > 0);
          }
          umma_commit(smem_u32(first));
        }
        __syncwarp();
        if (!wait(first, c, 0x03)) break;
        if (c + 1 < chunks) load_q(c + 1);
        __syncwarp();
      }
      if (!wait(pready, c, 0x04)) break;
      tc_fence_after();
      if (issuer) {
        if (WITH_OUT) {
#pragma unroll
          for (int k = 0; k < CT / 16; ++k) umma_bf16_ts(tmem + C::O_COL, tmem + (uint32_t)(k / 4 * 64 + k % 4 * 8), v0 + (uint64_t)(k * C::ROW), PV, 1);
        }
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
          for (int k = 0; k < CT / 16; ++k)
            umma_bf16(tmem + C::S_COL, kr0 + (uint64_t)(term * (C::TILE_BYTES >> 4) + k * C::ROW), v0 + (uint64_t)(k * C::ROW), KV,
                      WITH_OUT || c > 0 || term > 0 || k > 0);
        umma_commit(smem_u32(second));
      }
      __syncwarp();
      if (!wait(second, c, 0x05)) break;
      if (c + 1 < chunks) {
        load_k(c + 1);
        load_v(c + 1);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------------------------------------------------- the rest
    const int quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane;      // r: token of the chunk, lane of tensor memory
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    // row of the state in this lane: a product of 64 rows leaves 16 to each quarter's first lanes
    const int row = C::M == 128 ? r : quarter * 16 + (lane & 15);
    const bool has_row = (C::M == 128 || lane < 16) && row < D;
    bool ok = true;
    auto wait = [&](uint64_t* bar, int c, int code) {
      ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(bar), (uint32_t)(c & 1), abort_flag, s_status, WAIT_LINEAR_TC + code, WAIT_LIMIT));
      return ok;
    };
    auto arrive = [&](uint64_t* bar) {
      tc_fence_before();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    // the columns of state and sums that are this warp's: pieces of 16 from c0 on
    constexpr int PIECES = D / 32;
    const int c0 = half * (D / 2);
    // 16 columns of this lane's row of the state into the operand's rows
    auto put_state = [&](int col, const uint32_t (&v)[16]) {
      if (!has_row) return;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int run = (col & 63) / 8 + x, to = D == 32 ? run ^ ((row >> 1) & 3) : run ^ (row & 7);
        auto two = [&](int y) { return pack_bf16(__uint_as_float(v[8 * x + y]), __uint_as_float(v[8 * x + y + 1])); };
        *reinterpret_cast<uint4*>(s_s + (col / 64) * C::STATE_SLAB + row * C::ROW + to * 16) = make_uint4(two(0), two(2), two(4), two(6));
      }
    };
    // all of this warp's columns times f
    auto scale_columns = [&](uint32_t first, float f) {
      uint32_t v[PIECES][16];
#pragma unroll
      for (int i = 0; i < PIECES; ++i) tmem_ld16_async(lanes + first + (uint32_t)(c0 + 16 * i), v[i]);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
#pragma unroll
        for (int x = 0; x < 16; ++x) v[i][x] = __float_as_uint(__uint_as_float(v[i][x]) * f);
        tmem_st16(lanes + first + (uint32_t)(c0 + 16 * i), v[i]);
      }
    };
    if (WITH_OUT) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int col = c0 + 16 * i;
        uint32_t v[16];
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
          const float4 f = has_row ? *reinterpret_cast<const float4*>(from + row * D + col + x) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[x] = __float_as_uint(f.x); v[x + 1] = __float_as_uint(f.y); v[x + 2] = __float_as_uint(f.z); v[x + 3] = __float_as_uint(f.w);
        }
        tmem_st16(lanes + C::S_COL + (uint32_t)col, v);
        put_state(col, v);
      }
      tmem_wait_st();
      arrive(sready);
    }
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + h * p.o.h;
    for (int c = 0; c < chunks; ++c) {
      const int t = t0 + c * CT, m = min(CT, t1 - t);
      if (!wait(kfull, c, 0x10)) break;
      if (WITH_OUT) {
        if (!wait(first, c, 0x11)) break;
        tc_fence_after();
        // weights within the chunk: blocks of 32 columns below the diagonal, on it, and above it; either half lies over scores of its own
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int i = 2 * half + y;
          uint32_t w[16];
          if (i > quarter) {
#pragma unroll
            for (int x = 0; x < 16; ++x) w[x] = 0u;
          } else {
            uint32_t v[32];
            tmem_ld32(lanes + 32 * i, v);
            if (i < quarter) {
              const float f = pw[r - 32 * i - 31];      // decay^(r - j) = decay^(r - 32 i - 31) decay^(31 - (j - 32 i))
              const Two f2 = pack2(f, f);
#pragma unroll
              for (int x = 0; x < 16; x += 2) {
                const float4 g = *reinterpret_cast<const float4*>(pr + 2 * x);
                float a0, a1, a2, a3;
                unpack2(mul2_of(pack2(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1])), mul2_of(f2, pack2(g.x, g.y))), a0, a1);
                unpack2(mul2_of(pack2(__uint_as_float(v[2 * x + 2]), __uint_as_float(v[2 * x + 3])), mul2_of(f2, pack2(g.z, g.w))), a2, a3);
                w[x] = pack_bf16(a0, a1);
                w[x + 1] = pack_bf16(a2, a3);
              }
            } else {
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                const float lo = lane >= 2 * x ? __uint_as_float(v[2 * x]) * pw[lane - 2 * x] : 0.f;
                const float hi = lane >= 2 * x + 1 ? __uint_as_float(v[2 * x + 1]) * pw[lane - 2 * x - 1] : 0.f;
                w[x] = pack_bf16(lo, hi);
              }
            }
          }
          tmem_st16(lanes + 64 * half + 16 * y, w);
        }
        scale_columns(C::O_COL, pw[r + 1]);
      }
      if (WITH_OUT || c > 0) scale_columns(C::S_COL, pw[m]);
      // K' = decay^(m-1-r) k in three bf16 terms, 24 bits: the state is as good as fp32.  Runs of 16 bytes in a turned order, so that
      // eight rows of 128 bytes do not meet in the same banks; the swizzle moves runs within a row and need not be undone.
      const bool here = r < m;
      const float f = here ? pw[m - 1 - r] : 0.f;
      if (!wait(vfull, c, 0x12)) break;
      const Two f2 = pack2(f, f);
#pragma unroll
      for (int i = 0; i < C::SLABS * C::ROW / 32; ++i) {
        const int run = half * (C::SLABS * C::ROW / 32) + i, s = run / (C::ROW / 16);
        const int o = s * C::SLAB_BYTES + r * C::ROW + ((run + (D == 32 ? r >> 1 : r)) & (C::ROW / 16 - 1)) * 16;
        const uint4 u = *reinterpret_cast<const uint4*>(s_k + o);
        const uint32_t in[4] = {u.x, u.y, u.z, u.w};
        uint32_t a[3][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          Two y = mul2_of(pack2(__uint_as_float(in[x] << 16), __uint_as_float(in[x] & 0xFFFF0000u)), f2);
#pragma unroll
          for (int term = 0; term < 3; ++term) {
            float lo, hi;
            unpack2(y, lo, hi);
            a[term][x] = here ? pack_bf16(lo, hi) : 0u;
            if (term < 2) y = sub2_of(y, pack2(__uint_as_float(a[term][x] << 16), __uint_as_float(a[term][x] & 0xFFFF0000u)));
          }
        }
        *reinterpret_cast<uint4*>(s_k + o) = make_uint4(a[0][0], a[0][1], a[0][2], a[0][3]);
        *reinterpret_cast<uint4*>(s_k1 + o) = make_uint4(a[1][0], a[1][1], a[1][2], a[1][3]);
        *reinterpret_cast<uint4*>(s_k2 + o) = make_uint4(a[2][0], a[2][1], a[2][2], a[2][3]);
        // rows behind the last token may hold anything, and weights of 0 would make NaN of it
        if (!here) *reinterpret_cast<uint4*>(s_v + o) = make_uint4(0u, 0u, 0u, 0u);
      }
      tmem_wait_st();
      arrive(pready);
      if (!wait(second, c, 0x13)) break;
      tc_fence_after();
      const bool last = c + 1 == chunks;
      // the state first: the next chunk's products wait for it, and for out having been read
      if (WITH_OUT || last) {
        uint32_t v[PIECES][16], y[PIECES][16];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          tmem_ld16_async(lanes + C::S_COL + (uint32_t)(c0 + 16 * i), v[i]);
          if (WITH_OUT) tmem_ld16_async(lanes + C::O_COL + (uint32_t)(c0 + 16 * i), y[i]);
        }
        tmem_wait_ld();
        if (WITH_OUT && !last) {
#pragma unroll
          for (int i = 0; i < PIECES; ++i) put_state(c0 + 16 * i, v[i]);
          arrive(sready);
        }
        if (last && (!WITH_OUT || t1 == len) && has_row) {
          float* to = WITH_OUT ? p.state_out + at : seg_state;
#pragma unroll
          for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
              *reinterpret_cast<float4*>(to + row * D + c0 + 16 * i + x) =
                  make_float4(__uint_as_float(v[i][x]), __uint_as_float(v[i][x + 1]), __uint_as_float(v[i][x + 2]), __uint_as_float(v[i][x + 3]));
        }
        if (WITH_OUT && here) {
#pragma unroll
          for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              auto two = [&](int e) { return pack_bf16(__uint_as_float(y[i][8 * x + e]) * p.scale, __uint_as_float(y[i][8 * x + e + 1]) * p.scale); };
              *reinterpret_cast<uint4*>(out + (int64_t)(t + r) * p.o.t + c0 + 16 * i + 8 * x) = make_uint4(two(0), two(2), two(4), two(6));
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
  if (warp == WORKERS) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::TMEM) : "memory");
  }
}

template <int D>
cudaError_t launch(const LinearTcParams& p, cudaStream_t s) {
  static OncePerContext once;
  cudaError_t e = once([] {
    const cudaError_t r = cudaFuncSetAttribute(linear_tc_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, true>::SMEM);
    return r != cudaSuccess ? r : cudaFuncSetAttribute(linear_tc_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, false>::SMEM);
  });
  if (e != cudaSuccess) return e;
  const LinearParams& c = p.c;
  if (c.segments > 1) {
    linear_tc_kernel<D, false><<<dim3((unsigned)c.segments - 1, (unsigned)c.heads, (unsigned)c.batch), THREADS, Cfg<D, false>::SMEM, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess || (e = launch_linear_scan(c, D, s)) != cudaSuccess) return e;
  }
  linear_tc_kernel<D, true><<<dim3((unsigned)c.segments, (unsigned)c.heads, (unsigned)c.batch), THREADS, Cfg<D, true>::SMEM, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_linear_tc(const LinearParams& c, int D, cudaStream_t s) {
  LinearTcParams p{};
  const int kv_heads = c.heads / c.group;
  if (!token_map(&p.map_q, c.q, D, c.tokens, c.heads, c.batch) || !token_map(&p.map_k, c.k, D, c.tokens, kv_heads, c.batch) ||
      !token_map(&p.map_v, c.v, D, c.tokens, kv_heads, c.batch))
    return cudaErrorInvalidValue;
  p.c = c;
  p.q_h = c.q.h != 0; p.q_b = c.q.b != 0; p.k_h = c.k.h != 0; p.k_b = c.k.b != 0; p.v_h = c.v.h != 0; p.v_b = c.v.b != 0;
  return D == 32 ? launch<32>(p, s) : D == 64 ? launch<64>(p, s) : launch<128>(p, s);
}

}  // namespace tok
}  // namespace tt

// Cross attention of many bf16 queries on the tensor cores (tt_cross_attention without a mask).
//
//   S = Q K^T (tiles of 128 queries x 64 or 128 keys),  P = 2^(c S - c m),  O += P V,  l += sum P,  c = scale * log2(e)
//
// A thread owns a query's row: its scores come from tensor memory into registers, its weights go back there as the second product's
// operand, the sums O stay there.  The running maximum m only moves when a weight would pass 2^8, so O is hardly ever rescaled.
// The work is tiles of queries x tiles of keys; a block takes an equal run of it, whatever tiles that cuts in two (a
// grid of one block per tile left half of the device idle in its last round), and where a tile is cut its blocks
// leave partial sums that cross_tc_join_kernel adds in order.
//
// Bound by the warps that turn scores into weights: the exponentials alone (16 a cycle and multiprocessor) take 1024 cycles for a
// tile of 128 x 128 whose two products take 512 with heads of 64 and 1024 with heads of 128.  Eight entries of 4 heads of 64, 4800 queries on
// 4800 keys: 276 us, 684 TFLOP/s, 1690 cycles a tile of 128 x 128; four entries of 2 heads of 128, 4800 queries on 9000 to 14400 keys: 226 us, 1018
// TFLOP/s.  Weights are rounded to bf16 once, as far as out itself is; their sum is of the weights before that.
#include "tokens.h"

#include <cuda.h>

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int BM = 128;                      // queries of a tile
constexpr int MAX_ENTRIES = 256;             // of the batch in a launch: their work is added up in shared memory
constexpr int LEAST = 512;                   // keys to a block, at least: fewer cost more in the join than they save

struct CrossTcParams {
  TensorMap128 map_q, map_k, map_v;      // [D][token][head][batch], boxes of 128 queries and of BN keys
  View o;
  const int32_t* q_lengths;
  const int32_t* kv_lengths;
  float* part;                           // two places a block: rows' maximum and total, then their sums
  int32_t* status;
  int32_t q_tokens, kv_tokens, heads, group, batch, b0;   // entries b0 .. b0 + batch - 1
  int32_t q_h, q_b, k_h, k_b, v_h, v_b;  // 0 where the axis is shared, else 1
  float scale_log2;
};

template <int D>
struct Cfg {
  // Two tiles of queries to a block, one block to a multiprocessor; each tile has columns of tensor memory of its own for scores (BN),
  // weights (BN / 2) and sums (D).
  static constexpr int TILES = 2, BN = D == 128 ? 64 : 128;
  // With heads of up to 64 the special-function units are what there is least of: the two tiles' warps of a quarter, which share one, take
  // turns at their exponentials, and one does the rest of its work meanwhile (276 us where both at once take 306; with heads of 128, whose
  // products take as long as the exponentials, 241 with turns and 226 without).
  static constexpr bool TURNS = D != 128;
  static constexpr int HALVES = BN / 64;                            // weights are handed over 64 keys at a time
  static constexpr int PLACES = D == 128 ? 2 : 1;                   // of a tile's weights: those of one tile of keys are made while the last ones' product runs
  static constexpr int ROWS = TILES * BM;
  static constexpr int ROW = D == 32 ? 64 : 128;                    // bytes of a row in a slab
  static constexpr int SLABS = D == 128 ? 2 : 1;
  static constexpr int Q_SLAB = BM * ROW, KV_SLAB = BN * ROW;
  static constexpr int Q_BYTES = SLABS * Q_SLAB, KV_BYTES = SLABS * KV_SLAB;
  static constexpr uint32_t LAYOUT = D == 32 ? 4u : 2u;             // 64- or 128-byte swizzle
  static constexpr int STAGES = 4;
  static constexpr int THREADS = TILES * (128 + 64);
  static constexpr uint32_t P_COL = TILES * BN, O_COL = P_COL + TILES * PLACES * BN / 2, TMEM = 512;
  static constexpr int SMEM = TILES * Q_BYTES + 2 * STAGES * KV_BYTES + 512 + 1024;
  static constexpr int64_t PART = (int64_t)ROWS * (D + 2);          // floats of a partial result
  static_assert(O_COL + TILES * D <= TMEM && SMEM + 6 * 1024 <= 227 * 1024, "tensor and shared memory");
};

// The launch's work: iterations (tile of queries x tile of keys) in the order entry, head, tile of queries, tile of keys.
struct Work {
  int64_t before[MAX_ENTRIES + 1];       // iterations before an entry's
  int32_t rows[MAX_ENTRIES], keys[MAX_ENTRIES];
};
template <int D>
__device__ __forceinline__ void add_up(Work& w, const CrossTcParams& p) {
  for (int i = threadIdx.x; i < p.batch; i += blockDim.x) {
    w.rows[i] = clamp_length(p.q_lengths, p.b0 + i, p.q_tokens);
    w.keys[i] = clamp_length(p.kv_lengths, p.b0 + i, p.kv_tokens);
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    int64_t sum = 0;
    for (int i0 = 0; i0 < p.batch; i0 += 32) {
      const int i = i0 + threadIdx.x;
      int64_t mine = i < p.batch ? (int64_t)((w.rows[i] + Cfg<D>::ROWS - 1) / Cfg<D>::ROWS) * p.heads * max(1, (w.keys[i] + Cfg<D>::BN - 1) / Cfg<D>::BN) : 0;
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t other = __shfl_up_sync(0xffffffffu, mine, o);
        if ((int)threadIdx.x >= o) mine += other;
      }
      if (i < p.batch) w.before[i + 1] = sum + mine;
      sum += __shfl_sync(0xffffffffu, mine, 31);
    }
    if (threadIdx.x == 0) w.before[0] = 0;
  }
  __syncthreads();
}
template <int D>
__device__ __forceinline__ int64_t share_of(const Work& w, const CrossTcParams& p) {
  const int64_t each = (w.before[p.batch] + gridDim.x - 1) / gridDim.x;
  return each < LEAST / Cfg<D>::BN ? LEAST / Cfg<D>::BN : each;
}

// A block's way through its work: the run it is at, and the step to the next.
struct Cursor {
  int64_t at, end;
  int b, h, row0, j0, j1, n;             // entry, head, first row; of the tile's n tiles of keys those from j0 to j1
  __device__ __forceinline__ bool done() const { return at >= end; }
  template <int D>
  __device__ __forceinline__ void find(const Work& w, const CrossTcParams& p) {
    if (done()) return;
    while (w.before[b + 1] <= at) ++b;
    n = max(1, (w.keys[b] + Cfg<D>::BN - 1) / Cfg<D>::BN);
    const int tiles = (w.rows[b] + Cfg<D>::ROWS - 1) / Cfg<D>::ROWS;
    const int64_t rel = at - w.before[b], t = rel / n;
    h = (int)(t / tiles);
    row0 = (int)(t - (int64_t)h * tiles) * Cfg<D>::ROWS;
    j0 = (int)(rel - t * n);
    j1 = (int)min((int64_t)n, j0 + (end - at));
  }
  template <int D>
  __device__ __forceinline__ void start(const Work& w, const CrossTcParams& p) {
    const int64_t each = share_of<D>(w, p);
    at = min((int64_t)blockIdx.x * each, w.before[p.batch]);
    end = min(at + each, w.before[p.batch]);
    b = 0;
    find<D>(w, p);
  }
  template <int D>
  __device__ __forceinline__ void next(const Work& w, const CrossTcParams& p) {
    at += j1 - j0;
    find<D>(w, p);
  }
};

template <int D>
__global__ void __launch_bounds__(Cfg<D>::THREADS, 1) cross_tc_kernel(const __grid_constant__ CrossTcParams p) {
  using C = Cfg<D>;
  constexpr int STAGES = C::STAGES, TILES = C::TILES;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Work work;
  uint8_t* s_q = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* s_k = s_q + TILES * C::Q_BYTES;
  uint8_t* s_v = s_k + STAGES * C::KV_BYTES;
  uint64_t* qfull = reinterpret_cast<uint64_t*>(s_v + STAGES * C::KV_BYTES);
  uint64_t* qempty = qfull + 1;                // the empty ones are signalled by every tile's warp
  uint64_t* kfull = qempty + 1;                // [STAGES]
  uint64_t* kempty = kfull + STAGES;           // [STAGES]
  uint64_t* vfull = kempty + STAGES;           // [STAGES]
  uint64_t* vempty = vfull + STAGES;           // [STAGES]
  uint64_t* sfull = vempty + STAGES;           // [TILES] scores are there, and the keys have been read
  uint64_t* sread = sfull + TILES;             // [TILES] scores are in registers
  uint64_t* pfull = sread + TILES;             // [TILES][PLACES][HALVES] weights are there, 64 keys each
  uint64_t* pdone = pfull + C::HALVES * C::PLACES * TILES;      // [TILES][PLACES] their product is done, and the values have been read
  uint64_t* turns = pdone + C::PLACES * TILES;      // [4][2] a quarter's turn at the exponentials: the other tile's warp has had its own
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(turns + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_status = reinterpret_cast<int*>(tmem_slot + 2);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(qfull), 1);
    mbar_init(smem_u32(qempty), TILES);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(kfull + s), 1);
      mbar_init(smem_u32(vfull + s), 1);
      mbar_init(smem_u32(kempty + s), TILES);
      mbar_init(smem_u32(vempty + s), TILES);
    }
    for (int t = 0; t < TILES; ++t) {
      mbar_init(smem_u32(sfull + t), 1);
      mbar_init(smem_u32(sread + t), 4);
      for (int x = 0; x < C::HALVES * C::PLACES; ++x) mbar_init(smem_u32(pfull + C::HALVES * C::PLACES * t + x), 4);
      for (int x = 0; x < C::PLACES; ++x) mbar_init(smem_u32(pdone + C::PLACES * t + x), 1);
    }
    for (int x = 0; x < 8; ++x) mbar_init(smem_u32(turns + x), 1);
    *abort_flag = 0;
    *s_status = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  add_up<D>(work, p);
  Cursor cur;
  cur.start<D>(work, p);
  if (cur.done()) return;                      // the whole block
  if (warp == TILES * 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();                     // the join gets ready meanwhile
  const uint32_t tmem = *tmem_slot;

  // the it-th weights of tile t: their place among all, and how often that has been used before
  auto at_place = [](int t, uint32_t it) { return t * C::PLACES + (int)(it & (C::PLACES - 1)); };
  auto turn = [](uint32_t it) { return C::PLACES == 2 ? it >> 1 : it; };
  bool ok = true;
  auto wait_all = [&](uint64_t* bar, uint32_t phase, int code) {      // a whole warp: its lanes go on or stop together
    if (__builtin_expect(__all_sync(0xffffffffu, mbar_test(smem_u32(bar), phase & 1u)), 1)) return true;
    ok = __all_sync(0xffffffffu, mbar_wait_uniform(smem_u32(bar), phase & 1u, abort_flag, s_status, WAIT_CROSS_TC + code, WAIT_LIMIT));
    return ok;
  };

  if (warp >= TILES * 4) {
    // ------------------------------------------------------------------------- loads and products
    // Two warps for each tile of queries: one issues the scores' products, the other the weights'; the first tile's also load queries and
    // keys, and values.  What an iteration costs here is latency: about 10 cycles an instruction, 50 a product, 200 a wait.  One warp for both
    // kinds took 3200 cycles an iteration, and the weights' warps waited for it half of the time.  Loops run on values that the compiler knows to be the whole
    // warp's (broadcast, or counted), waits are straight-line code, and lanes vote once an iteration.
    const bool issuer = elect_one();
    const int role = warp - TILES * 4, t = role >> 1;
    const bool keys = (role & 1) == 0, loads = t == 0;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), scores = tm + (uint32_t)(t * C::BN), weights = tm + C::P_COL + (uint32_t)(t * C::PLACES * (C::BN / 2)),
                   sums = tm + C::O_COL + (uint32_t)(t * D);
    auto arrived = [&](uint64_t* bar, uint32_t parity, int code) {
      if (__all_sync(0xffffffffu, mbar_test(smem_u32(bar), parity & 1u))) return;
      ok &= mbar_wait_uniform(smem_u32(bar), parity & 1u, abort_flag, s_status, WAIT_CROSS_TC + code, WAIT_LIMIT);
    };
    // tiles of keys are loaded STAGES ahead of their use: `ahead` is the next to load
    Cursor ahead = cur;
    int ab = __shfl_sync(0xffffffffu, p.b0 + ahead.b, 0), ah = __shfl_sync(0xffffffffu, ahead.h / p.group, 0), aj = __shfl_sync(0xffffffffu, ahead.j0, 0),
        left = __shfl_sync(0xffffffffu, ahead.j1 - ahead.j0, 0);      // of its run
    uint8_t* ring = keys ? s_k : s_v;
    uint64_t* full = keys ? kfull : vfull;
    const void* map = keys ? &p.map_k : &p.map_v;
    const int mul_h = keys ? p.k_h : p.v_h, mul_b = keys ? p.k_b : p.v_b;
    auto load_next = [&](uint32_t stage) {
      if (!loads || left == 0) return;
      if (issuer) {
        mbar_arrive_expect_tx(smem_u32(full + stage), C::KV_BYTES);
#pragma unroll
        for (int s = 0; s < C::SLABS; ++s)
          tma_load_4d(smem_u32(ring + stage * C::KV_BYTES + s * C::KV_SLAB), map, smem_u32(full + stage), s * 64, aj * C::BN, ah * mul_h, ab * mul_b);
      }
      ++aj;
      if (--left == 0) {                       // on to the next run
        ahead.next<D>(work, p);
        if (__shfl_sync(0xffffffffu, (int)ahead.done(), 0) == 0) {
          ab = __shfl_sync(0xffffffffu, p.b0 + ahead.b, 0);
          ah = __shfl_sync(0xffffffffu, ahead.h / p.group, 0);
          aj = __shfl_sync(0xffffffffu, ahead.j0, 0);
          left = __shfl_sync(0xffffffffu, ahead.j1 - ahead.j0, 0);
        }
      }
    };
    uint32_t stage = 0, phase = 0, runs = 0, it = 0;
    if (keys) {
      constexpr uint32_t QK = make_idesc(BM, C::BN);
      const uint64_t q0 = make_smem_desc(smem_u32(s_q + t * C::Q_BYTES), 8 * C::ROW, C::LAYOUT), k0 = make_smem_desc(smem_u32(s_k), 8 * C::ROW, C::LAYOUT);
      auto load_queries = [&]() {
        if (issuer && loads) {
          mbar_arrive_expect_tx(smem_u32(qfull), TILES * C::Q_BYTES);
          for (int i = 0; i < TILES; ++i)
            for (int s = 0; s < C::SLABS; ++s)
              tma_load_4d(smem_u32(s_q + i * C::Q_BYTES + s * C::Q_SLAB), &p.map_q, smem_u32(qfull), s * 64, cur.row0 + i * BM, cur.h * p.q_h, (p.b0 + cur.b) * p.q_b);
        }
        __syncwarp();
      };
      load_queries();
#pragma unroll
      for (int s = 0; s < STAGES; ++s) load_next(s);
      while (__shfl_sync(0xffffffffu, (int)cur.done(), 0) == 0) {
        const int n = __shfl_sync(0xffffffffu, cur.j1 - cur.j0, 0);
        arrived(qfull, runs++, 0x20);
        for (int j = 0; j < n; ++j, ++it) {
          arrived(full + stage, phase, 0x28 + (int)stage);
          if (it > 0) arrived(sread + t, it - 1, 0x30 + t);
          tc_fence_after();
          if (issuer) {
            const uint64_t kd = k0 + (uint64_t)stage * (C::KV_BYTES >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_bf16(scores, q0 + (uint64_t)((k / 4) * (C::Q_SLAB >> 4) + (k % 4) * 2), kd + (uint64_t)((k / 4) * (C::KV_SLAB >> 4) + (k % 4) * 2), QK, k > 0);
            umma_commit(smem_u32(sfull + t));
            umma_commit(smem_u32(kempty + stage));
            if (j + 1 == n) umma_commit(smem_u32(qempty));      // the run's queries have been read behind this product
          }
          if (j + 1 == n) cur.next<D>(work, p);
          // the tile's place is free when every tile of queries has read it (a parity of another tile's sfull would not do: that tile may
          // be two iterations ahead)
          if (loads) {
            arrived(kempty + stage, phase, 0x10 + (int)stage);
            load_next(stage);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          if (__any_sync(0xffffffffu, !ok)) break;
        }
        if (__any_sync(0xffffffffu, !ok)) break;
        if (__shfl_sync(0xffffffffu, (int)cur.done(), 0) == 0) {
          if (loads) arrived(qempty, runs - 1, 0x00);
          load_queries();
        }
      }
    } else {
      constexpr uint32_t PV = make_idesc(BM, D) | B_BY_ROWS;
      const uint64_t v0 = make_rows_desc(smem_u32(s_v), C::KV_SLAB, 8 * C::ROW, C::LAYOUT);
#pragma unroll
      for (int s = 0; s < STAGES; ++s) load_next(s);
      while (__shfl_sync(0xffffffffu, (int)cur.done(), 0) == 0) {
        const int n = __shfl_sync(0xffffffffu, cur.j1 - cur.j0, 0);
        // keys of the run's last tile: fewer than BN where it is the last of all
        const int rem = __shfl_sync(0xffffffffu, work.keys[cur.b] - (cur.j1 - 1) * C::BN, 0);
        cur.next<D>(work, p);
        for (int j = 0; j < n; ++j, ++it) {
          arrived(full + stage, phase, 0x38 + (int)stage);
          if (j + 1 == n && rem < C::BN) {
            // rows behind the last key may hold anything, and their weights of 0 would make NaN of it
            for (int s = 0; s < C::SLABS; ++s)
              for (int i = rem * C::ROW + lane * 16; i < C::KV_SLAB; i += 512)
                *reinterpret_cast<uint4*>(s_v + stage * C::KV_BYTES + s * C::KV_SLAB + i) = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
          }
          const uint64_t vd = v0 + (uint64_t)stage * (C::KV_BYTES >> 4);
#pragma unroll
          for (int x = 0; x < C::HALVES; ++x) {
            arrived(pfull + C::HALVES * at_place(t, it) + x, turn(it), 0x40 + C::HALVES * t + x);
            tc_fence_after();
            if (issuer) {
#pragma unroll
              for (int k = 4 * x; k < 4 * x + 4; ++k)
                umma_bf16_ts(sums, weights + (uint32_t)((it & (C::PLACES - 1)) * (C::BN / 2) + k * 8), vd + (uint64_t)(k * C::ROW), PV, k > 0 ? 1u : j > 0 ? 1u : 0u);
            }
          }
          if (issuer) {
            umma_commit(smem_u32(pdone + at_place(t, it)));
            umma_commit(smem_u32(vempty + stage));
          }
          if (loads) {
            arrived(vempty + stage, phase, 0x18 + (int)stage);
            load_next(stage);
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1u; }
          if (__any_sync(0xffffffffu, !ok)) break;
        }
        if (__any_sync(0xffffffffu, !ok)) break;
      }
    }
  } else {
    // ------------------------------------------------------------------------------ weights
    const int t = warp >> 2, quarter = warp & 3, r = t * BM + quarter * 32 + lane;      // row of the block's tile
    const uint32_t s_addr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(t * C::BN);
    const uint32_t p_addr = tmem + ((uint32_t)(quarter * 32) << 16) + C::P_COL + (uint32_t)(t * C::PLACES * (C::BN / 2));
    const uint32_t o_addr = tmem + ((uint32_t)(quarter * 32) << 16) + C::O_COL + (uint32_t)(t * D);
    const float c = p.scale_log2;
    const unsigned long long c2 = pack2(c, c);
    uint32_t it = 0;
    while (ok && !cur.done()) {
      const int count = cur.j1 - cur.j0, last_keys = work.keys[cur.b] - (cur.j1 - 1) * C::BN;      // of the run's last tile: all of its places or fewer
      float m = -INFINITY;
      unsigned long long l[4] = {pack2(0.f, 0.f), pack2(0.f, 0.f), pack2(0.f, 0.f), pack2(0.f, 0.f)};      // four chains
      for (int j = 0; j < count; ++j, ++it) {
      if (!wait_all(sfull + t, it, 0x50 + t)) break;
      tc_fence_after();
      uint32_t v[C::BN / 32][32];
#pragma unroll
      for (int i = 0; i < C::BN / 32; ++i) tmem_ld32_async(s_addr + 32 * i, v[i]);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(sread + t));
      if (__builtin_expect(j + 1 == count && last_keys < C::BN, 0)) {
#pragma unroll
        for (int i = 0; i < C::BN / 32; ++i)
#pragma unroll
          for (int x = 0; x < 32; ++x)
            if (32 * i + x >= last_keys) v[i][x] = 0xFF800000u;
      }
      float top[C::BN / 32];
#pragma unroll
      for (int i = 0; i < C::BN / 32; ++i) {
        top[i] = max3(__uint_as_float(v[i][0]), __uint_as_float(v[i][1]), __uint_as_float(v[i][31]));
#pragma unroll
        for (int x = 2; x < 30; x += 2) top[i] = max3(top[i], __uint_as_float(v[i][x]), __uint_as_float(v[i][x + 1]));
        top[i] = max3(top[i], top[i], __uint_as_float(v[i][30]));
      }
      float now = max3(top[0], top[0], top[1]);
      if constexpr (C::BN == 128) now = max3(now, top[2], top[3]);
      // the product of the weights that lay here must be done
      if (it >= C::PLACES && !wait_all(pdone + at_place(t, it), turn(it) - 1, 0x58 + t)) break;
      // the maximum only moves when a weight would pass 2^8: until then the sums keep their scale, which loses nothing in fp32
      const bool moved = (now - m) * c > 8.f;
      if (__builtin_expect(__any_sync(0xffffffffu, moved), 0)) {
        if (j > 0) {
          // the sums are rescaled: the last product must be done as well
          if (C::PLACES > 1 && !wait_all(pdone + at_place(t, it - 1), turn(it - 1), 0x5C + t)) break;
          tc_fence_after();
          const float fade = moved ? exp2_fast((m - now) * c) : 1.f;
          const unsigned long long f2 = pack2(fade, fade);
#pragma unroll
          for (int x = 0; x < 4; ++x) l[x] = mul2_of(l[x], f2);
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
      // the first tile begins, then they alternate: both go through the same iterations
      if (C::TURNS && (t == 1 || it > 0) && !wait_all(turns + 2 * quarter + t, t == 1 ? it : it - 1, 0x64 + t)) break;
      const float mc = m == -INFINITY ? 0.f : -m * c;
      const unsigned long long mc2 = pack2(mc, mc);
#pragma unroll
      for (int i = 0; i < C::BN / 32; ++i) {
        uint32_t w[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          float lo, hi;
          const unsigned long long a = fma2_of(pack2(__uint_as_float(v[i][2 * x]), __uint_as_float(v[i][2 * x + 1])), c2, mc2);
          unpack2(a, lo, hi);
          lo = exp2_fast(lo);
          hi = exp2_fast(hi);
          l[x & 3] = add2_of(l[x & 3], pack2(lo, hi));
          w[x] = pack_bf16(lo, hi);
        }
        if (C::TURNS && i == C::BN / 32 - 2 && lane == 0) mbar_arrive(smem_u32(turns + 2 * quarter + 1 - t));      // the other's wait takes about as long as the rest
        __syncwarp();                  // its first lane has signalled
        tmem_st16(p_addr + (uint32_t)((it & (C::PLACES - 1)) * (C::BN / 2) + 16 * i), w);
        if (i & 1) {
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(pfull + C::HALVES * at_place(t, it) + (i >> 1)));
        }
      }
      }
      // the run's end
      if (!ok || !wait_all(pdone + at_place(t, it - 1), turn(it - 1), 0x60 + t)) break;
      tc_fence_after();
      float a0, a1;
      unpack2(add2_of(add2_of(l[0], l[1]), add2_of(l[2], l[3])), a0, a1);
      const float total = a0 + a1;
      const bool here = cur.row0 + r < work.rows[cur.b];
      if (cur.j0 == 0 && cur.j1 == cur.n) {
        const float inv = total == 0.f ? 0.f : 1.f / total;      // nothing seen: zeros
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + (p.b0 + cur.b) * p.o.b + (int64_t)(cur.row0 + r) * p.o.t + cur.h * p.o.h;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          uint32_t o[32];
          __syncwarp();                // only some lanes' rows are stored
          tmem_ld32(o_addr + 32 * i, o);
          if (here) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              auto two = [&](int y) { return pack_bf16(__uint_as_float(o[8 * x + y]) * inv, __uint_as_float(o[8 * x + y + 1]) * inv); };
              *reinterpret_cast<uint4*>(dst + 32 * i + 8 * x) = make_uint4(two(0), two(2), two(4), two(6));
            }
          }
        }
      } else {
        float* place = p.part + ((int64_t)blockIdx.x * 2 + (cur.j0 == 0)) * C::PART;
        reinterpret_cast<float2*>(place)[r] = make_float2(m * c, total);
        float* dst = place + 2 * C::ROWS + r * D;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          uint32_t o[32];
          __syncwarp();                // only some lanes' rows are stored
          tmem_ld32(o_addr + 32 * i, o);
          if (here) {
#pragma unroll
            for (int x = 0; x < 32; x += 4)
              *reinterpret_cast<float4*>(dst + 32 * i + x) = make_float4(__uint_as_float(o[x]), __uint_as_float(o[x + 1]), __uint_as_float(o[x + 2]), __uint_as_float(o[x + 3]));
          }
        }
      }
      cur.next<D>(work, p);
    }
  }

  // ------------------------------------------------------------------------------- teardown
  __syncwarp();
  if (*abort_flag) {
    // a wait ran out: give copies and MMAs in flight time to land before their memory is released
    for (int i = 0; i < 64; ++i) __nanosleep(16000);
  }
  tc_fence_before();
  __syncthreads();
  // behind the barrier: the first thread may have been through with its own work when another warp's wait ran out
  if (threadIdx.x == 0 && *abort_flag && p.status) atomicCAS(p.status, 0, *(volatile int*)s_status);
  if (warp == TILES * 4) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::TMEM) : "memory");
  }
}

// One block per block of the kernel above: if its run begins inside a tile and is the first to do so, it joins the tile's parts, from the
// run that the tile begins in (second place) to the one that it ends in (first places).  out = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.
template <int D>
__global__ void __launch_bounds__(256) cross_tc_join_kernel(const __grid_constant__ CrossTcParams p) {
  using C = Cfg<D>;
  __shared__ Work work;
  add_up<D>(work, p);
  Cursor cur;
  cur.start<D>(work, p);
  pdl_wait();                                  // also of blocks that have nothing to do: the grid ends behind the kernel above
  if (cur.done() || cur.j0 == 0) return;
  const int64_t each = share_of<D>(work, p), from = cur.at - cur.j0, first = from / each;
  if (first + 1 != blockIdx.x) return;
  const int64_t last = (from + cur.n - 1) / each;
  const float* before = p.part + (first * 2 + 1) * C::PART;
  constexpr int LANES = D / 4;
  for (int r = threadIdx.x / LANES + (int)blockIdx.y * (256 / LANES); r < C::ROWS && cur.row0 + r < work.rows[cur.b]; r += 256 / LANES * (int)gridDim.y) {
    const int d = threadIdx.x % LANES * 4;
    float2 st = reinterpret_cast<const float2*>(before)[r];
    float m = st.x, l = st.y;
    float4 o = *reinterpret_cast<const float4*>(before + 2 * C::ROWS + r * D + d);
    for (int64_t i = first + 1; i <= last; ++i) {
      const float* place = p.part + i * 2 * C::PART;
      st = reinterpret_cast<const float2*>(place)[r];
      const float4 x = *reinterpret_cast<const float4*>(place + 2 * C::ROWS + r * D + d);
      const float now = fmaxf(m, st.x), base = now == -INFINITY ? 0.f : now;
      const float f = exp2_fast(m - base), g = exp2_fast(st.x - base);
      m = now;
      l = l * f + st.y * g;
      o = make_float4(o.x * f + x.x * g, o.y * f + x.y * g, o.z * f + x.z * g, o.w * f + x.w * g);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.o.p) + (p.b0 + cur.b) * p.o.b + (int64_t)(cur.row0 + r) * p.o.t + cur.h * p.o.h + d;
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  }
}

// Blocks of a launch over `batch` entries: one to a multiprocessor, fewer where a block would get less than LEAST keys.
template <int D>
int64_t grid_of(int batch, int q_tokens, int kv_tokens, int heads) {
  using C = Cfg<D>;
  const int64_t most = (int64_t)PLAN_SMS, tiles = (int64_t)((q_tokens + C::ROWS - 1) / C::ROWS) * heads * batch, n = (kv_tokens + C::BN - 1) / C::BN;
  if (tiles >= most * (LEAST / C::BN)) return most;
  const int64_t blocks = (tiles * n + LEAST / C::BN - 1) / (LEAST / C::BN);
  return blocks < most ? blocks : most;
}

template <int D>
cudaError_t launch(CrossTcParams& p, int batch, cudaStream_t s) {      // (the join is launched ahead of the end of the kernel: two entries' 256 queries 24 us, behind it 26.5)
  using C = Cfg<D>;
  static OncePerContext once;
  cudaError_t e = once([] { return cudaFuncSetAttribute(cross_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); });
  if (e != cudaSuccess) return e;
  for (p.b0 = 0; p.b0 < batch; p.b0 += MAX_ENTRIES) {
    p.batch = batch - p.b0 < MAX_ENTRIES ? batch - p.b0 : MAX_ENTRIES;
    const unsigned blocks = (unsigned)grid_of<D>(p.batch, p.q_tokens, p.kv_tokens, p.heads);
    cross_tc_kernel<D><<<blocks, C::THREADS, C::SMEM, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    // eight blocks to a tile's rows: two entries' 256 queries of 4 heads of 64 on 4800 keys 24 us, with four 28 (eight maps 276 and 274)
    if ((e = launch_kernel(cross_tc_join_kernel<D>, dim3(blocks, 8), 256, 0, s, p, true)) != cudaSuccess) return e;
  }
  return cudaSuccess;
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
uint64_t cross_tc_scratch(int batch, int q_tokens, int kv_tokens, int heads, int D) {
  const int entries = batch < MAX_ENTRIES ? batch : MAX_ENTRIES;
  const int64_t floats = D == 32   ? grid_of<32>(entries, q_tokens, kv_tokens, heads) * Cfg<32>::PART
                         : D == 64 ? grid_of<64>(entries, q_tokens, kv_tokens, heads) * Cfg<64>::PART
                                   : grid_of<128>(entries, q_tokens, kv_tokens, heads) * Cfg<128>::PART;
  return (uint64_t)floats * 2u * 4u;
}

cudaError_t launch_cross_tc(const CrossParams& c, int D, cudaStream_t s) {
  CrossTcParams p{};
  const int kv_heads = c.heads / c.group, keys = D == 128 ? Cfg<128>::BN : Cfg<64>::BN;
  if (!token_map(&p.map_q, c.q, D, c.q_tokens, c.heads, c.batch) || !token_map(&p.map_k, c.k, D, c.kv_tokens, kv_heads, c.batch, keys) ||
      !token_map(&p.map_v, c.v, D, c.kv_tokens, kv_heads, c.batch, keys))
    return cudaErrorInvalidValue;
  p.o = c.o; p.q_lengths = c.q_lengths; p.kv_lengths = c.kv_lengths; p.part = c.part; p.status = c.status;
  p.q_tokens = c.q_tokens; p.kv_tokens = c.kv_tokens; p.heads = c.heads; p.group = c.group;
  p.q_h = c.q.h != 0; p.q_b = c.q.b != 0; p.k_h = c.k.h != 0; p.k_b = c.k.b != 0; p.v_h = c.v.h != 0; p.v_b = c.v.b != 0;
  p.scale_log2 = c.scale_log2;
  return D == 32 ? launch<32>(p, c.batch, s) : D == 64 ? launch<64>(p, c.batch, s) : launch<128>(p, c.batch, s);
}

}  // namespace tok
}  // namespace tt

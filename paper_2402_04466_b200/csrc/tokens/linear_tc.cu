// Linear attention over several bf16 tokens on the tensor cores (tt_linear_attention): chunks of 128 tokens.
//
// With the fp32 state S before a chunk, l the head's decay, tokens i, j counted from 0, m their number:
//   scores  A = Q K^T;   P_ij = l^(i-j) A_ij for i >= j, else 0
//   out_i   = scale * ( l^(i+1) (Q S)_i + (P V)_i )       (the two sums apart: a P V that is not finite is taken again, see own_sums)
//   state   S' = l^m S + K'^T V,  K'_j = l^(m-1-j) k_j      (formed as its transpose, V^T K')
// K' goes into the state's product as three bf16 terms, 24 bits, and the state is kept in fp32, in registers: the tensor cores cut a
// sum off where fp32 would round it, which over the chunks of a sequence left it 1.3e-6 too small.  So each product is one of a chunk (of two,
// where only the segment's sum is wanted) that starts from nothing.  P and, for Q S, a copy of the state
// are rounded to bf16 once each, as far as out itself is.
//
// A sequence is sequential in its chunks, and a chunk is a chain of copies, products and register work, 12 000 cycles when one follows the
// other (two blocks to a multiprocessor then took 125 us for eight maps of 14400 tokens, 4 heads of 64).  So one block holds the
// chunks of a sequence in flight: a warp loads, one issues the products of out (A), one those of the state (B), eight warps make P and out
// from scores and sums, and eight make K' and carry the state.  Scores, P V, operands and K' have two places each where
// the memory allows (heads of up to 64).  What is left in sequence is the state's product and its scaling.
//
// Those eight maps take 104 to 110 us by the machine, 33 of them the segments' sums and 4 the scan: 2.2 TB/s, 4800 cycles for a chunk's out and state.  What bounds it is
// not memory (36 us) but shared memory, 290 KB moved a chunk, of which K' is half, and the 16 warps that make operands of what the products left.
#include "linear_common.cuh"
#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int CT = 128;                // tokens of a chunk
constexpr int GROUP = 8;               // warps of a group: two to a quarter of the tokens, for half of the columns each
// warps: the state's group, B, loads, A, one that idles, out's group (whose first warp has to be a multiple of four: its quarter of tensor memory)
constexpr int W_B = GROUP, W_LOAD = GROUP + 1, W_A = GROUP + 2, W_OUT = GROUP + 4;

struct LinearTcParams {
  TensorMap128 map_q, map_k, map_v;    // [D][token][head][batch], box of 128 tokens
  LinearParams c;
  int32_t q_h, q_b, k_h, k_b, v_h, v_b;   // 0 where the axis is shared, else 1
};

template <int D, bool WITH_OUT>
struct Cfg {
  static constexpr int THREADS = (WITH_OUT ? W_OUT + GROUP : W_LOAD + 1) * 32;
  static constexpr int ROW = D == 32 ? 64 : 128;                    // bytes of a row in a slab
  static constexpr int SLABS = D == 128 ? 2 : 1;
  static constexpr int SLAB_BYTES = CT * ROW;
  static constexpr int TILE_BYTES = SLABS * SLAB_BYTES;             // 128 tokens of one operand
  static constexpr int STATE_SLAB = D * ROW, STATE_BYTES = SLABS * STATE_SLAB;
  static constexpr uint32_t LAYOUT = D == 32 ? 4u : 2u;             // 64- or 128-byte swizzle
  static constexpr int M = D == 128 ? 128 : 64;                     // rows of the state's product
  static constexpr int PLACES = WITH_OUT ? (D == 128 ? 1 : 2) : D == 128 ? 2 : 4;       // of operands, scores and sums
  static constexpr int KP_PLACES = D == 128 ? 1 : 2;                // of K'
  // Where only a segment's sum is wanted and heads are of up to 64, K's three terms are side by side, one operand of 3 D columns: the product is
  // 8 instructions, not 24.  Else the terms follow one another into the same sums.  (Side by side with out as well: 118 us where this took 107.)
  static constexpr bool SIDE = !WITH_OUT && D <= 64;
  static constexpr int N = SIDE ? 3 * D : D;                        // columns of the state's product
  // the state's product lies first, then scores (weights take the place of those of the same warps), P V and Q S
  static constexpr uint32_t A_COL = N, PV_COL = A_COL + (PLACES < 2 ? 1 : 2) * CT, QS_COL = PV_COL + PLACES * D;
  static constexpr int EVERY = WITH_OUT ? 1 : 2, S_PLACES = WITH_OUT ? 1 : 2;      // chunks to a product of the state, and places of such products
  static constexpr uint32_t COLS = WITH_OUT ? QS_COL + D : S_PLACES * N;
  static constexpr uint32_t TMEM = COLS <= 32 ? 32 : COLS <= 64 ? 64 : COLS <= 128 ? 128 : COLS <= 256 ? 256 : 512;
  static constexpr int TABLE_BYTES = (CT + 4) * 4 + 128;
  static constexpr int SMEM = (WITH_OUT ? 3 : 2) * PLACES * TILE_BYTES + 3 * KP_PLACES * TILE_BYTES + (WITH_OUT ? STATE_BYTES : 0) + TABLE_BYTES + 512 + 1024;
  static_assert(COLS <= 512 && SMEM <= 227 * 1024, "tensor and shared memory");
};

// out of token t, the r-th of its chunk, in N columns from `col` on, P V term by term on the fp32 units; q_s: what Q S contributes.
template <int D, int N>
__device__ __noinline__ void own_sums(const LinearParams& p, int b, int h, int t, int r, int col, const float* pw, const float (&q_s)[N]) {
  const int hk = h / p.group;
  const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q.p) + b * p.q.b + h * p.q.h + (int64_t)t * p.q.t;
  const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(p.k.p) + b * p.k.b + hk * p.k.h + (int64_t)(t - r) * p.k.t;
  const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v.p) + b * p.v.b + hk * p.v.h + (int64_t)(t - r) * p.v.t + col;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = q_s[i];
  for (int j = 0; j <= r; ++j) {
    float w = 0.f;
#pragma unroll 4
    for (int i = 0; i < D; ++i) w = fmaf(__bfloat162float(q[i]), __bfloat162float(k[j * p.k.t + i]), w);
    w *= p.scale * pw[r - j];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = fmaf(w, __bfloat162float(v[j * p.v.t + i]), sum[i]);
  }
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + h * p.o.h + (int64_t)t * p.o.t + col;
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = __float2bfloat16(sum[i]);
}

// Elements of a lane's part of the state behind the tokens from t0 to t1, taken token by token: keys' columns col + i where bit i of `which` is set, value column
// `row`.  from: the state before, or null.
template <int D>
__device__ __noinline__ void own_state(const LinearParams& p, int b, int h, int t0, int t1, const float* from, float* to, int col, int row, uint32_t which) {
  const int hk = h / p.group;
  const __nv_bfloat16* k = reinterpret_cast<const __nv_bfloat16*>(p.k.p) + b * p.k.b + hk * p.k.h + col;
  const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.v.p) + b * p.v.b + hk * p.v.h + row;
  const float decay = decay_power(p.log_decay[h], 1);
#pragma unroll 1
  for (int i = 0; which; ++i, which >>= 1) {
    if ((which & 1u) == 0u) continue;
    float s = from ? from[(col + i) * D + row] : 0.f;
    // a NaN stays one: a state that had gone bad before costs no time
    for (int t = t0; t < t1 && !isnan(s); t += 8)
      for (int x = t; x < min(t + 8, t1); ++x) s = fmaf(s, decay, __bfloat162float(k[x * p.k.t + i]) * __bfloat162float(v[x * p.v.t]));
    to[(col + i) * D + row] = s;
  }
}

template <int D, bool WITH_OUT>
__global__ void __launch_bounds__(Cfg<D, WITH_OUT>::THREADS, 1) linear_tc_kernel(const __grid_constant__ LinearTcParams pp) {
  using C = Cfg<D, WITH_OUT>;
  constexpr int PLACES = C::PLACES, KPP = C::KP_PLACES;
  const LinearParams& p = pp.c;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* s_k = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* s_v = s_k + PLACES * C::TILE_BYTES;
  // K': [KPP][three terms].  It lies behind the values: heads of 32 fill half of the 64 rows of the state's product, and the other half is
  // read, for nothing, from one slab further on, which has to be the block's own memory.
  uint8_t* s_kp = s_v + PLACES * C::TILE_BYTES;
  uint8_t* s_q = s_kp + 3 * KPP * C::TILE_BYTES;                     // WITH_OUT only, as the next
  uint8_t* s_s = s_q + (WITH_OUT ? PLACES * C::TILE_BYTES : 0);      // the state as an operand, rows along K
  float* pw = reinterpret_cast<float*>(s_s + (WITH_OUT ? C::STATE_BYTES : 0));   // decay^0 .. decay^128
  float* pr = pw + CT + 4;                                           // decay^31 .. decay^0
  uint64_t* qfull = reinterpret_cast<uint64_t*>(pr + 32);            // [PLACES], as the next five
  uint64_t* kfull = qfull + 4;
  uint64_t* vfull = kfull + 4;
  uint64_t* qempty = vfull + 4;        // scores and Q S are done
  uint64_t* kempty = qempty + 4;       // scores are done, K' is made
  uint64_t* vempty = kempty + 4;       // both products of V are done
  uint64_t* kready = vempty + 4;       // [KP_PLACES] K' is there
  uint64_t* sdone = kready + 2;        // [KP_PLACES] the state's product is done
  uint64_t* afull = sdone + 2;         // [PLACES] scores are there
  uint64_t* pready = afull + 2;        // [PLACES] P is there
  uint64_t* odone = pready + 2;        // P V and Q S are there
  uint64_t* oread = odone + 1;         // they are in registers
  uint64_t* sready = oread + 1;        // the state is an operand
  uint64_t* sread = sready + 1;        // [S_PLACES] the state's product is in registers
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sread + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* s_status = reinterpret_cast<int*>(tmem_slot + 2);

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x;
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;
  const int len = clamp_length(p.lengths, b, p.tokens), t0 = seg * p.seg_tokens, t1 = min(len, t0 + p.seg_tokens);
  if (WITH_OUT ? seg > 0 && t0 >= len : t0 + p.seg_tokens >= len) return;      // what the last segment adds is not needed
  const int chunks = __shfl_sync(0xffffffffu, (t1 - t0 + CT - 1) / CT, 0);
  const int64_t at = ((int64_t)slot * p.heads + h) * D * D;
  float* seg_state = p.segments > 1 ? p.seg_state + (((int64_t)b * p.heads + h) * p.segments + seg) * D * D : nullptr;
  const float* from = p.segments > 1 ? seg_state : p.state + at;
  if (chunks == 0) {                   // an entry without tokens: its state as it was
    if (WITH_OUT && p.state_out + at != from)
      for (int i = threadIdx.x; i < D * D; i += C::THREADS) p.state_out[at + i] = from[i];
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < PLACES; ++s) {
      mbar_init(smem_u32(qfull + s), 1);
      mbar_init(smem_u32(kfull + s), 1);
      mbar_init(smem_u32(vfull + s), 1);
      mbar_init(smem_u32(qempty + s), 1);
      mbar_init(smem_u32(kempty + s), WITH_OUT ? GROUP + 1 : GROUP);
      mbar_init(smem_u32(vempty + s), WITH_OUT ? 2 : 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(afull + s), 1);
      mbar_init(smem_u32(pready + s), GROUP);
      mbar_init(smem_u32(sdone + s), 1);
      mbar_init(smem_u32(kready + s), GROUP);
      mbar_init(smem_u32(sread + s), GROUP);
    }
    mbar_init(smem_u32(odone), 1);
    mbar_init(smem_u32(oread), GROUP);
    mbar_init(smem_u32(sready), GROUP);
    *abort_flag = 0;
    *s_status = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == W_B) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  const float log_decay = p.log_decay[h];
  if (threadIdx.x < CT + 1) pw[threadIdx.x] = decay_power(log_decay, threadIdx.x);
  if (threadIdx.x < 32) pr[threadIdx.x] = decay_power(log_decay, 31 - threadIdx.x);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);

  bool ok = true;
  // A whole warp waits and stops together.  Each thing of chunk c is the c-th of its barrier, or the c / PLACES-th of its place's.  Only parities are
  // told apart: a barrier that may be two things ahead of one who waits for the first has a place for each.
  // (The wait behind the first look is the plain loop: the one whose first tries are straight-line code, of which there are twenty here, takes eight maps from 107 to
  // 110 us.)
  auto wait = [&](uint64_t* bar, int phase, int code) {
    if (__builtin_expect(__all_sync(0xffffffffu, mbar_test(smem_u32(bar), (uint32_t)phase & 1u)), 1)) return ok;
    ok = __all_sync(0xffffffffu, ok && mbar_wait(smem_u32(bar), (uint32_t)phase & 1u, abort_flag, s_status, WAIT_LINEAR_TC + code, WAIT_LIMIT));
    return ok;
  };
  auto place = [](int c) { return c & (PLACES - 1); };
  auto turn = [](int c) { return PLACES == 4 ? c >> 2 : PLACES == 2 ? c >> 1 : c; };
  auto kp_place = [](int c) { return KPP == 2 ? c & 1 : 0; };
  auto kp_turn = [](int c) { return KPP == 2 ? c >> 1 : c; };
  // where only a segment's sum is wanted, its chunks are taken from the last to the first: their weights are then a product
  auto token_of = [&](int c) { return t0 + (WITH_OUT ? c : chunks - 1 - c) * CT; };

  if (warp == W_LOAD) {
    // ------------------------------------------------------------------------------ loads
    const bool issuer = elect_one();
    const int hk = h / p.group;
    auto load = [&](uint8_t* dst, const void* map, uint64_t* bar, int t, int hh, int bb) {
      mbar_arrive_expect_tx(smem_u32(bar), C::TILE_BYTES);
#pragma unroll
      for (int s = 0; s < C::SLABS; ++s) tma_load_4d(smem_u32(dst + s * C::SLAB_BYTES), map, smem_u32(bar), s * 64, t, hh, bb);
    };
    for (int c = 0; c < chunks; ++c) {
      const int s = place(c), t = token_of(c);
      if (c >= PLACES && !wait(kempty + s, turn(c) - 1, 0x00)) break;
      if (issuer) load(s_k + s * C::TILE_BYTES, &pp.map_k, kfull + s, t, hk * pp.k_h, b * pp.k_b);
      if (WITH_OUT) {
        if (c >= PLACES && !wait(qempty + s, turn(c) - 1, 0x01)) break;
        if (issuer) load(s_q + s * C::TILE_BYTES, &pp.map_q, qfull + s, t, h * pp.q_h, b * pp.q_b);
      }
      if (c >= PLACES && !wait(vempty + s, turn(c) - 1, 0x02)) break;
      if (issuer) load(s_v + s * C::TILE_BYTES, &pp.map_v, vfull + s, t, hk * pp.v_h, b * pp.v_b);
    }
  } else if (warp == W_B) {
    // --------------------------------------------------------------- products of the state
    const bool issuer = elect_one();
    constexpr uint32_t VK = make_idesc(C::M, C::N) | A_BY_ROWS | B_BY_ROWS;
    const uint64_t v0 = make_rows_desc(smem_u32(s_v), C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    // the terms' runs of columns are a tile apart, where they are one operand
    const uint64_t k0 = make_rows_desc(smem_u32(s_kp), C::SIDE ? C::TILE_BYTES : C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    for (int c = 0; c < chunks; ++c) {
      const int group = c / C::EVERY, at = group & (C::S_PLACES - 1);
      if (!wait(kready + kp_place(c), kp_turn(c), 0x10)) break;
      if (c % C::EVERY == 0 && group >= C::S_PLACES && !wait(sread + at, group / C::S_PLACES - 1, 0x12 + at)) break;
      tc_fence_after();
      if (issuer) {
        const uint64_t v = v0 + (uint64_t)(place(c) * (C::TILE_BYTES >> 4)), k = k0 + (uint64_t)(kp_place(c) * 3 * (C::TILE_BYTES >> 4));
        const uint32_t more = c % C::EVERY ? 1u : 0u, to = tmem + (uint32_t)(at * C::N);
        // the smallest terms first: the tensor cores cut their sums off, by a part of what the sum has grown to
#pragma unroll
        for (int term = C::SIDE ? 0 : 2; term >= 0; --term)
#pragma unroll
          for (int i = 0; i < CT / 16; ++i)
            umma_bf16(to, v + (uint64_t)(i * C::ROW), k + (uint64_t)(term * (C::TILE_BYTES >> 4) + i * C::ROW), VK, i > 0 || term < (C::SIDE ? 0 : 2) ? 1u : more);
        umma_commit(smem_u32(sdone + kp_place(c)));
        umma_commit(smem_u32(vempty + place(c)));
      }
      __syncwarp();
    }
    // the last commits arrive before the block goes
    if (ok) wait(vempty + place(chunks - 1), turn(chunks - 1), 0x11);
  } else if (WITH_OUT && warp == W_A) {
    // ------------------------------------------------------------------- products of out
    const bool issuer = elect_one();
    constexpr uint32_t QK = make_idesc(CT, CT), QS = make_idesc(CT, D), PV = QS | B_BY_ROWS;
    const uint64_t q0 = make_smem_desc(smem_u32(s_q), 8 * C::ROW, C::LAYOUT), k0 = make_smem_desc(smem_u32(s_k), 8 * C::ROW, C::LAYOUT);
    const uint64_t st0 = make_smem_desc(smem_u32(s_s), 8 * C::ROW, C::LAYOUT);      // rows are value columns, along them the keys'
    const uint64_t v0 = make_rows_desc(smem_u32(s_v), C::SLAB_BYTES, 8 * C::ROW, C::LAYOUT);
    auto scores = [&](int c) {
      const int s = place(c);
      if (!wait(qfull + s, turn(c), 0x20) || !wait(kfull + s, turn(c), 0x21)) return false;
      tc_fence_after();
      if (issuer) {
        const uint64_t o = (uint64_t)(s * (C::TILE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t x = (uint64_t)((k / 4) * (C::SLAB_BYTES >> 4) + (k % 4) * 2);
          umma_bf16(tmem + C::A_COL + (uint32_t)(s * CT), q0 + o + x, k0 + o + x, QK, k > 0);
        }
        umma_commit(smem_u32(afull + s));
        umma_commit(smem_u32(kempty + s));
      }
      __syncwarp();
      return true;
    };
    auto state_part = [&](int c) {     // Q S: the state is an operand, and the last chunk's Q S and P V have been read
      if (!wait(sready, c, 0x22) || (c > 0 && !wait(oread, c - 1, 0x23))) return false;
      tc_fence_after();
      if (issuer) {
        const uint64_t q = q0 + (uint64_t)(place(c) * (C::TILE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          umma_bf16(tmem + C::QS_COL, q + (uint64_t)((k / 4) * (C::SLAB_BYTES >> 4) + (k % 4) * 2), st0 + (uint64_t)((k / 4) * (C::STATE_SLAB >> 4) + (k % 4) * 2), QS, k > 0);
        umma_commit(smem_u32(qempty + place(c)));
      }
      __syncwarp();
      return true;
    };
    scores(0);
    for (int c = 0; c < chunks && ok; ++c) {
      const int s = place(c);
      // with two places the next scores are formed meanwhile, where the last but one's weights have been used
      if (PLACES == 2 && c + 1 < chunks && ((c > 0 && !wait(odone, c - 1, 0x25)) || !scores(c + 1))) break;
      if (PLACES == 1 && !state_part(c)) break;
      // the values have landed, and their rows behind the last token are zeros, when K' is there
      if (!wait(kready + kp_place(c), kp_turn(c), 0x27) || !wait(pready + s, turn(c), 0x24)) break;
      tc_fence_after();
      if (issuer) {
        const uint64_t v = v0 + (uint64_t)(s * (C::TILE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < CT / 16; ++k)
          umma_bf16_ts(tmem + C::PV_COL + (uint32_t)(s * D), tmem + C::A_COL + (uint32_t)(s * CT + (k >> 2) * 64 + (k & 3) * 8), v + (uint64_t)(k * C::ROW), PV, k > 0);
        umma_commit(smem_u32(vempty + s));
      }
      __syncwarp();
      if (PLACES == 2 && !state_part(c)) break;
      if (issuer) umma_commit(smem_u32(odone));
      __syncwarp();
      if (PLACES == 1 && c + 1 < chunks && (!wait(odone, c, 0x26) || !scores(c + 1))) break;
    }
  } else if (WITH_OUT && warp >= W_OUT) {
    // ---------------------------------------------------------------------------- P and out
    const int quarter = warp & 3, half = (warp - W_OUT) >> 2, r = quarter * 32 + lane;      // r: token of the chunk, lane of tensor memory
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    constexpr int PIECES = D / 32;     // of 16 columns, from c0 on
    const int c0 = half * (D / 2);
    const float scale = p.scale;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.o.p) + b * p.o.b + h * p.o.h;
    auto arrive = [&](uint64_t* bar) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    auto store = [&](int c) {          // out of chunk c, whose products are there
      tc_fence_after();
      const int t = t0 + c * CT + r;
      const float f = scale * pw[r + 1];
      const Two f2 = pack2(f, f);
      constexpr int BATCH = PIECES == 2 ? 2 : 1;      // pieces at a time
#pragma unroll
      for (int i0 = 0; i0 < PIECES; i0 += BATCH) {
        uint32_t y[BATCH][16], z[BATCH][16];
        __syncwarp();                  // lanes whose token is none, or whose sums were taken again, have parted from the rest
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          tmem_ld16_async(lanes + C::PV_COL + (uint32_t)(place(c) * D + c0 + 16 * (i0 + i)), y[i]);
          tmem_ld16_async(lanes + C::QS_COL + (uint32_t)(c0 + 16 * (i0 + i)), z[i]);
        }
        tmem_wait_ld();
        if (i0 + BATCH == PIECES) arrive(oread);
        Two bad = pack2(0.f, 0.f);     // stays 0 unless one of P V is an infinity or NaN
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
#pragma unroll
          for (int x = 0; x < 16; x += 2) bad = fma2_of(pack2(__uint_as_float(y[i][x]), __uint_as_float(y[i][x + 1])), pack2(0.f, 0.f), bad);
        float b0, b1;
        unpack2(bad, b0, b1);
        if (t >= t1) continue;
        // the weights of 0 behind a token make NaN of what is not finite in a later token's values: such sums are taken again, of the tokens up to this
        // one only
        const bool again = b0 + b1 != 0.f;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          __nv_bfloat16* dst = out + (int64_t)t * p.o.t + c0 + 16 * (i0 + i);
#pragma unroll
          for (int x = 0; x < 16; x += 2) {
            float lo, hi;
            unpack2(fma2_of(pack2(__uint_as_float(z[i][x]), __uint_as_float(z[i][x + 1])), f2, pack2(__uint_as_float(y[i][x]), __uint_as_float(y[i][x + 1]))), lo, hi);
            y[i][x / 2] = pack_bf16(lo, hi);
          }
          *reinterpret_cast<uint4*>(dst) = make_uint4(y[i][0], y[i][1], y[i][2], y[i][3]);
          *reinterpret_cast<uint4*>(dst + 8) = make_uint4(y[i][4], y[i][5], y[i][6], y[i][7]);
        }
        if (__builtin_expect(again, 0)) {
          float a[16 * BATCH];
#pragma unroll
          for (int i = 0; i < BATCH; ++i)
#pragma unroll
            for (int x = 0; x < 16; ++x) a[16 * i + x] = __uint_as_float(z[i][x]) * f;
          own_sums<D>(p, b, h, t, r, c0 + 16 * i0, pw, a);
        }
      }
    };
    for (int c = 0; c < chunks; ++c) {
      const int s = place(c);
      if (!wait(afull + s, turn(c), 0x31)) break;
      tc_fence_after();
      // weights within the chunk: blocks of 32 columns below the diagonal, on it, and above it
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int i = 2 * half + y;
        uint32_t w[16];
        if (i > quarter) {
#pragma unroll
          for (int x = 0; x < 16; ++x) w[x] = 0u;
        } else {
          uint32_t v[32];
          tmem_ld32(lanes + C::A_COL + (uint32_t)(s * CT + 32 * i), v);
          if (i < quarter) {
            const float f = scale * pw[r - 32 * i - 31];      // decay^(r - j) = decay^(r - 32 i - 31) decay^(31 - (j - 32 i))
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
              const float lo = lane >= 2 * x ? __uint_as_float(v[2 * x]) * (scale * pw[lane - 2 * x]) : 0.f;
              const float hi = lane >= 2 * x + 1 ? __uint_as_float(v[2 * x + 1]) * (scale * pw[lane - 2 * x - 1]) : 0.f;
              w[x] = pack_bf16(lo, hi);
            }
          }
        }
        __syncwarp();                  // on the diagonal every lane has weights of its own number
        tmem_st16(lanes + C::A_COL + (uint32_t)(s * CT + 64 * half + 16 * y), w);
      }
      tmem_wait_st();
      arrive(pready + s);
      // with two places the chunk before is stored while this one's product runs
      if (PLACES == 2) {
        if (c > 0) {
          if (!wait(odone, c - 1, 0x32)) break;
          store(c - 1);
        }
      } else {
        if (!wait(odone, c, 0x30)) break;
        store(c);
      }
    }
    if (PLACES == 2 && ok && wait(odone, chunks - 1, 0x34)) store(chunks - 1);
  } else if (warp < GROUP) {
    // ------------------------------------------------------------------------ K' and the state
    const int quarter = warp & 3, half = warp >> 2, r = quarter * 32 + lane;      // r: token of the chunk
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    // value column of the state in this lane (its columns are the keys'): a product of 64 rows leaves 16 to each quarter's first lanes
    const int row = C::M == 128 ? r : quarter * 16 + (lane & 15);
    const bool has_row = (C::M == 128 || lane < 16) && row < D;
    constexpr int PIECES = D / 32;     // of 16 columns, from c0 on
    const int c0 = half * (D / 2);
    auto arrive = [&](uint64_t* bar) {
      tc_fence_before();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(bar));
    };
    float S[PIECES][16];               // this lane's part of the state
    auto put_state = [&]() {           // into the operand's rows
      if (!has_row) return;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int col = c0 + 16 * i, run = (col & 63) / 8 + x, to = D == 32 ? run ^ ((row >> 1) & 3) : run ^ (row & 7);
          auto two = [&](int e) { return pack_bf16(S[i][8 * x + e], S[i][8 * x + e + 1]); };
          *reinterpret_cast<uint4*>(s_s + (col / 64) * C::STATE_SLAB + row * C::ROW + to * 16) = make_uint4(two(0), two(2), two(4), two(6));
        }
    };
    auto add_product = [&](int group, float g) {      // S = g S + product, which is done
      __syncwarp();
      tc_fence_after();
      const uint32_t from_col = lanes + (uint32_t)((group & (C::S_PLACES - 1)) * C::N + c0);
      if constexpr (C::SIDE) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          uint32_t y[3][16];
#pragma unroll
          for (int term = 0; term < 3; ++term) tmem_ld16_async(from_col + (uint32_t)(term * D + 16 * i), y[term]);
          tmem_wait_ld();
#pragma unroll
          for (int x = 0; x < 16; ++x) S[i][x] += __uint_as_float(y[0][x]) + (__uint_as_float(y[1][x]) + __uint_as_float(y[2][x]));
        }
      } else {
        uint32_t y[PIECES][16];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) tmem_ld16_async(from_col + (uint32_t)(16 * i), y[i]);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
          for (int x = 0; x < 16; ++x) S[i][x] = fmaf(S[i][x], g, __uint_as_float(y[i][x]));
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(sread + (group & (C::S_PLACES - 1))));
    };
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
      for (int x = 0; x < 16; ++x) S[i][x] = WITH_OUT && has_row ? from[(c0 + 16 * i + x) * D + row] : 0.f;
    float behind = 1.f;                // decay^(tokens behind the chunk), where only the sum is wanted
    for (int c = 0; c < chunks; ++c) {
      const int s = place(c), m = min(CT, t1 - token_of(c));
      // the K' that lay here has been used (with out and two places the state's wait below has seen to it)
      if (c >= KPP && (KPP == 1 || !WITH_OUT) && !wait(sdone + kp_place(c), kp_turn(c) - 1, 0x40)) break;
      // K' = decay^(m-1-r) k in three bf16 terms; where only the segment's sum is wanted, decay^(tokens behind it) k, and the state is never
      // scaled.  Runs of 16 bytes in a turned order, so that eight rows of 128 bytes do not meet in the same banks; the
      // swizzle moves runs within a row and need not be undone.
      const bool here = r < m;
      const float f = here ? pw[m - 1 - r] * behind : 0.f;
      if (!WITH_OUT) behind *= pw[CT];
      if (!wait(kfull + s, turn(c), 0x42) || !wait(vfull + s, turn(c), 0x43)) break;
      const Two f2 = pack2(f, f);
      const uint8_t* kk = s_k + s * C::TILE_BYTES;
      uint8_t* kp = s_kp + kp_place(c) * 3 * C::TILE_BYTES;
      // all reads come first: a store might, for all the compiler knows, change what a later read finds
      constexpr int RUNS = C::SLABS * C::ROW / 32;      // to a thread
      constexpr int BATCH = 2;
#pragma unroll
      for (int i0 = 0; i0 < RUNS; i0 += BATCH) {
        uint4 u[BATCH];
        int o[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const int run = half * RUNS + i0 + i, slab = run / (C::ROW / 16);
          o[i] = slab * C::SLAB_BYTES + r * C::ROW + ((run + (D == 32 ? r >> 1 : r)) & (C::ROW / 16 - 1)) * 16;
          u[i] = *reinterpret_cast<const uint4*>(kk + o[i]);
          if (!here) u[i] = make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          const uint32_t in[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
          uint32_t a[3][4];
          Two y[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) y[x] = mul2_of(pack2(__uint_as_float(in[x] << 16), __uint_as_float(in[x] & 0xFFFF0000u)), f2);
          // cut off, not rounded: three times eight bits are all of fp32's 24
#pragma unroll
          for (int term = 0; term < 3; ++term)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              float lo, hi;
              unpack2(y[x], lo, hi);
              a[term][x] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
              if (term < 2) y[x] = sub2_of(y[x], pack2(__uint_as_float(__float_as_uint(lo) & 0xFFFF0000u), __uint_as_float(__float_as_uint(hi) & 0xFFFF0000u)));
            }
#pragma unroll
          for (int term = 0; term < 3; ++term) *reinterpret_cast<uint4*>(kp + term * C::TILE_BYTES + o[i]) = make_uint4(a[term][0], a[term][1], a[term][2], a[term][3]);
          // rows behind the last token may hold anything, and weights of 0 would make NaN of it
          if (!here) *reinterpret_cast<uint4*>(s_v + s * C::TILE_BYTES + o[i]) = make_uint4(0u, 0u, 0u, 0u);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(kempty + s));
      arrive(kready + kp_place(c));
      if (WITH_OUT) {
        if (c > 0) {
          if (!wait(sdone + kp_place(c - 1), kp_turn(c - 1), 0x44)) break;
          add_product(c - 1, pw[CT]);
          if (!wait(odone, c - 1, 0x45)) break;      // the state's copy as an operand has been used
        }
        put_state();
        arrive(sready);
      } else if (c >= 3 && (c & 1)) {
        add_product((c - 3) / 2, 1.f);      // of chunks c - 3 and c - 2: the wait above has seen to them
      }
    }
    if (ok && wait(sdone + kp_place(chunks - 1), kp_turn(chunks - 1), 0x46)) {
      if (WITH_OUT) {
        add_product(chunks - 1, pw[t1 - token_of(chunks - 1)]);
      } else {
        for (int group = chunks < 2 ? 0 : (chunks - 2) / 2; group < (chunks + 1) / 2; ++group) add_product(group, 1.f);
      }
      if ((!WITH_OUT || t1 == len) && has_row) {
        float* to = WITH_OUT ? p.state_out + at : seg_state;
        Two bad[2] = {pack2(0.f, 0.f), pack2(0.f, 0.f)};      // two chains
#pragma unroll
        for (int i = 0; i < 16 * PIECES; i += 2) bad[i / 2 & 1] = fma2_of(pack2(S[i / 16][i % 16], S[i / 16][i % 16 + 1]), pack2(0.f, 0.f), bad[i / 2 & 1]);
        float b0, b1;
        unpack2(add2_of(bad[0], bad[1]), b0, b1);
        if (__builtin_expect(b0 + b1 == 0.f, 1)) {
#pragma unroll
          for (int i = 0; i < 16 * PIECES; ++i) to[(c0 + i) * D + row] = S[i / 16][i % 16];
        } else {
          // the terms that K' is cut into make NaN where k v is an infinity
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            uint32_t which = 0;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              if (isfinite(S[i][x])) to[(c0 + 16 * i + x) * D + row] = S[i][x];
              else which |= 1u << x;
            }
            own_state<D>(p, b, h, t0, t1, WITH_OUT ? from : nullptr, to, c0 + 16 * i, row, which);
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
  }
  tc_fence_before();
  __syncthreads();
  // behind the barrier: the first thread may have been through with its own work when another warp's wait ran out
  if (threadIdx.x == 0 && *abort_flag && p.status) atomicCAS(p.status, 0, *(volatile int*)s_status);
  if (warp == W_B) {
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
    linear_tc_kernel<D, false><<<dim3((unsigned)c.segments - 1, (unsigned)c.heads, (unsigned)c.batch), Cfg<D, false>::THREADS, Cfg<D, false>::SMEM, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess || (e = launch_linear_scan(c, D, s)) != cudaSuccess) return e;
  }
  linear_tc_kernel<D, true><<<dim3((unsigned)c.segments, (unsigned)c.heads, (unsigned)c.batch), Cfg<D, true>::THREADS, Cfg<D, true>::SMEM, s>>>(p);
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

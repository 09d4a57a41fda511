// The gated delta rule over several tokens, second part (tt_delta_rule): the chain of states, a window of 32 tokens at a time.
//
// With G_i the sum of log_decay up to and including token i of a window and T and P what delta_window.cuh works out,
//   R_i = beta_i (v_i - e^G_i S^T k_i),  U = T R,  out_i = scale e^G_i S^T q_i + sum_j P_ij u_j,  S' = e^G_C S + sum_j e^(G_C - G_j) k_j u_j^T.
// What bounds a sequence is the chain S -> R -> U -> S', not bytes and not the tensor pipe: instructions that wait for one another.  The columns of values are independent
// of each other: 16 of them are a run, and a run has one warp, or four where runs are few, that take its state along in registers, and one to four behind them that turn what the
// chain leaves into out, a window later for its last product.  Four more warps load, two windows and more ahead.  All of a block's warps meet once a window.
//
// Everything on the chain is kept transposed, columns of values along M: the accumulators of one m16n8k16 product are then the other operand's registers of the next,
// X^T = S^T K^T, U^T = R^T T^T, S'^T = U'^T K.  Four warps of a run split the keys' elements of the state and the tokens of R and U; what they exchange goes through shared memory as
// those registers.  Heads of 64, cycles a window: one warp 3300, two 2050, four 1600.  A tcgen05 product of 16
// columns takes 40 cycles however few its columns are, and its way through tensor memory twice that: the chain would be longer, not shorter.  Windows of 64 have four times the
// triangle (with the warps as they were then, 909 us to 748 for the same maps).
//
// Eight maps of 14400 tokens, 4 heads of 64: 410 us, of which reading and writing it all once would be 37; 64 sequences of up to 497 tokens, 4 heads of 128: 154 us of 17.
//
// The state is fp32, and so is everything between two products: an operand that is not bf16 to begin with is cut into three bf16 terms (8 + 8 + 8 bits), of whose
// products those of 2^-16 and more count.  Only what out alone reads is rounded further: in bf16 calls S, U and P count with 16 bits.  (P rounded
// to bf16 once is not enough: of keys that repeat the corrections are many times larger than what is left of their sum.)
#include "delta_window.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = DELTA_C, TT = DELTA_TT, TK = DELTA_TK, GROUP = DELTA_GROUP;

// G warps of the chain and OG of out to a run, RUNS runs to a block.  ALONE: the warps that load prepare the windows too, each block its head's, and there are no records in
// global memory.
template <typename T_, int D_, int G_, int OG_, int RUNS_, bool ALONE_ = false>
struct Shape {
  using T = T_;
  static constexpr int D = D_, G = G_, OG = OG_, RUNS = RUNS_;
  static constexpr bool ALONE = ALONE_;
  using Window = DeltaWindow<T, D>;
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;       // of keys
  static constexpr int SEEN = sizeof(T) == 2 ? 2 : 3;        // of S, U and P in out
  using Record = DeltaRecord<SEEN>;
  static constexpr int CHAIN = G * RUNS, OUT = OG * RUNS;    // warps
  static constexpr int THREADS = (CHAIN + OUT) * 32 + GROUP;
  static constexpr int KS = D / 16;                          // products along a key
  static constexpr int SK = KS / G, NT = 2 * SK;             // of them a warp's, and its tiles of 8 keys' elements of the state
  static constexpr int MINE = TT / G, OUT_MINE = TT / OG;    // tiles of tokens of a warp
  static constexpr int COLS = 16 * RUNS;
  static constexpr int KP = D + 8, VP = COLS + 16 / (int)sizeof(T), QP = TERMS == 1 ? D + 8 : D + 4, OP = 16 + 16 / (int)sizeof(T);   // pitches
  static constexpr int TILE = C * KP;                        // bf16 elements of one term of a window's keys
  // Windows in flight.  Keys are waited for two steps ahead of the chain, which asks a step ahead, the rest one: what is fetched has places for those and the
  // chain's.  fp32 keys wait in `raw` to be cut.
  static constexpr int AHEAD = TERMS == 1 ? 2 : 1, PLACES = AHEAD + 2, K_PLACES = TERMS == 1 ? (G == 1 ? AHEAD + 3 : 8) : 3;
  static constexpr int RAW = TERMS == 1 ? 0 : AHEAD * C * (D + 4) * 4;
  static constexpr int K = K_PLACES * TERMS * TILE * 2, Q = PLACES * C * QP * (int)sizeof(T), V = PLACES * C * VP * (int)sizeof(T);
  static constexpr int RECORDS = PLACES * (int)sizeof(Record);
  static constexpr int X = G == 1 ? 0 : RUNS * G * TT * 512, R = G == 1 ? 0 : RUNS * 3 * TK * 512, U = R;
  static constexpr int SEEN_U = 2 * RUNS * SEEN * TK * 512, S = 2 * RUNS * SEEN * KS * 512, O = RUNS * C * OP * (int)sizeof(T);
  static constexpr int ROOM = ALONE ? (int)sizeof(typename Window::Room) : 0;
  static constexpr int SMEM = RAW + K + Q + V + RECORDS + X + R + U + SEEN_U + S + O + ROOM;
  static_assert(!ALONE || TERMS == 1, "keys and queries lie as the preparation reads them");
  static constexpr bool FITS = SMEM + 1024 <= 227 * 1024;
};

// A tile's S^T (e^G q): `state` the lane's registers of S^T, q its token's elements, up that token's e^G
template <typename H>
__device__ __noinline__ float4 read_faded(const uint32_t* state, const typename H::T* q, float up) {
  float sum[4] = {};
#pragma unroll 1
  for (int x = 0; x < H::KS; ++x) {
    uint32_t a[H::SEEN][4], f[3][2];
#pragma unroll
    for (int e = 0; e < H::SEEN; ++e) load16(a[e], state + (e * H::KS + x) * 128);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const typename H::T* z = q + x * 16 + 8 * e;
      uint32_t terms[3];
      cut(up * to_float(z[0]), up * to_float(z[1]), terms);
#pragma unroll
      for (int c = 0; c < 3; ++c) f[c][e] = terms[c];
    }
    product(sum, a, f);
  }
  return make_float4(sum[0], sum[1], sum[2], sum[3]);
}

// A window from token `first` on with something in it that is not finite, or of whose products one is not, token by token: the weights of 0 that a window's products give earlier tokens
// would make NaN of it.  s: a warp's part of the state of run `run`, whose G warps come here together.
template <typename H>
__device__ __forceinline__ void take_one_by_one(const DeltaParams& p, float (&s)[H::NT][4], float (&shares)[H::G][2][16], int b, int h, int first, int n, int run, int warp, const typename H::T* k,
                                             const typename H::T* q, const typename H::T* v, typename H::T* o) {
  using T = typename H::T;
  constexpr int G = H::G, NT = H::NT;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t gate0 = (int64_t)b * p.tokens * p.heads + h;
  for (int i = first; i < min(n, first + C); ++i) {
    const T* kk = k + (int64_t)i * p.k.t + warp * NT * 8 + 2 * t;
    const T* qq = q + (int64_t)i * p.q.t + warp * NT * 8 + 2 * t;
    const float fade = p.log_decay ? expf(p.log_decay[gate0 + (int64_t)i * p.heads]) : 1.f;
    auto sum_of = [&](const T* x, int which, float (&r)[2]) {
      r[0] = r[1] = 0.f;
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e >> 1] = fmaf(to_float(x[8 * m + (e & 1)]), s[m][e], r[e >> 1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        r[e] += __shfl_xor_sync(0xffffffffu, r[e], 1);
        r[e] += __shfl_xor_sync(0xffffffffu, r[e], 2);
        if (G > 1 && t == 0) shares[warp][which][g + 8 * e] = r[e];
      }
      if constexpr (G > 1) {
        barrier_of<32 * G>(2 + run);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          r[e] = 0.f;
#pragma unroll
          for (int m = 0; m < G; ++m) r[e] += shares[m][which][g + 8 * e];
        }
      }
    };
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[m][e] *= fade;
    float said[2], sum[2];
    sum_of(kk, 0, said);
    const float beta = p.beta[gate0 + (int64_t)i * p.heads];
    const T* vv = v + (int64_t)i * p.v.t + 16 * run + g;
    const float u[2] = {beta * (to_float(vv[0]) - said[0]), beta * (to_float(vv[8]) - said[1])};
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[m][e] = fmaf(to_float(kk[8 * m + (e & 1)]), u[e >> 1], s[m][e]);
    sum_of(qq, 1, sum);
    if (warp == 0 && t == 0) {
      T* to = o + (int64_t)i * p.o.t + 16 * run + g;
      to[0] = (T)(p.scale * sum[0]);
      to[8] = (T)(p.scale * sum[1]);
    }
  }
}

// The same out of line, not in the way of what runs always: 2 x 4801 fp32 tokens 211 -> 207 us.
template <typename H>
__device__ __noinline__ void take_one_by_one_apart(const DeltaParams& p, float (&s)[H::NT][4], float (&shares)[H::G][2][16], int b, int h, int first, int n, int run, int warp, const typename H::T* k,
                                                   const typename H::T* q, const typename H::T* v, typename H::T* o) {
  take_one_by_one<H>(p, s, shares, b, h, first, n, run, warp, k, q, v, o);
}

template <typename H>
__global__ void __launch_bounds__(H::THREADS, 1) delta_chunk_kernel(const __grid_constant__ DeltaParams p) {
  using T = typename H::T;
  using Record = typename H::Record;
  constexpr int D = H::D, G = H::G, OG = H::OG, RUNS = H::RUNS, TERMS = H::TERMS, SEEN = H::SEEN, KS = H::KS, SK = H::SK, NT = H::NT, MINE = H::MINE, COLS = H::COLS, KP = H::KP, VP = H::VP, QP = H::QP,
                OP = H::OP;
  constexpr int EACH = 16 / (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int slow[4][RUNS];                                              // [window % 4]: the window is taken token by token
  __shared__ float shares[RUNS][G][2][16];                                   // of either sum of a token taken so
  uint8_t* place = smem;
  auto room = [&](int bytes) {
    uint8_t* r = place;
    place += bytes;
    return r;
  };
  float* raw = reinterpret_cast<float*>(room(H::RAW));                       // [window % AHEAD][C][D + 4]
  __nv_bfloat16* keys = reinterpret_cast<__nv_bfloat16*>(room(H::K));        // [place][term][C][KP]
  T* queries = reinterpret_cast<T*>(room(H::Q));                             // [place][C][QP]
  T* values = reinterpret_cast<T*>(room(H::V));                              // [place][C][VP]
  Record* records = reinterpret_cast<Record*>(room(H::RECORDS));             // [place]
  float* x_part = reinterpret_cast<float*>(room(H::X));                      // [run][warp][tile][lane][4]
  uint32_t* r_frag = reinterpret_cast<uint32_t*>(room(H::R));                // [run][term][TK][lane][4]
  uint32_t* u_frag = reinterpret_cast<uint32_t*>(room(H::U));                // [run][term][TK][lane][4], faded to the window's end
  uint32_t* u_seen = reinterpret_cast<uint32_t*>(room(H::SEEN_U));           // [parity][run][term][TK][lane][4]
  uint32_t* s_seen = reinterpret_cast<uint32_t*>(room(H::S));                // [parity][run][term][KS][lane][4]
  T* outs = reinterpret_cast<T*>(room(H::O));                                // [run][C][OP]
  auto* window = reinterpret_cast<typename H::Window::Room*>(room(H::ROOM));

  const int b = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * COLS;
  const int token0 = p.first_window * C, n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  const int windows = n > token0 ? min(p.windows, (n - token0 + C - 1) / C) : 0;
  if (slot < 0 || (windows == 0 && (p.first_window > 0 || p.state_out == p.state))) {
    pdl_wait();                        // the grid ends behind the preparation's
    return;                            // the whole block
  }
  if (threadIdx.x < 4 * RUNS) slow[threadIdx.x / RUNS][threadIdx.x % RUNS] = 0;
  const int all_warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col0;
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col0;
  auto keys_of = [&](int w) { return keys + ((uint32_t)w % H::K_PLACES) * TERMS * H::TILE; };
  auto queries_of = [&](int w) { return queries + ((uint32_t)w % H::PLACES) * C * QP; };
  auto values_of = [&](int w) { return values + ((uint32_t)w % H::PLACES) * C * VP; };
  auto record_of = [&](int w) -> Record& { return records[(uint32_t)w % H::PLACES]; };

  if (all_warp >= H::CHAIN + H::OUT) {
    // ------------------------------------------------------------------------------- loads
    const int tid = threadIdx.x - (H::CHAIN + H::OUT) * 32;
    const Rows<T, D> k_rows(k, p.k.t, tid), q_rows(q, p.q.t, tid);
    const Rows<T, COLS> v_rows(v, p.v.t, tid);
    const uint8_t* left = H::ALONE ? nullptr : reinterpret_cast<const uint8_t*>(reinterpret_cast<const Record*>(p.records) + ((int64_t)b * p.heads + h) * p.windows);
    auto raw_of = [&](int w) { return reinterpret_cast<T*>(raw) + (w % H::AHEAD) * C * (D + 4); };
    pdl_wait();                                  // for the records
    if (p.more) pdl_launch_dependents();
    // window w's keys and what else window w - 1 needs; nothing behind the last, but counted as the others are
    auto fetch = [&](int w) {
      if (w < windows) {
        if constexpr (TERMS == 1) k_rows.fetch(reinterpret_cast<T*>(keys_of(w)), KP, token0 + w * C, n);
        else k_rows.fetch(raw_of(w), D + 4, token0 + w * C, n);
      }
      if (--w >= 0 && w < windows) {
        q_rows.fetch(queries_of(w), QP, token0 + w * C, n);
        v_rows.fetch(values_of(w), VP, token0 + w * C, n);
        uint8_t* to = reinterpret_cast<uint8_t*>(&record_of(w));
        if constexpr (!H::ALONE)
#pragma unroll
        for (int i = 0; i < (int)sizeof(Record); i += 16 * GROUP)
          if ((int)sizeof(Record) % (16 * GROUP) == 0 || i + tid * 16 < (int)sizeof(Record)) copy16(to + i + tid * 16, left + (int64_t)w * sizeof(Record) + i + tid * 16, true);
      }
      copies_commit();
    };
    float decay = 0.f, beta = 0.f;               // ALONE: of the lanes' tokens of the window that is prepared next
    auto find_gates = [&](int w) {
      const int token = token0 + w * C + lane;
      const int64_t gate = ((int64_t)b * p.tokens + token) * p.heads + h;
      decay = tid < 32 && token < n && p.log_decay ? p.log_decay[gate] : 0.f;
      beta = tid < 32 && token < n ? p.beta[gate] : 0.f;
    };
#pragma unroll
    for (int i = 0; i < H::AHEAD; ++i) fetch(i);
    for (int step = -2; step <= windows; ++step) {
      const int w = step + 2;
      copies_wait<H::AHEAD - 1>();
      if constexpr (H::ALONE) {
        // a window's queries have come a step behind its keys
        if (w >= 1 && w <= windows)
          H::Window::prepare(record_of(w - 1), *window, keys_of(w - 1), queries_of(w - 1), decay, beta, p.scale, tid / 32, lane, [] { barrier_of<GROUP>(1); }, [] { barrier_of<GROUP>(1); });
        find_gates(w);
      }
      if (TERMS == 3 && w < windows) {
        barrier_of<GROUP>(1);
        __nv_bfloat16* ks = keys_of(w);
        const float* from = reinterpret_cast<const float*>(raw_of(w));
        constexpr int PASSES = C * (D / 4) / GROUP;
        float4 f[PASSES];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) f[i] = *reinterpret_cast<const float4*>(from + (tid + i * GROUP) / (D / 4) * (D + 4) + (tid + i * GROUP) % (D / 4) * 4);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          uint32_t low[3], high[3];
          cut(f[i].x, f[i].y, low);
          cut(f[i].z, f[i].w, high);
#pragma unroll
          for (int x = 0; x < 3; ++x)
            *reinterpret_cast<uint2*>(ks + x * H::TILE + (tid + i * GROUP) / (D / 4) * KP + (tid + i * GROUP) % (D / 4) * 4) = make_uint2(low[x], high[x]);
        }
        barrier_of<GROUP>(1);
      }
      fetch(w + H::AHEAD);
      __syncthreads();
    }
  } else if (all_warp >= H::CHAIN) {
    // ------------------------------------------------------------------------------- out
    constexpr int MINE = H::OUT_MINE;
    const int run = (all_warp - H::CHAIN) / OG, warp = (all_warp - H::CHAIN) % OG;      // tiles of tokens warp, warp + OG, ...
    T* stage = outs + run * C * OP;
    float acc[MINE][2][4];               // columns of values g and g + 8, tokens 2t and 2t + 1
    uint32_t weights[MINE][TK][SEEN][2];
    for (int step = -2; step <= windows; ++step) {
      // the last product of the window before
      if (step >= 1 && !slow[(step - 1) & 3][run]) {
        const int w = step - 1;
        uint32_t a[TK][SEEN][4];
#pragma unroll
        for (int x = 0; x < TK; ++x)
#pragma unroll
          for (int e = 0; e < SEEN; ++e) load16(a[x][e], u_seen + ((((w & 1) * RUNS + run) * SEEN + e) * TK + x) * 128 + lane * 4);
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          const int tile = warp + OG * m;
#pragma unroll
          for (int x = 0; x < TK; ++x)
            if (x <= tile / 2) product(acc[m][x], a[x], weights[m][x]);
          T* to = stage + (8 * tile + 2 * t) * OP + g;
          to[0] = (T)(acc[m][0][0] + acc[m][1][0]);
          to[OP] = (T)(acc[m][0][1] + acc[m][1][1]);
          to[8] = (T)(acc[m][0][2] + acc[m][1][2]);
          to[OP + 8] = (T)(acc[m][0][3] + acc[m][1][3]);
        }
        __syncwarp();
#pragma unroll
        for (int e = lane; e < MINE * 8 * (16 / EACH); e += 32) {
          const int i = e / (16 / EACH), r = 8 * (warp + OG * (i / 8)) + i % 8, c = e % (16 / EACH) * EACH;
          const int token = token0 + w * C + r;
          if (token < n) *reinterpret_cast<uint4*>(o + (int64_t)token * p.o.t + 16 * run + c) = *reinterpret_cast<const uint4*>(stage + r * OP + c);
        }
        __syncwarp();
      }
      if (step >= 0 && step < windows) {
        const int w = step;
        const T* qs = queries_of(w);
        const Record& record = record_of(w);
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          const int tile = warp + OG * m;
#pragma unroll
          for (int x = 0; x < TK; ++x)
            if (x <= tile / 2)
#pragma unroll
              for (int e = 0; e < SEEN; ++e) {
                const uint2 f = *reinterpret_cast<const uint2*>(record.weights[delta_place(tile, x)][e][lane]);
                weights[m][x][e][0] = f.x; weights[m][x][e][1] = f.y;
              }
#pragma unroll
          for (int e = 0; e < 2; ++e) acc[m][e][0] = acc[m][e][1] = acc[m][e][2] = acc[m][e][3] = 0.f;
        }
#pragma unroll 2
        for (int x = 0; x < KS; x += 2) {        // 32 elements
          uint32_t a[2][SEEN][4];
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < SEEN; ++e) load16(a[z][e], s_seen + ((((w & 1) * RUNS + run) * SEEN + e) * KS + x + z) * 128 + lane * 4);
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            const int i0 = 8 * (warp + OG * m);
            uint32_t f[2][TERMS][2];
            if constexpr (TERMS == 1) {
              uint32_t z[4];
              ldmatrix4<false>(z, smem_u32(qs + (i0 + (lane & 7)) * QP + x * 16 + (lane >> 3) * 8));
              f[0][0][0] = z[0]; f[0][0][1] = z[1]; f[1][0][0] = z[2]; f[1][0][1] = z[3];
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 z = *reinterpret_cast<const float2*>(qs + (i0 + g) * QP + x * 16 + 8 * e + 2 * t);
                uint32_t terms[3];
                cut(z.x, z.y, terms);
#pragma unroll
                for (int c = 0; c < 3; ++c) f[e >> 1][c][e & 1] = terms[c];
              }
            }
            product(acc[m][0], a[0], f[0]);
            product(acc[m][1], a[1], f[1]);
          }
        }
        // S^T q may pass what 32 bits hold where what the window's decay leaves of it does not: S^T (e^G q) then
        bool odd = false;
        if (record.whole < 0x1p-24f) {
          float sum = 0.f;
#pragma unroll
          for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fmaf(acc[m][0][e] + acc[m][1][e], 0.f, sum);
          odd = __any_sync(0xffffffffu, sum != 0.f);
        }
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          const float2 up = *reinterpret_cast<const float2*>(record.up + 8 * (warp + OG * m) + 2 * t);
          const float gain[2] = {p.scale * up.x, p.scale * up.y};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[m][0][e] = (acc[m][0][e] + acc[m][1][e]) * gain[e & 1];
            acc[m][1][e] = 0.f;
          }
        }
        if (__builtin_expect(odd, 0)) {
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            const int i0 = 8 * (warp + OG * m);
            const float4 sum = read_faded<H>(s_seen + ((w & 1) * RUNS + run) * SEEN * KS * 128 + lane * 4, qs + (i0 + g) * QP + 2 * t, record.up[i0 + g]);
            acc[m][0][0] = p.scale * sum.x; acc[m][0][1] = p.scale * sum.y; acc[m][0][2] = p.scale * sum.z; acc[m][0][3] = p.scale * sum.w;
          }
        }
      }
      __syncthreads();
    }
  } else {
    // ------------------------------------------------------------------------------- the chain
    const int run = all_warp / G, warp = all_warp % G;
    const int64_t state = ((int64_t)slot * p.heads + h) * D * D + col0 + 16 * run;
    // columns of values g and g + 8; the keys' elements 2t and 2t + 1 of the warp's tiles of 8
    float s[NT][4];
    if (p.first_window > 0) pdl_wait();          // for the states of the range before
    auto at = [&](int x, int e) { return (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + g + 8 * (e >> 1); };
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[x][e] = p.state[state + at(x, e)];
    // what the state before window w says of the window's keys, or this warp's part of it
    float says[TT][4];
    // Several warps to a run: whether a correction was not finite is known while the next window's keys are asked for; then the state is set back.  (Looked for before the state is
    // changed: eight maps of 14400 tokens 426 us instead of 413, call by call.)
    float before[G == 1 ? 1 : NT][4];
    uint32_t odd = 0;
    bool again = false;
    auto ask = [&](int w) {
      const __nv_bfloat16* ks = keys_of(w);
#pragma unroll
      for (int x = 0; x < SK; ++x) {
        uint32_t a[3][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t terms[3];
          cut(s[2 * x + (e >> 1)][2 * (e & 1)], s[2 * x + (e >> 1)][2 * (e & 1) + 1], terms);
#pragma unroll
          for (int c = 0; c < 3; ++c) a[c][e] = terms[c];
        }
#pragma unroll
        for (int e = 0; e < SEEN; ++e)
          *reinterpret_cast<uint4*>(s_seen + ((((w & 1) * RUNS + run) * SEEN + e) * KS + warp * SK + x) * 128 + lane * 4) = make_uint4(a[e][0], a[e][1], a[e][2], a[e][3]);
        uint32_t f[TT][TERMS][2];
#pragma unroll
        for (int c = 0; c < TT; c += 2)
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            uint32_t z[4];
            ldmatrix4<false>(z, smem_u32(ks + e * H::TILE + (8 * c + (lane & 7) + 8 * (lane >> 4)) * KP + (warp * SK + x) * 16 + ((lane >> 3) & 1) * 8));
            f[c][e][0] = z[0]; f[c][e][1] = z[1]; f[c + 1][e][0] = z[2]; f[c + 1][e][1] = z[3];
          }
        // the tiles side by side: each product of a tile waits for the one before
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int c = 0; c < TT; ++c)
              if (sum - i >= 0 && sum - i < TERMS) {
                if (x == 0 && sum == 2 && i == (TERMS == 1 ? 2 : 0)) mma16816_first(says[c], a[i], f[c][sum - i][0], f[c][sum - i][1]);
                else mma16816(says[c], a[i], f[c][sum - i][0], f[c][sum - i][1]);
              }
      }
      if constexpr (G > 1) again = __any_sync(0xffffffffu, odd != 0) != 0;
      if constexpr (G > 1)
#pragma unroll
        for (int c = 0; c < TT; ++c) *reinterpret_cast<float4*>(x_part + ((run * G + warp) * TT + c) * 128 + lane * 4) = make_float4(says[c][0], says[c][1], says[c][2], says[c][3]);
    };
    auto advance_slowly = [&](int w) {
      if constexpr (H::ALONE) {                  // a kernel that needs a stack takes the host half a microsecond more to launch
        take_one_by_one<H>(p, s, shares[run], b, h, token0 + w * C, n, run, warp, k, q, v, o);
        return;
      }
      float held[NT][4];
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) held[m][e] = s[m][e];
      take_one_by_one_apart<H>(p, held, shares[run], b, h, token0 + w * C, n, run, warp, k, q, v, o);
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[m][e] = held[m][e];
    };
    auto advance = [&](int w) {
      const __nv_bfloat16* ks = keys_of(w);
      const T* vs = values_of(w) + 16 * run + g;
      const Record& record = record_of(w);
      uint32_t inv[MINE][TK][3][2];
      auto fetch_inverse = [&]() {
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
          for (int x = 0; x < TK; ++x)
            if (x <= (warp + G * m) / 2)
#pragma unroll
              for (int e = 0; e < 3; ++e) {
                const uint2 z = *reinterpret_cast<const uint2*>(record.inverse[delta_place(warp + G * m, x)][e][lane]);
                inv[m][x][e][0] = z.x; inv[m][x][e][1] = z.y;
              }
      };
      if (G > 1) fetch_inverse();      // on its way while R is worked out
      // R and U are this warp's of tiles of tokens warp, warp + G, ...
      float2 down[MINE];
      float r[MINE][4];
#pragma unroll
      for (int m = 0; m < MINE; ++m) {
        const int tile = warp + G * m, token = 8 * tile + 2 * t;
        const float2 beta = *reinterpret_cast<const float2*>(record.beta + token), up = *reinterpret_cast<const float2*>(record.up + token);
        down[m] = *reinterpret_cast<const float2*>(record.down + token);
        const T* vv = vs + token * VP;
        float x[4];
        if constexpr (G == 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = says[m][e];
        } else {
          float4 part[G];
#pragma unroll
          for (int e = 0; e < G; ++e) part[e] = *reinterpret_cast<const float4*>(x_part + ((run * G + e) * TT + tile) * 128 + lane * 4);
#pragma unroll
          for (int d = 1; d < G; d *= 2)
#pragma unroll
            for (int e = 0; e + d < G; e += 2 * d) { part[e].x += part[e + d].x; part[e].y += part[e + d].y; part[e].z += part[e + d].z; part[e].w += part[e + d].w; }
          x[0] = part[0].x; x[1] = part[0].y; x[2] = part[0].z; x[3] = part[0].w;
        }
        r[m][0] = beta.x * fmaf(-up.x, x[0], to_float(vv[0]));
        r[m][1] = beta.y * fmaf(-up.y, x[1], to_float(vv[VP]));
        r[m][2] = beta.x * fmaf(-up.x, x[2], to_float(vv[8]));
        r[m][3] = beta.y * fmaf(-up.y, x[3], to_float(vv[VP + 8]));
        if constexpr (G > 1) keep<3>(r_frag + run * 3 * TK * 128, TK * 128, lane, tile, r[m]);
      }
      if constexpr (G > 1) barrier_of<32 * G>(2 + run);
      else __syncwarp();
      // U^T = R^T T^T
      uint32_t a[TK][3][4];
      auto operand = [&](const uint32_t* frag, const float (&x)[MINE][4]) {
        if constexpr (G == 1) {
#pragma unroll
          for (int i = 0; i < TK; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t terms[3];
              cut(x[2 * i + (e >> 1)][2 * (e & 1)], x[2 * i + (e >> 1)][2 * (e & 1) + 1], terms);
#pragma unroll
              for (int c = 0; c < 3; ++c) a[i][c][e] = terms[c];
            }
        } else {
#pragma unroll
          for (int i = 0; i < TK; ++i)
#pragma unroll
            for (int c = 0; c < 3; ++c) load16(a[i][c], frag + ((run * 3 + c) * TK + i) * 128 + lane * 4);
        }
      };
      operand(r_frag, r);
      if (G == 1) fetch_inverse();
      float u[MINE][4];
      {
        // small products first, tiles side by side, either 16 tokens apart
        float sums[MINE][TK][4];
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int i = 0; i <= sum; ++i)
#pragma unroll
            for (int x = 0; x < TK; ++x)
#pragma unroll
              for (int m = 0; m < MINE; ++m)
                if (x <= (warp + G * m) / 2) {
                  if (sum == 2 && i == 0) mma16816_first(sums[m][x], a[x][i], inv[m][x][sum - i][0], inv[m][x][sum - i][1]);
                  else mma16816(sums[m][x], a[x][i], inv[m][x][sum - i][0], inv[m][x][sum - i][1]);
                }
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) u[m][e] = warp + G * m >= 2 ? sums[m][0][e] + sums[m][1][e] : sums[m][0][e];
      }
      if (lane == 0 && warp == 0) slow[(w + 2) & 3][run] = 0;      // out was through with that two windows ago
      // A correction that is not finite (of R, as a diagonal of T is 1, of T, or as a sum): the window is taken token by token, from the state before it.
      if constexpr (G == 1) {
        bool odd = false;
#pragma unroll
        for (int m = 0; m < MINE; ++m) odd |= fmaf(u[m][0], 0.f, fmaf(u[m][1], 0.f, fmaf(u[m][2], 0.f, u[m][3] * 0.f))) != 0.f;
        if (__builtin_expect(__any_sync(0xffffffffu, odd), 0)) {
          if (lane == 0) slow[w & 3][run] = 1;
          advance_slowly(w);
          return;
        }
      }
#pragma unroll
      for (int m = 0; m < MINE; ++m) {
        const int tile = warp + G * m;
        keep<SEEN>(u_seen + ((w & 1) * RUNS + run) * SEEN * TK * 128, TK * 128, lane, tile, u[m]);
        u[m][0] *= down[m].x; u[m][1] *= down[m].y; u[m][2] *= down[m].x; u[m][3] *= down[m].y;
        if constexpr (G > 1) keep<3>(u_frag + run * 3 * TK * 128, TK * 128, lane, tile, u[m]);
      }
      if constexpr (G > 1) {
        barrier_of<32 * G>(2 + run);
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) before[m][e] = s[m][e];
      }
      operand(u_frag, u);
      if constexpr (G > 1) {
        // each of the run's warps has all of its corrections here, and comes to the same
        __nv_bfloat162 sum = __float2bfloat162_rn(0.f);
#pragma unroll
        for (int x = 0; x < TK; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&a[x][0][e]), __float2bfloat162_rn(0.f), sum);
        odd = *reinterpret_cast<const uint32_t*>(&sum) & 0x7FFF7FFFu;
      }
      // S'^T = e^G_C S^T + U'^T K
      const float whole = record.whole;
      // several tiles side by side: 16 cycles a product with four sums in turn, 12 with eight
      constexpr int SIDE = NT % 4 == 0 && TERMS == 1 ? 4 : 2;
#pragma unroll
      for (int m = 0; m < NT; m += SIDE) {
        uint32_t f[SIDE][2][TERMS][2];
#pragma unroll
        for (int z = 0; z < SIDE; ++z)
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            uint32_t y[4];
            ldmatrix4<true>(y, smem_u32(ks + e * H::TILE + lane * KP + (warp * NT + m + z) * 8));
            f[z][0][e][0] = y[0]; f[z][0][e][1] = y[1]; f[z][1][e][0] = y[2]; f[z][1][e][1] = y[3];
          }
        float d[SIDE][2][4];
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int i = 0; i <= sum; ++i)
#pragma unroll
            for (int z = 0; z < SIDE; ++z)
#pragma unroll
              for (int x = 0; x < 2; ++x)
                if (sum - i < TERMS) {
                  if (sum == 2 && i == (TERMS == 1 ? 2 : 0)) mma16816_first(d[z][x], a[x][i], f[z][x][sum - i][0], f[z][x][sum - i][1]);
                  else mma16816(d[z][x], a[x][i], f[z][x][sum - i][0], f[z][x][sum - i][1]);
                }
#pragma unroll
        for (int z = 0; z < SIDE; ++z)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[m + z][e] = fmaf(whole, s[m + z][e], d[z][0][e] + d[z][1][e]);
      }
    };
    for (int step = -2; step <= windows; ++step) {
      if (step >= 0 && step < windows) advance(step);
      if constexpr (G == 1) {
        if (step >= -1 && step + 1 < windows) ask(step + 1);
      } else {
#pragma unroll 1
        for (int turn = 0; turn < 2; ++turn) {     // the second where the window has been taken token by token
          if (step >= -1 && step + 1 < windows) ask(step + 1);
          else again = __any_sync(0xffffffffu, odd != 0) != 0;
          if (__builtin_expect(turn == 1 || !again, 1)) break;
          if (lane == 0) slow[step & 3][run] = 1;
          odd = 0;
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[m][e] = before[m][e];
          advance_slowly(step);
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) p.state_out[state + at(x, e)] = s[x][e];
  }
}

// Few bf16 sequences of at most two windows are prepared by the blocks that take them: one launch and no records.  The second window is prepared beside the chain of the first;
// a third would make the chain wait.  Five sequences of 60 tokens, 2 heads of 64: 8.3 us on the GPU either way, 9.8 instead of 14.4 for the host.  Where blocks run one behind the
// other it counts that each of a head's does the same work again (18 of 64 tokens, 4 heads of 64: 14.4 us instead of 12.3), and with heads of 128 that there is more of it (4
// of 64 tokens, 4 heads: 10.3 instead of 8.4).
bool alone(int batch, int tokens, int heads, int D, bool bf16) { return bf16 && D < 128 && tokens <= 2 * C && (int64_t)batch * heads * (D / 16) <= PLAN_SMS; }

template <typename H>
cudaError_t launch_shape(const DeltaParams& p, cudaStream_t s) {
  static_assert(H::FITS, "shared memory");
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(delta_chunk_kernel<H>, cudaFuncAttributeMaxDynamicSharedMemorySize, H::SMEM); });
  if (e != cudaSuccess) return e;
  // ahead of the end of the preparation: blocks find their slots and fetch their states meanwhile
  return launch_kernel(delta_chunk_kernel<H>, dim3(H::D / H::COLS, (unsigned)p.heads, (unsigned)p.batch), H::THREADS, H::SMEM, s, p, !H::ALONE);
}
// One warp to a run where runs are many, four where they are few, and one for heads of 32, whose state is one warp's worth.  Measured, us:
//   bf16, heads of 64, 128 runs of 14400 tokens: one 747, four 410; heads of 128, 2048 runs of 497 tokens: one 201, four 289;
//   fp32, heads of 64, 16 runs of 4801 tokens: one 452, four 207; 512 runs of 1000: one 148, four 233 (of heads of 128 four runs do not fit a block);
//   heads of 32, 8 runs of 4801 tokens: one 150 bf16 and 199 fp32, two 155 and 231; 256 runs of 1000: one 53 and 77, two 54 and 83.
template <typename T, int D>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  if constexpr (sizeof(T) == 2 && D < 128)
    if (alone(p.batch, p.tokens, p.heads, D, true)) return launch_shape<Shape<T, D, D == 32 ? 1 : 4, D == 32 ? 1 : 2, D == 32 ? 2 : 1, true>>(p, s);
  if constexpr (D == 32) {
    return launch_shape<Shape<T, D, 1, 1, 2>>(p, s);
  } else {
    if constexpr (Shape<T, D, 1, 1, 4>::FITS)
      if ((int64_t)p.batch * p.heads * (D / 16) > 2 * PLAN_SMS) return launch_shape<Shape<T, D, 1, 1, 4>>(p, s);
    return launch_shape<Shape<T, D, 4, sizeof(T) == 2 ? 2 : 4, 1>>(p, s);
  }
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

// The windows are prepared and taken in ranges: a range's preparation runs beside the chain of the range before, with records of its own, both launched ahead of the
// end of what is before them.  Eight maps of 14400 tokens, 4 heads of 64, when they took 414 us: ranges one behind the other 442; with a first range of a quarter, whose
// preparation alone has nothing beside it, 417.  A range more is 5 us more, so there is one as long as its records fit `most` bytes, of which two lie in the L2 cache.
static int range_of(int batch, int tokens, int heads, bool bf16, uint64_t* bytes) {
  constexpr int64_t most = 48 << 20;
  const int64_t each = (int64_t)batch * heads * (int64_t)(bf16 ? sizeof(DeltaRecord<2>) : sizeof(DeltaRecord<3>)), all = ((int64_t)tokens + C - 1) / C;
  const int64_t fit = most / each < 1 ? 1 : most / each, ranges = (all + fit - 1) / fit, windows = (all + ranges - 1) / ranges;
  *bytes = (uint64_t)(windows * each);
  return (int)windows;
}
uint64_t delta_scratch(int batch, int tokens, int heads, int D, bool bf16) {
  if (alone(batch, tokens, heads, D, bf16)) return 0;
  uint64_t bytes;
  const int windows = range_of(batch, tokens, heads, bf16, &bytes);
  return windows * C < tokens ? 2 * bytes : bytes;
}

cudaError_t launch_delta_chunk(DeltaParams p, bool bf16, int D, cudaStream_t s) {
  const int all = (p.tokens + C - 1) / C;
  if (alone(p.batch, p.tokens, p.heads, D, bf16)) {
    p.windows = all;
    return launch<__nv_bfloat16>(p, D, s);
  }
  uint8_t* const room = static_cast<uint8_t*>(p.records);
  uint64_t bytes;
  p.windows = range_of(p.batch, p.tokens, p.heads, bf16, &bytes);
  for (p.first_window = 0; p.first_window < all; p.first_window += p.windows) {
    p.more = p.first_window + p.windows < all;
    p.records = room + p.first_window / p.windows % 2 * bytes;
    cudaError_t e = launch_delta_prepare(p, bf16, D, s);
    if (e == cudaSuccess) e = bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
    if (e != cudaSuccess) return e;
    p.state = p.state_out;
  }
  return cudaSuccess;
}

}  // namespace tok
}  // namespace tt

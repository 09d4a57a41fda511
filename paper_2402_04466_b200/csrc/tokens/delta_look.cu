// The gated delta rule over several tokens, second part where runs are few (tt_delta_rule): the chain of states, a window of 32 tokens at a time, a step ahead of itself.
//
// With G_i the sum of log_decay up to and including token i of window w and T and P what delta_prepare.cu has worked out,
//   R_i = beta_i (v_i - e^G_i x_i),  x_i = S_w^T k_i,  U = T R,  out_i = scale e^G_i S_w^T q_i + sum_j P_ij u_j,  S_(w+1) = e^G_C S_w + sum_j k_j u'_j^T,  u'_j = e^(G_C - G_j) u_j.
// What bounds a sequence is the chain from one window's U to the next one's, and what that takes is products behind each other: 35 cycles for one that waits for another, 12 to 16 for
// any of a warp alone.  Instead of U -> S -> x the chain goes around the state,
//   x_i of window w + 1 = e^G_C (S_w^T k_i) + sum_j (k_j . k_i) u'_j,
// whose first term needs the state of a window ago only and whose second the products of two windows' keys, which need none.  So four warps take the chain U' -> x -> R -> U -> U', a
// tile of 8 tokens each, and four others the states, a quarter of the keys' elements each in registers, a window behind: S_w, then z = S_w^T k_i for the window after the
// next one.  Two or four warps turn what both leave into out, another window behind, and four load.  All meet once a window.
//
// A block owns 16 value columns of one head's state (the columns are independent of each other).  Everything is kept transposed, columns of
// values along M: the accumulators of one m16n8k16 product are then the other operand's registers of the next; R and U go from warp to warp as those registers, 16 bytes to
// a lane.  ???
//
// The state is fp32, and so is everything between two products: an operand that is not bf16 to begin with is cut into three bf16 terms (8 + 8 + 8 bits), of whose
// products those of 2^-16 and more count.  Only what out alone reads is rounded further: in bf16 calls S, U and P count with 16 bits.
#include "delta_common.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = DELTA_C, TT = DELTA_TT, TK = DELTA_TK, GROUP = DELTA_GROUP;

template <typename T_, int D_>
struct Shape {
  using T = T_;
  static constexpr int D = D_;
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;       // of keys and queries
  static constexpr int SEEN = sizeof(T) == 2 ? 2 : 3;        // of S, U and P in out
  using Record = DeltaRecord<SEEN, true>;
  static constexpr int CHAIN = TT, STATE = D == 32 ? 2 : 4, OUT = TERMS == 1 ? 2 : 4;      // warps
  static constexpr int THREADS = (CHAIN + STATE + OUT) * 32 + GROUP;
  static constexpr int KS = D / 16;                          // products along a key
  static constexpr int SK = KS / STATE, NT = 2 * SK;         // of them a state warp's, and its tiles of 8 keys' elements
  static constexpr int KP = TERMS == 1 ? D + 8 : D + 4, VP = 16 + 16 / (int)sizeof(T);   // pitches: keys and queries, values and out
  // Windows in flight beyond the next; keys are used from a window ahead of the chain to one behind it, queries one behind, records from the chain's to one behind.
  static constexpr int DEEP = TERMS == 1 ? 1 : 0, K_PLACES = 4 + DEEP, V_PLACES = 2 + DEEP, Q_PLACES = 2 + DEEP, R_PLACES = 3 + DEEP;
  static constexpr int TILE = C * KP;
  static constexpr int K = K_PLACES * TILE * (int)sizeof(T), Q = Q_PLACES * TILE * (int)sizeof(T), V = V_PLACES * C * VP * (int)sizeof(T);
  static constexpr int RECORDS = R_PLACES * (int)sizeof(Record);
  static constexpr int Z = 2 * STATE * TT * 512, R = 3 * TK * 512, U = 2 * 3 * TK * 512;
  static constexpr int SEEN_U = 2 * SEEN * TK * 512, S = 2 * SEEN * KS * 512, O = C * VP * (int)sizeof(T);
  static constexpr int SMEM = K + Q + V + RECORDS + Z + R + U + SEEN_U + S + O;
  static_assert(SMEM + 1024 <= 227 * 1024, "shared memory");
};

// a.b of TA and TB terms, small products first, into two sums in turn
template <int TA, int TB>
__device__ __forceinline__ void product_two(float (&acc)[2][4], const uint32_t (&a)[TA][4], const uint32_t (&b)[TB][2]) {
  constexpr int MOST = TA > TB ? TA : TB;
#pragma unroll
  for (int sum = MOST - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i <= sum; ++i)
      if (i < TA && sum - i < TB) mma16816(acc[(sum + i) & 1], a[i], b[sum - i][0], b[sum - i][1]);
}

template <typename H>
__global__ void __launch_bounds__(H::THREADS, 1) delta_look_kernel(const __grid_constant__ DeltaParams p) {
  using T = typename H::T;
  using Record = typename H::Record;
  constexpr int D = H::D, TERMS = H::TERMS, SEEN = H::SEEN, KS = H::KS, SK = H::SK, NT = H::NT, KP = H::KP, VP = H::VP;
  constexpr int EACH = 16 / (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int slow[2];                                                    // [parity]: the window is taken token by token
  __shared__ int odd_flags[H::CHAIN];
  __shared__ float shares[H::STATE][2][16];                                  // of either sum of a token taken so
  uint8_t* place = smem;
  auto room = [&](int bytes) {
    uint8_t* r = place;
    place += bytes;
    return r;
  };
  T* keys = reinterpret_cast<T*>(room(H::K));                                // [place][C][KP]
  T* queries = reinterpret_cast<T*>(room(H::Q));                             // [place][C][KP]
  T* values = reinterpret_cast<T*>(room(H::V));                              // [place][C][VP]
  Record* records = reinterpret_cast<Record*>(room(H::RECORDS));             // [place]
  float* z_part = reinterpret_cast<float*>(room(H::Z));                      // [parity][state warp][tile][lane][4]
  uint32_t* r_frag = reinterpret_cast<uint32_t*>(room(H::R));                // [term][TK][lane][4]
  uint32_t* u_frag = reinterpret_cast<uint32_t*>(room(H::U));                // [parity][term][TK][lane][4], faded to the window's end
  uint32_t* u_seen = reinterpret_cast<uint32_t*>(room(H::SEEN_U));           // [parity][term][TK][lane][4]
  uint32_t* s_seen = reinterpret_cast<uint32_t*>(room(H::S));                // [parity][term][KS][lane][4]
  T* outs = reinterpret_cast<T*>(room(H::O));                                // [C][VP]

  const int b = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * 16;
  const int token0 = p.first_window * C, n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int windows = n > token0 ? min(p.windows, (n - token0 + C - 1) / C) : 0;
  if (windows == 0 && (p.first_window > 0 || p.state_out == p.state)) return;
  const int all_warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col0;
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col0;
  auto keys_of = [&](int w) { return keys + (w % H::K_PLACES) * H::TILE; };
  auto queries_of = [&](int w) { return queries + (w % H::Q_PLACES) * H::TILE; };
  auto values_of = [&](int w) { return values + (w % H::V_PLACES) * C * VP; };
  auto record_of = [&](int w) -> Record& { return records[w % H::R_PLACES]; };
  // the second operand of products along elements 16 x .. 16 x + 15 of 8 rows of keys or queries
  auto rows_operand = [&](const T* rows, int x, uint32_t (&f)[TERMS][2]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (TERMS == 1) {
        f[0][e] = *reinterpret_cast<const uint32_t*>(rows + g * KP + 16 * x + 8 * e + 2 * t);
      } else {
        const float2 y = *reinterpret_cast<const float2*>(rows + g * KP + 16 * x + 8 * e + 2 * t);
        uint32_t terms[3];
        cut(y.x, y.y, terms);
#pragma unroll
        for (int c = 0; c < 3; ++c) f[c][e] = terms[c];
      }
    }
  };
  constexpr int FIRST = -2 - H::DEEP;          // step in which the first keys are fetched
  // All of a block's warps run through the same steps and meet behind each.  Where something in a window turned out not to be finite, the state's warps take it token by token
  // while the others wait.
  if (all_warp >= H::CHAIN + H::STATE + H::OUT) {
    // ------------------------------------------------------------------------------- loads
    const int tid = threadIdx.x - (H::CHAIN + H::STATE + H::OUT) * 32;
    const Rows<T, D> k_rows(k, p.k.t, tid), q_rows(q, p.q.t, tid);
    const Rows<T, 16> v_rows(v, p.v.t, tid);
    const uint8_t* left = reinterpret_cast<const uint8_t*>(reinterpret_cast<const Record*>(p.records) + ((int64_t)b * p.heads + h) * p.windows);
    auto here = [&](int w) { return w >= 0 && w < windows; };
    for (int step = FIRST; step <= windows; ++step) {
      // what step + 1 + DEEP uses for the first time
      const int w = step + 1 + H::DEEP;
      if (here(w + 1)) k_rows.fetch(keys_of(w + 1), KP, token0 + (w + 1) * C, n);
      if (here(w)) {
        v_rows.fetch(values_of(w), VP, token0 + w * C, n);
        uint8_t* to = reinterpret_cast<uint8_t*>(&record_of(w));
#pragma unroll
        for (int i = 0; i < (int)sizeof(Record); i += 16 * GROUP)
          if (i + 16 * GROUP <= (int)sizeof(Record) || i + tid * 16 < (int)sizeof(Record)) copy16(to + i + tid * 16, left + (int64_t)w * sizeof(Record) + i + tid * 16, true);
      }
      if (here(w - 1)) q_rows.fetch(queries_of(w - 1), KP, token0 + (w - 1) * C, n);
      copies_commit();
      copies_wait<H::DEEP>();
      __syncthreads();
      if (here(step) && slow[step & 1]) __syncthreads();
    }
  } else if (all_warp >= H::CHAIN + H::STATE) {
    // ------------------------------------------------------------------------------- out, of the window before
    constexpr int MINE = TT / H::OUT;
    const int warp = all_warp - H::CHAIN - H::STATE;      // tiles of tokens warp, warp + OUT, ...
    for (int step = FIRST; step <= windows; ++step) {
      const int w = step - 1;
      if (w >= 0 && !slow[w & 1]) {
        const T* qs = queries_of(w);
        const Record& record = record_of(w);
        float acc[MINE][2][4] = {};          // columns of values g and g + 8, tokens 2t and 2t + 1
#pragma unroll 2
        for (int x = 0; x < KS; ++x) {
          uint32_t a[SEEN][4];
#pragma unroll
          for (int e = 0; e < SEEN; ++e) load16(a[e], s_seen + (((w & 1) * SEEN + e) * KS + x) * 128 + lane * 4);
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            uint32_t f[TERMS][2];
            rows_operand(qs + 8 * (warp + H::OUT * m) * KP, x, f);
            product_two(acc[m], a, f);
          }
        }
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          const int tile = warp + H::OUT * m;
          const float2 up = *reinterpret_cast<const float2*>(record.up + 8 * tile + 2 * t);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[m][0][e] = (acc[m][0][e] + acc[m][1][e]) * (p.scale * (e & 1 ? up.y : up.x));
            acc[m][1][e] = 0.f;
          }
        }
#pragma unroll
        for (int x = 0; x < TK; ++x) {
          uint32_t a[SEEN][4];
#pragma unroll
          for (int e = 0; e < SEEN; ++e) load16(a[e], u_seen + (((w & 1) * SEEN + e) * TK + x) * 128 + lane * 4);
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            const int tile = warp + H::OUT * m;
            if (x <= tile / 2) {
              uint32_t f[SEEN][2];
#pragma unroll
              for (int e = 0; e < SEEN; ++e) {
                const uint2 y = *reinterpret_cast<const uint2*>(record.weights[delta_place(tile, x)][e][lane]);
                f[e][0] = y.x; f[e][1] = y.y;
              }
              product_two(acc[m], a, f);
            }
          }
        }
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          T* to = outs + (8 * (warp + H::OUT * m) + 2 * t) * VP + g;
          to[0] = (T)(acc[m][0][0] + acc[m][1][0]);
          to[VP] = (T)(acc[m][0][1] + acc[m][1][1]);
          to[8] = (T)(acc[m][0][2] + acc[m][1][2]);
          to[VP + 8] = (T)(acc[m][0][3] + acc[m][1][3]);
        }
        __syncwarp();
#pragma unroll
        for (int e = lane; e < MINE * 8 * (16 / EACH); e += 32) {
          const int i = e / (16 / EACH), r = 8 * (warp + H::OUT * (i / 8)) + i % 8, c = e % (16 / EACH) * EACH;
          const int token = token0 + w * C + r;
          if (token < n) *reinterpret_cast<uint4*>(o + (int64_t)token * p.o.t + c) = *reinterpret_cast<const uint4*>(outs + r * VP + c);
        }
      }
      __syncthreads();
      if (step >= 0 && step < windows && slow[step & 1]) __syncthreads();
    }
  } else if (all_warp >= H::CHAIN) {
    // ------------------------------------------------------------------------------- states
    const int warp = all_warp - H::CHAIN;
    const int64_t state = ((int64_t)slot * p.heads + h) * D * D + col0;
    // columns of values g and g + 8; the keys' elements 2t and 2t + 1 of the warp's tiles of 8
    float s[NT][4];
    auto at = [&](int x, int e) { return (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + g + 8 * (e >> 1); };
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[x][e] = p.state[state + at(x, e)];
    uint32_t a[SK][3][4];                // the state as an operand
    auto cut_state = [&]() {
#pragma unroll
      for (int x = 0; x < SK; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t terms[3];
          cut(s[2 * x + (e >> 1)][2 * (e & 1)], s[2 * x + (e >> 1)][2 * (e & 1) + 1], terms);
#pragma unroll
          for (int c = 0; c < 3; ++c) a[x][c][e] = terms[c];
        }
    };
    // what the state says of window w's keys, this warp's part
    auto ask = [&](int w) {
      const T* ks = keys_of(w);
      float says[TT][4];
#pragma unroll
      for (int c = 0; c < TT; ++c) says[c][0] = says[c][1] = says[c][2] = says[c][3] = 0.f;
#pragma unroll
      for (int x = 0; x < SK; ++x) {
        uint32_t f[TT][TERMS][2];
#pragma unroll
        for (int c = 0; c < TT; ++c) rows_operand(ks + 8 * c * KP, warp * SK + x, f[c]);
        // the tiles side by side: each product of a tile waits for the one before
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int c = 0; c < TT; ++c)
              if (sum - i >= 0 && sum - i < TERMS) mma16816(says[c], a[x][i], f[c][sum - i][0], f[c][sum - i][1]);
      }
#pragma unroll
      for (int c = 0; c < TT; ++c) *reinterpret_cast<float4*>(z_part + (((w & 1) * H::STATE + warp) * TT + c) * 128 + lane * 4) = make_float4(says[c][0], says[c][1], says[c][2], says[c][3]);
    };
    // S_(w+1)^T = e^G_C S_w^T + U'^T K
    auto advance = [&](int w) {
      const T* ks = keys_of(w);
      const float whole = record_of(w).whole;
      uint32_t u[TK][3][4];
#pragma unroll
      for (int x = 0; x < TK; ++x)
#pragma unroll
        for (int c = 0; c < 3; ++c) load16(u[x][c], u_frag + (((w & 1) * 3 + c) * TK + x) * 128 + lane * 4);
#pragma unroll
      for (int m = 0; m < NT; m += 2) {
        uint32_t f[2][TK][TERMS][2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int col = (warp * NT + m + z) * 8;
          if constexpr (TERMS == 1) {
            uint32_t y[4];
            ldmatrix4<true>(y, smem_u32(ks + lane * KP + col));
            f[z][0][0][0] = y[0]; f[z][0][0][1] = y[1]; f[z][1][0][0] = y[2]; f[z][1][0][1] = y[3];
          } else {
#pragma unroll
            for (int x = 0; x < TK; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const T* y = ks + (16 * x + 8 * e + 2 * t) * KP + col + g;
                uint32_t terms[3];
                cut(y[0], y[KP], terms);
#pragma unroll
                for (int c = 0; c < 3; ++c) f[z][x][c][e] = terms[c];
              }
          }
        }
        float d[2][TK][4] = {};
#pragma unroll
        for (int sum = 2; sum >= 0; --sum)
#pragma unroll
          for (int i = 0; i <= sum; ++i)
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int x = 0; x < TK; ++x)
                if (sum - i < TERMS) mma16816(d[z][x], u[x][i], f[z][x][sum - i][0], f[z][x][sum - i][1]);
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[m + z][e] = fmaf(whole, s[m + z][e], d[z][0][e] + d[z][1][e]);
      }
    };
    // A window with something in it that is not finite, token by token: the weights of 0 that a window's products give earlier tokens would make NaN of it.
    auto advance_slowly = [&](int w) {
      const int64_t gate0 = (int64_t)b * p.tokens * p.heads + h;
      for (int i = token0 + w * C; i < min(n, token0 + w * C + C); ++i) {
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
            if (t == 0) shares[warp][which][g + 8 * e] = r[e];
          }
          barrier_of<32 * H::STATE>(2);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            r[e] = 0.f;
#pragma unroll
            for (int m = 0; m < H::STATE; ++m) r[e] += shares[m][which][g + 8 * e];
          }
        };
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[m][e] *= fade;
        float said[2], sum[2];
        sum_of(kk, 0, said);
        const float beta = p.beta[gate0 + (int64_t)i * p.heads];
        const T* vv = v + (int64_t)i * p.v.t + g;
        const float u[2] = {beta * (to_float(vv[0]) - said[0]), beta * (to_float(vv[8]) - said[1])};
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[m][e] = fmaf(to_float(kk[8 * m + (e & 1)]), u[e >> 1], s[m][e]);
        sum_of(qq, 1, sum);
        if (warp == 0 && t == 0) {
          T* to = o + (int64_t)i * p.o.t + g;
          to[0] = (T)(p.scale * sum[0]);
          to[8] = (T)(p.scale * sum[1]);
        }
      }
    };
    for (int step = FIRST; step <= windows; ++step) {
      const bool inside = step >= 0 && step < windows;
      if (step >= -1) {
        if (step > 0 && !slow[(step - 1) & 1]) advance(step - 1);
        if (step < windows) {
          cut_state();
          if (step >= 0)
#pragma unroll
            for (int e = 0; e < SEEN; ++e)
#pragma unroll
              for (int x = 0; x < SK; ++x)
                *reinterpret_cast<uint4*>(s_seen + (((step & 1) * SEEN + e) * KS + warp * SK + x) * 128 + lane * 4) = make_uint4(a[x][e][0], a[x][e][1], a[x][e][2], a[x][e][3]);
          if (step + 1 < windows) ask(step + 1);
        }
      }
      __syncthreads();
      if (inside && slow[step & 1]) {
        advance_slowly(step);
        if (step + 1 < windows) {
          cut_state();
          ask(step + 1);
        }
        __syncthreads();
      }
    }
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) p.state_out[state + at(x, e)] = s[x][e];
  } else {
    // ------------------------------------------------------------------------------- the chain
    const int warp = all_warp, token = 8 * warp + 2 * t;      // a tile of tokens; sums over tokens reach up to it
    const bool both = warp >= 2;
    for (int step = FIRST; step <= windows; ++step) {
      const bool inside = step >= 0 && step < windows;
      if (inside) {
        const int w = step;
        const Record& record = record_of(w);
        const T* vv = values_of(w) + token * VP + g;
        // x of the window's first state, or of one that was taken token by token, is what the state's warps have left
        const bool fresh = w == 0 || slow[(w - 1) & 1] != 0;
        float4 part[H::STATE];
#pragma unroll
        for (int e = 0; e < H::STATE; ++e) part[e] = *reinterpret_cast<const float4*>(z_part + (((w & 1) * H::STATE + e) * TT + warp) * 128 + lane * 4);
        float x[4];
        uint32_t a[TK][3][4];
        if (!fresh) {
          const Record& last = record_of(w - 1);
          uint32_t f[TK][3][2];
#pragma unroll
          for (int i = 0; i < TK; ++i)
#pragma unroll
            for (int c = 0; c < 3; ++c) {
              load16(a[i][c], u_frag + ((((w - 1) & 1) * 3 + c) * TK + i) * 128 + lane * 4);
              const uint2 y = *reinterpret_cast<const uint2*>(last.next[warp][i][c][lane]);
              f[i][c][0] = y.x; f[i][c][1] = y.y;
            }
          float sums[TK][2][4] = {};
#pragma unroll
          for (int sum = 2; sum >= 0; --sum)
#pragma unroll
            for (int i = 0; i <= sum; ++i)
#pragma unroll
              for (int y = 0; y < TK; ++y) mma16816(sums[y][(sum + i) & 1], a[y][i], f[y][sum - i][0], f[y][sum - i][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = (sums[0][0][e] + sums[1][0][e]) + (sums[0][1][e] + sums[1][1][e]);
        }
#pragma unroll
        for (int d = 1; d < H::STATE; d *= 2)
#pragma unroll
          for (int e = 0; e + d < H::STATE; e += 2 * d) { part[e].x += part[e + d].x; part[e].y += part[e + d].y; part[e].z += part[e + d].z; part[e].w += part[e + d].w; }
        if (fresh) {
          x[0] = part[0].x; x[1] = part[0].y; x[2] = part[0].z; x[3] = part[0].w;
        } else {
          const float whole = record_of(w - 1).whole;
          x[0] = fmaf(whole, part[0].x, x[0]); x[1] = fmaf(whole, part[0].y, x[1]); x[2] = fmaf(whole, part[0].z, x[2]); x[3] = fmaf(whole, part[0].w, x[3]);
        }
        uint32_t inv[TK][3][2];
#pragma unroll
        for (int i = 0; i < TK; ++i)
          if (i == 0 || both)
#pragma unroll
            for (int c = 0; c < 3; ++c) {
              const uint2 y = *reinterpret_cast<const uint2*>(record.inverse[delta_place(warp, i)][c][lane]);
              inv[i][c][0] = y.x; inv[i][c][1] = y.y;
            }
        const float2 beta = *reinterpret_cast<const float2*>(record.beta + token), up = *reinterpret_cast<const float2*>(record.up + token),
                     down = *reinterpret_cast<const float2*>(record.down + token);
        float r[4];
        r[0] = beta.x * fmaf(-up.x, x[0], to_float(vv[0]));
        r[1] = beta.y * fmaf(-up.y, x[1], to_float(vv[VP]));
        r[2] = beta.x * fmaf(-up.x, x[2], to_float(vv[8]));
        r[3] = beta.y * fmaf(-up.y, x[3], to_float(vv[VP + 8]));
        keep<3>(r_frag, TK * 128, lane, warp, r);
        bool odd = __any_sync(0xffffffffu, fmaf(r[0], 0.f, fmaf(r[1], 0.f, fmaf(r[2], 0.f, r[3] * 0.f))) != 0.f);
        if (lane == 0) odd_flags[warp] = odd;
        barrier_of<32 * H::CHAIN>(1);
        // U^T = R^T T^T
        float sums[TK][2][4] = {};
#pragma unroll
        for (int i = 0; i < TK; ++i)
          if (i == 0 || both) {
#pragma unroll
            for (int c = 0; c < 3; ++c) load16(a[i][c], r_frag + (c * TK + i) * 128 + lane * 4);
          }
#pragma unroll
        for (int i = 0; i < TK; ++i)
          if (i == 0 || both) product_two(sums[i], a[i], inv[i]);
        // where something in the window or its state is not finite, nothing of this counts
#pragma unroll
        for (int m = 0; m < H::CHAIN; ++m) odd |= odd_flags[m] != 0;
        if (threadIdx.x == 0) slow[w & 1] = odd;
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = (sums[0][0][e] + sums[1][0][e]) + (sums[0][1][e] + sums[1][1][e]);
        const float faded[4] = {u[0] * down.x, u[1] * down.y, u[2] * down.x, u[3] * down.y};
        keep<3>(u_frag + (w & 1) * 3 * TK * 128, TK * 128, lane, warp, faded);
        keep<SEEN>(u_seen + (w & 1) * SEEN * TK * 128, TK * 128, lane, warp, u);
      }
      __syncthreads();
      if (inside && slow[step & 1]) __syncthreads();
    }
  }
}

template <typename H>
cudaError_t launch_shape(const DeltaParams& p, cudaStream_t s) {
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(delta_look_kernel<H>, cudaFuncAttributeMaxDynamicSharedMemorySize, H::SMEM); });
  if (e != cudaSuccess) return e;
  delta_look_kernel<H><<<dim3(H::D / 16, (unsigned)p.heads, (unsigned)p.batch), H::THREADS, H::SMEM, s>>>(p);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch_shape<Shape<T, 32>>(p, s) : D == 64 ? launch_shape<Shape<T, 64>>(p, s) : launch_shape<Shape<T, 128>>(p, s);
}

}  // namespace

cudaError_t launch_delta_look(const DeltaParams& p, bool bf16, int D, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
}

}  // namespace tok
}  // namespace tt

// The gated delta rule over several tokens, second part (tt_delta_rule): the chain of states, a window of 32 tokens at a time.
//
// With G_i the sum of log_decay up to and including token i of a window and T and P what delta_prepare.cu has worked out,
//   R_i = beta_i (v_i - e^G_i S^T k_i),  U = T R,  out_i = scale e^G_i S^T q_i + sum_j P_ij u_j,  S' = e^G_C S + sum_j e^(G_C - G_j) k_j u_j^T.
// What bounds a sequence is the chain S -> R -> U -> S'.  A block has three groups of four warps, which meet once a window: loads, two windows and more ahead; the chain; and out,
// whose last product is taken a window behind.
//
// A block owns NS runs of 16 value columns of one head's state (the columns are independent of each other).  Everything on the chain is kept transposed, columns of
// values along M: the accumulators of one m16n8k16 product are then the other operand's registers of the next.  Each warp of the chain has a quarter of the keys' elements of the
// state in registers, as sums and as operands: X^T = S^T K^T comes in four parts, which the warps add up where they read them, then U^T = R^T T^T and
// S'^T = U'^T K.  R and U go from warp to warp as operands' registers, 16 bytes to a lane.  (A tcgen05 product of 16 columns takes 40 cycles however few its
// columns are, and its way through tensor memory twice that: the chain would be longer, not shorter.)
//
// The state is fp32, and so is everything between two products: an operand that is not bf16 to begin with is cut into three bf16 terms (8 + 8 + 8 bits), of whose
// products those of 2^-16 and more count.  Only what out alone reads is rounded further: in bf16 calls S, U and P count with 16 bits.  (P rounded
// to bf16 once is not enough: of keys that repeat the corrections are many times larger than what is left of their sum.)
#include "delta_common.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = DELTA_C, TT = DELTA_TT, TK = DELTA_TK, GROUP = DELTA_GROUP, THREADS = 3 * GROUP;
enum { CHAIN = 0, OUT = 1, LOAD = 2 };

template <typename T_, int D_, int NS_>
struct Shape {
  using T = T_;
  static constexpr int D = D_, NS = NS_;
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;       // of keys
  static constexpr int SEEN = sizeof(T) == 2 ? 2 : 3;        // of S, U and P in out
  using Record = DeltaRecord<SEEN>;
  static constexpr int KS = D / 16;                          // products along a key
  static constexpr int NT = D / 32;                          // tiles of 8 keys' elements of the state to a warp
  static constexpr int SK = NT > 1 ? NT / 2 : 1;             // products along those
  static constexpr int COLS = 16 * NS;
  static constexpr int KP = D + 8, VP = COLS + 16 / (int)sizeof(T), QP = TERMS == 1 ? D + 8 : D + 4;   // pitches
  static constexpr int TILE = C * KP;                        // bf16 elements of one term of a window's keys
  // Windows in flight when the next but one to the chain's is waited for: what is fetched has places for them, that one, the chain's and the one between.  fp32 keys
  // wait in `raw` to be cut.
  static constexpr int AHEAD = TERMS == 1 ? 2 : 1, PLACES = AHEAD + 3;
  static constexpr int K_PLACES = TERMS == 1 ? PLACES : 3, Q_PLACES = AHEAD + 1;
  static constexpr int RAW = TERMS == 1 ? 0 : AHEAD * C * (D + 4) * 4;
  static constexpr int K = K_PLACES * TERMS * TILE * 2, Q = Q_PLACES * C * QP * (int)sizeof(T), V = PLACES * C * VP * (int)sizeof(T);
  static constexpr int RECORDS = PLACES * (int)sizeof(Record);
  static constexpr int X = NS * 4 * TT * 512, R = NS * 3 * TK * 512, U = NS * 3 * TK * 512, SEEN_U = 2 * NS * SEEN * TK * 512, S = 2 * NS * SEEN * KS * 512;
  static constexpr int O = C * VP * (int)sizeof(T);
  static constexpr int SMEM = RAW + K + Q + V + RECORDS + X + R + U + SEEN_U + S + O;
  static constexpr bool FITS = SMEM + 1024 <= 227 * 1024;
};

__device__ __forceinline__ void barrier(int id) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "n"(GROUP) : "memory"); }

template <typename H>
__global__ void __launch_bounds__(THREADS, 1) delta_chunk_kernel(const __grid_constant__ DeltaParams p) {
  using T = typename H::T;
  using Record = typename H::Record;
  constexpr int D = H::D, NS = H::NS, TERMS = H::TERMS, SEEN = H::SEEN, KS = H::KS, NT = H::NT, SK = H::SK, COLS = H::COLS, KP = H::KP, VP = H::VP, QP = H::QP;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int slow[2];                                                    // [parity]: the window was taken token by token
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
  T* outs = reinterpret_cast<T*>(room(H::O));                                // [C][VP]

  const int b = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * COLS;
  const int token0 = p.first_window * C, n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int windows = n > token0 ? min(p.windows, (n - token0 + C - 1) / C) : 0;
  if (windows == 0 && (p.first_window > 0 || p.state_out == p.state)) return;
  const int role = __shfl_sync(0xffffffffu, (int)(threadIdx.x / GROUP), 0), warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5) & 3, 0);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, tid = threadIdx.x % GROUP;
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col0;
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col0;
  const int64_t gate0 = (int64_t)b * p.tokens * p.heads + h;
  const int64_t state = ((int64_t)slot * p.heads + h) * D * D + col0;
  auto keys_of = [&](int w) { return keys + (w % H::K_PLACES) * TERMS * H::TILE; };
  auto values_of = [&](int w) { return values + (w % H::PLACES) * C * VP; };
  auto record_of = [&](int w) -> Record& { return records[w % H::PLACES]; };

  if (role == LOAD) {
    // ------------------------------------------------------------------------------- loads
    const Rows<T, D> k_rows(k, p.k.t, tid);
    const Rows<T, COLS> v_rows(v, p.v.t, tid);
    const uint8_t* left = reinterpret_cast<const uint8_t*>(reinterpret_cast<const Record*>(p.records) + ((int64_t)b * p.heads + h) * p.windows);
    auto raw_of = [&](int w) { return reinterpret_cast<T*>(raw) + (w % H::AHEAD) * C * (D + 4); };
    auto fetch = [&](int w) {                    // nothing behind the last window, but counted as the others are
      if (w < windows) {
        if constexpr (TERMS == 1) k_rows.fetch(reinterpret_cast<T*>(keys_of(w)), KP, token0 + w * C, n);
        else k_rows.fetch(raw_of(w), D + 4, token0 + w * C, n);
        v_rows.fetch(values_of(w), VP, token0 + w * C, n);
        uint8_t* to = reinterpret_cast<uint8_t*>(&record_of(w));
#pragma unroll
        for (int i = 0; i < (int)sizeof(Record); i += 16 * GROUP)
          if ((int)sizeof(Record) % (16 * GROUP) == 0 || i + tid * 16 < (int)sizeof(Record)) copy16(to + i + tid * 16, left + (int64_t)w * sizeof(Record) + i + tid * 16, true);
      }
      copies_commit();
    };
#pragma unroll
    for (int i = 0; i < H::AHEAD; ++i) fetch(i);
    for (int step = -2; step <= windows; ++step) {
      const int w = step + 2;
      if (w < windows) {
        copies_wait<H::AHEAD - 1>();
        if constexpr (TERMS == 3) {
          barrier(1 + LOAD);
          __nv_bfloat16* ks = keys_of(w);
          const float* from = reinterpret_cast<const float*>(raw_of(w));
          for (int i = tid; i < C * (D / 2); i += GROUP) {
            const int r = i / (D / 2), c = i % (D / 2) * 2;
            const float2 f = *reinterpret_cast<const float2*>(from + r * (D + 4) + c);
            uint32_t terms[3];
            cut(f.x, f.y, terms);
#pragma unroll
            for (int x = 0; x < 3; ++x) *reinterpret_cast<uint32_t*>(ks + x * H::TILE + r * KP + c) = terms[x];
          }
          barrier(1 + LOAD);
        }
        fetch(w + H::AHEAD);
      }
      __syncthreads();
    }
  } else if (role == OUT) {
    // ------------------------------------------------------------------------------- out
    // eight tokens to a warp
    constexpr int EACH = 16 / (int)sizeof(T);
    const int i0 = 8 * warp;
    const bool both = warp >= 2;
    const Rows<T, D> q_rows(q, p.q.t, tid);
    auto queries_of = [&](int w) { return queries + (w % H::Q_PLACES) * C * QP; };
    auto fetch = [&](int w) {
      if (w < windows) q_rows.fetch(queries_of(w), QP, token0 + w * C, n);
      copies_commit();
    };
#pragma unroll
    for (int i = 0; i < H::AHEAD - 1; ++i) fetch(i);
    float acc[NS][2][4];                 // columns of values 16 i + g and + 8, tokens 2t and 2t + 1
    uint32_t weights[TK][SEEN][2];
    for (int step = -2; step <= windows; ++step) {
      // the last product of the window before
      if (step >= 1 && !slow[(step - 1) & 1]) {
        const int w = step - 1;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
#pragma unroll
          for (int x = 0; x < TK; ++x)
            if (x == 0 || both) {
              uint32_t a[SEEN][4];
#pragma unroll
              for (int e = 0; e < SEEN; ++e) load16(a[e], u_seen + ((((w & 1) * NS + i) * SEEN + e) * TK + x) * 128 + lane * 4);
              product(acc[i][x], a, weights[x]);
            }
          T* to = outs + (i0 + 2 * t) * VP + 16 * i + g;
          to[0] = (T)(acc[i][0][0] + acc[i][1][0]);
          to[VP] = (T)(acc[i][0][1] + acc[i][1][1]);
          to[8] = (T)(acc[i][0][2] + acc[i][1][2]);
          to[VP + 8] = (T)(acc[i][0][3] + acc[i][1][3]);
        }
        __syncwarp();
        for (int e = lane; e < 8 * (COLS / EACH); e += 32) {
          const int r = i0 + e / (COLS / EACH), c = e % (COLS / EACH) * EACH;
          const int token = token0 + w * C + r;
          if (token < n) *reinterpret_cast<uint4*>(o + (int64_t)token * p.o.t + c) = *reinterpret_cast<const uint4*>(outs + r * VP + c);
        }
        __syncwarp();
      }
      if (step >= -1) fetch(step + H::AHEAD);
      if (step >= 0 && step < windows) {
        const int w = step;
        const T* qs = queries_of(w);
        const Record& record = record_of(w);
#pragma unroll
        for (int x = 0; x < TK; ++x)
          if (x == 0 || both)
#pragma unroll
            for (int e = 0; e < SEEN; ++e) {
              const uint2 f = *reinterpret_cast<const uint2*>(record.weights[delta_place(warp, x)][e][lane]);
              weights[x][e][0] = f.x; weights[x][e][1] = f.y;
            }
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) acc[i][e][0] = acc[i][e][1] = acc[i][e][2] = acc[i][e][3] = 0.f;
#pragma unroll
        for (int x = 0; x < KS; x += 2) {        // 32 elements
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
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              uint32_t a[SEEN][4];
#pragma unroll
              for (int e = 0; e < SEEN; ++e) load16(a[e], s_seen + ((((w & 1) * NS + i) * SEEN + e) * KS + x + z) * 128 + lane * 4);
              product(acc[i][z], a, f[z]);
            }
        }
        const float2 up = *reinterpret_cast<const float2*>(record.up + i0 + 2 * t);
        const float gain[2] = {p.scale * up.x, p.scale * up.y};
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[i][0][e] = (acc[i][0][e] + acc[i][1][e]) * gain[e & 1];
            acc[i][1][e] = 0.f;
          }
      }
      copies_wait<H::AHEAD - 1>();
      __syncthreads();
    }
  } else {
    // ------------------------------------------------------------------------------- the chain
    // rows: value columns 16 i + g and + 8; columns: elements 2t and 2t + 1 of the warp's tiles of 8
    float s[NS][NT][4];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][x][e] = p.state[state + (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + 16 * i + g + 8 * (e >> 1)];
    // the state before window w as an operand: what it says of the window's keys, this warp's part, and its terms for out
    auto ask = [&](int w) {
      const __nv_bfloat16* ks = keys_of(w);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        uint32_t a[SK][3][4];
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            uint32_t terms[3];
            cut(s[i][x][2 * r], s[i][x][2 * r + 1], terms);
#pragma unroll
            for (int e = 0; e < 3; ++e) {
              a[x / 2][e][2 * (x & 1) + r] = terms[e];
              if (NT == 1) a[0][e][2 + r] = 0u;
            }
          }
        float acc[TT][4];
#pragma unroll
        for (int c = 0; c < TT; ++c) acc[c][0] = acc[c][1] = acc[c][2] = acc[c][3] = 0.f;
        // four blocks of 8 tokens x 8 elements a load: 4 / NT tiles of tokens
#pragma unroll
        for (int c = 0; c < TT; c += 4 / NT) {
          uint32_t f[TERMS][4];
#pragma unroll
          for (int e = 0; e < TERMS; ++e)
            ldmatrix4<false>(f[e], smem_u32(ks + e * H::TILE + (8 * (c + (lane >> 3) / NT) + (lane & 7)) * KP + (warp * NT + (lane >> 3) % NT) * 8));
#pragma unroll
          for (int z = 0; z < 4 / NT; ++z)
#pragma unroll
            for (int x = 0; x < SK; ++x) {
              uint32_t one[TERMS][2];
#pragma unroll
              for (int e = 0; e < TERMS; ++e) {
                one[e][0] = f[e][z * NT + 2 * x];
                one[e][1] = NT == 1 ? 0u : f[e][(z * NT + 2 * x + 1) % 4];
              }
              product(acc[c + z], a[x], one);
            }
        }
#pragma unroll
        for (int c = 0; c < TT; ++c) *reinterpret_cast<float4*>(x_part + ((i * 4 + warp) * TT + c) * 128 + lane * 4) = make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
#pragma unroll
        for (int e = 0; e < SEEN; ++e) {
          uint32_t* to = s_seen + (((w & 1) * NS + i) * SEEN + e) * KS * 128 + lane * 4;
          if (NT == 1) {
            *reinterpret_cast<uint2*>(to + (warp >> 1) * 128 + (warp & 1) * 2) = make_uint2(a[0][e][0], a[0][e][1]);
          } else {
#pragma unroll
            for (int x = 0; x < SK; ++x) *reinterpret_cast<uint4*>(to + (warp * SK + x) * 128) = make_uint4(a[x][e][0], a[x][e][1], a[x][e][2], a[x][e][3]);
          }
        }
      }
    };
    // A window with something in it that is not finite, token by token, a value column to a thread: the weights of 0 that a window's products give earlier tokens would
    // make NaN of it.
    auto advance_slowly = [&](int w) {
      float* st = x_part;                  // [COLS][D + 1]
      static_assert(COLS * (D + 1) * 4 <= H::X + H::R, "the state takes the place of the chain's operands");
      auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int x = 0; x < NT; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) f(s[i][x][e], st[(16 * i + g + 8 * (e >> 1)) * (D + 1) + (warp * NT + x) * 8 + 2 * t + (e & 1)]);
      };
      each([](float& mine, float& there) { there = mine; });
      barrier(1 + CHAIN);
      if (tid < COLS) {
        float* mine = st + tid * (D + 1);
        for (int i = token0 + w * C; i < min(n, token0 + w * C + C); ++i) {
          const T* kk = k + (int64_t)i * p.k.t;
          const T* qq = q + (int64_t)i * p.q.t;
          const float fade = p.log_decay ? expf(p.log_decay[gate0 + (int64_t)i * p.heads]) : 1.f;
          float said = 0.f, sum = 0.f;
          for (int e = 0; e < D; ++e) said = fmaf(to_float(kk[e]), fade * mine[e], said);
          const float u = p.beta[gate0 + (int64_t)i * p.heads] * (to_float(v[(int64_t)i * p.v.t + tid]) - said);
          for (int e = 0; e < D; ++e) {
            mine[e] = fmaf(fade, mine[e], to_float(kk[e]) * u);
            sum = fmaf(to_float(qq[e]), mine[e], sum);
          }
          o[(int64_t)i * p.o.t + tid] = (T)(p.scale * sum);
        }
      }
      barrier(1 + CHAIN);
      each([](float& mine, float& there) { mine = there; });
      barrier(1 + CHAIN);                  // the operands take the place back
    };
    auto advance = [&](int w) {
      const __nv_bfloat16* ks = keys_of(w);
      const T* vs = values_of(w);
      const Record& record = record_of(w);
      // R, U: of tokens 8 warp .. 8 warp + 7, whose sums over tokens reach up to them
      const int token = 8 * warp + 2 * t;
      const bool both = warp >= 2;
      uint32_t inv[2][3][2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x == 0 || both)
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            const uint2 z = *reinterpret_cast<const uint2*>(record.inverse[delta_place(warp, x)][e][lane]);
            inv[x][e][0] = z.x; inv[x][e][1] = z.y;
          }
      const float2 beta = *reinterpret_cast<const float2*>(record.beta + token), up = *reinterpret_cast<const float2*>(record.up + token),
                   down = *reinterpret_cast<const float2*>(record.down + token);
      const float whole = record.whole;
      bool odd = false;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        float4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const float4*>(x_part + ((i * 4 + e) * TT + warp) * 128 + lane * 4);
        const T* vv = vs + token * VP + 16 * i + g;
        float r[4];
        r[0] = beta.x * fmaf(-up.x, (x[0].x + x[1].x) + (x[2].x + x[3].x), to_float(vv[0]));
        r[1] = beta.y * fmaf(-up.y, (x[0].y + x[1].y) + (x[2].y + x[3].y), to_float(vv[VP]));
        r[2] = beta.x * fmaf(-up.x, (x[0].z + x[1].z) + (x[2].z + x[3].z), to_float(vv[8]));
        r[3] = beta.y * fmaf(-up.y, (x[0].w + x[1].w) + (x[2].w + x[3].w), to_float(vv[VP + 8]));
        keep<3>(r_frag + i * 3 * TK * 128, TK * 128, lane, warp, r);
        odd |= fmaf(r[0], 0.f, fmaf(r[1], 0.f, fmaf(r[2], 0.f, r[3] * 0.f))) != 0.f;
      }
      // something in the window or the state is not finite: nothing has been changed yet
      odd = named_barrier_or(1 + CHAIN, GROUP, odd);
      if (tid == 0) slow[w & 1] = odd;
      if (__builtin_expect(odd, 0)) {
        advance_slowly(w);
        return;
      }
      // U^T = R^T T^T
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        float u[2][3][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int e = 0; e < 3; ++e) u[x][e][0] = u[x][e][1] = u[x][e][2] = u[x][e][3] = 0.f;
          if (x == 0 || both) {
            uint32_t a[3][4];
#pragma unroll
            for (int e = 0; e < 3; ++e) load16(a[e], r_frag + ((i * 3 + e) * TK + x) * 128 + lane * 4);
            product_apart(u[x], a, inv[x]);
          }
        }
        float sum[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = (u[0][0][e] + u[1][0][e]) + ((u[0][1][e] + u[1][1][e]) + (u[0][2][e] + u[1][2][e]));
        const float faded[4] = {sum[0] * down.x, sum[1] * down.y, sum[2] * down.x, sum[3] * down.y};
        keep<3>(u_frag + i * 3 * TK * 128, TK * 128, lane, warp, faded);
        keep<SEEN>(u_seen + ((w & 1) * NS + i) * SEEN * TK * 128, TK * 128, lane, warp, sum);
      }
      uint32_t kf[NT][2][TERMS][2];
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int e = 0; e < TERMS; ++e) {
          uint32_t f[4];
          ldmatrix4<true>(f, smem_u32(ks + e * H::TILE + lane * KP + (warp * NT + m) * 8));
          kf[m][0][e][0] = f[0]; kf[m][0][e][1] = f[1]; kf[m][1][e][0] = f[2]; kf[m][1][e][1] = f[3];
        }
      barrier(1 + CHAIN);
      // S'^T = e^G_C S^T + U'^T K
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        uint32_t a[2][3][4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 3; ++e) load16(a[x][e], u_frag + ((i * 3 + e) * TK + x) * 128 + lane * 4);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          float d[2][4] = {};
          product(d[0], a[0], kf[m][0]);
          product(d[1], a[1], kf[m][1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][m][e] = fmaf(whole, s[i][m][e], d[0][e] + d[1][e]);
        }
      }
    };
    for (int step = -2; step <= windows; ++step) {
      if (step >= 0 && step < windows) advance(step);
      if (step >= -1 && step + 1 < windows) ask(step + 1);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) p.state_out[state + (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + 16 * i + g + 8 * (e >> 1)] = s[i][x][e];
  }
}

template <typename H>
cudaError_t launch_shape(const DeltaParams& p, cudaStream_t s) {
  static_assert(H::FITS, "shared memory");
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(delta_chunk_kernel<H>, cudaFuncAttributeMaxDynamicSharedMemorySize, H::SMEM); });
  if (e != cudaSuccess) return e;
  delta_chunk_kernel<H><<<dim3(H::D / H::COLS, (unsigned)p.heads, (unsigned)p.batch), THREADS, H::SMEM, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  const int64_t runs = (int64_t)p.batch * p.heads * (D / 16);
  if constexpr (sizeof(T) == 2)
    if (runs > 2 * PLAN_SMS) return launch_shape<Shape<T, D, 2>>(p, s);
  return launch_shape<Shape<T, D, 1>>(p, s);
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

// Windows to a range: records of one fit `most` bytes, or there is but one window to a range.
static int range_of(int batch, int tokens, int heads, bool bf16) {
  constexpr int64_t most = 96 << 20;
  const int64_t each = (int64_t)batch * heads * (int64_t)(bf16 ? sizeof(DeltaRecord<2>) : sizeof(DeltaRecord<3>)), all = ((int64_t)tokens + C - 1) / C;
  const int64_t fit = most / each < 1 ? 1 : most / each, ranges = (all + fit - 1) / fit;
  return (int)((all + ranges - 1) / ranges);
}
uint64_t delta_scratch(int batch, int tokens, int heads, bool bf16) {
  return (uint64_t)batch * heads * range_of(batch, tokens, heads, bf16) * (bf16 ? sizeof(DeltaRecord<2>) : sizeof(DeltaRecord<3>));
}

cudaError_t launch_delta_chunk(DeltaParams p, bool bf16, int D, cudaStream_t s) {
  const int all = (p.tokens + C - 1) / C;
  p.windows = range_of(p.batch, p.tokens, p.heads, bf16);
  for (p.first_window = 0; p.first_window < all; p.first_window += p.windows) {
    cudaError_t e = launch_delta_prepare(p, bf16, D, s);
    if (e == cudaSuccess) e = bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
    if (e != cudaSuccess) return e;
    p.state = p.state_out;
  }
  return cudaSuccess;
}

}  // namespace tok
}  // namespace tt

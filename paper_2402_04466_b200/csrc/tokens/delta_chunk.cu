// The gated delta rule over several tokens (tt_delta_rule), a window of C tokens at a time.
//
// Within a window let G_i be the sum of log_decay up to and including token i.  The corrections u_i then solve a triangular system,
//   u_i + sum_{j<i} beta_i e^(G_i - G_j) (k_i . k_j) u_j = beta_i (v_i - e^G_i S^T k_i)   or   (1 + A) U = R,
//   out_i = scale (e^G_i S^T q_i + sum_{j<=i} e^(G_i - G_j) (q_i . k_j) u_j),   S' = e^G_C S + sum_j e^(G_C - G_j) k_j u_j^T.
// What bounds a sequence is the chain S -> R -> U = (1 + A)^-1 R -> S'.  A block has four groups of four warps, each with one kind of work on a window of its own, which
// meet once a window: two windows ahead, A; one ahead, its inverse; the chain; and out, whose last product is taken a window behind.
//
// A block owns NS runs of 16 value columns of one head's state (the columns are independent of each other).  Everything on the chain is kept transposed, columns of
// values along M: the accumulators of one m16n8k16 product are then the other operand's registers of the next.  Each warp of the chain has a quarter of the keys' elements of the
// state in registers, as sums and as operands: X^T = S^T K^T comes in four parts, which the warps add up where they read them, then U^T = R^T T^T and
// S'^T = U'^T K.  R and U go from warp to warp as operands' registers, 16 bytes to a lane.  (A tcgen05 product of 16 columns takes 40 cycles however few its
// columns are, and its way through tensor memory twice that: the chain would be longer, not shorter.)
//
// The state is fp32, and so is everything between two products: an operand that is not bf16 to begin with is cut into three bf16 terms (8 + 8 + 8 bits), of whose
// products those of 2^-16 and more count.  Only what out alone reads is rounded further: in bf16 calls S, U and P (the weights of U in out) count with 16 bits.  (P rounded
// to bf16 once is not enough: of keys that repeat the corrections are many times larger than what is left of their sum.)
#include "linear_common.cuh"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = 32;                        // tokens of a window
constexpr int TT = C / 8, TK = C / 16;       // tiles of them, products along them
constexpr int GROUP = 128;                   // threads of a group: the chain, out, the inverse, A
constexpr int THREADS = 4 * GROUP;
enum { CHAIN = 0, OUT = 1, INVERSE = 2, SYSTEM = 3 };

template <typename T_, int D_, int NS_>
struct Shape {
  using T = T_;
  static constexpr int D = D_, NS = NS_;
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;       // of queries and keys
  static constexpr int SEEN = sizeof(T) == 2 ? 2 : 3;        // of S, U and P in out
  static constexpr int KS = D / 16;                          // products along a key
  static constexpr int NT = D / 32;                          // tiles of 8 keys' elements of the state to a warp
  static constexpr int SK = NT > 1 ? NT / 2 : 1;             // products along those
  static constexpr int COLS = 16 * NS;
  static constexpr int KP = D + 8, AP = C + 4, VP = COLS + 16 / (int)sizeof(T), QP = TERMS == 1 ? D + 8 : D + 4;   // pitches
  static constexpr int TILE = C * KP;                        // bf16 elements of one term of a window's keys
  // a window's keys are fetched three steps ahead; fp32 ones wait in `raw` to be cut
  static constexpr int K_PLACES = TERMS == 1 ? 4 : 3, V_PLACES = 4, G_PLACES = 4;
  static constexpr int RAW = TERMS == 1 ? 0 : C * (D + 4) * 4;
  static constexpr int K = K_PLACES * TERMS * TILE * 2, Q = 2 * C * QP * (int)sizeof(T), V = V_PLACES * C * VP * (int)sizeof(T);
  static constexpr int TRI = 2 * C * AP * 4, INV = 2 * TT * TK * 3 * 256;
  static constexpr int X = NS * 4 * TT * 512, R = NS * 3 * TK * 512, U = NS * 3 * TK * 512, SEEN_U = 2 * NS * SEEN * TK * 512, S = 2 * NS * SEEN * KS * 512;
  static constexpr int O = C * VP * (int)sizeof(T);
  static constexpr int GATES = G_PLACES * (5 * C + 4) * 4;
  static constexpr int SMEM = RAW + K + Q + V + TRI + INV + X + R + U + SEEN_U + S + O + GATES;
  static constexpr bool FITS = SMEM + 1024 <= 227 * 1024;
};

// a pair as three bf16 terms; a in the lower halves
__device__ __forceinline__ void cut(float a, float b, uint32_t (&t)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    t[i] = pack_bf16(a, b);
    a -= __uint_as_float(t[i] << 16);
    b -= __uint_as_float(t[i] & 0xFFFF0000u);
  }
}
// acc += A B, A of TA terms and B of TB, small products first: what is below the last term of the longer of the two is left out
template <int TA, int TB>
__device__ __forceinline__ void product(float (&acc)[4], const uint32_t (&a)[TA][4], const uint32_t (&b)[TB][2]) {
  constexpr int MOST = TA > TB ? TA : TB;
#pragma unroll
  for (int sum = MOST - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
        if (i + j == sum) mma16816(acc, a[i], b[j][0], b[j][1]);
}
// The same for a product that the chain waits for: 35 cycles an instruction behind another of the same sums, so each size of product has its own.
__device__ __forceinline__ void product_apart(float (&acc)[3][4], const uint32_t (&a)[3][4], const uint32_t (&b)[3][2]) {
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
      if (i <= sum) mma16816(acc[sum], a[i], b[sum - i][0], b[sum - i][1]);
}
__device__ __forceinline__ void load16(uint32_t (&r)[4], const uint32_t* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
}
// Accumulators (rows g and g + 8, columns 2t and 2t + 1 of tile n) as the first operand's registers of a product along n: term i's at `to` + i * term.
template <int TERMS>
__device__ __forceinline__ void keep(uint32_t* to, int term, int lane, int n, const float (&c)[4]) {
  uint32_t lo[3], hi[3];
  cut(c[0], c[1], lo);
  cut(c[2], c[3], hi);
#pragma unroll
  for (int i = 0; i < TERMS; ++i) *reinterpret_cast<uint2*>(to + i * term + (n >> 1) * 128 + lane * 4 + (n & 1) * 2) = make_uint2(lo[i], hi[i]);
}
__device__ __forceinline__ void barrier(int id) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "n"(GROUP) : "memory"); }
__device__ __forceinline__ void copy16(void* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ bool finite2(uint32_t u) { return (u & 0x7F800000u) != 0x7F800000u && (u & 0x7F80u) != 0x7F80u; }
template <typename T>
__device__ __forceinline__ bool all_finite(uint4 v) {
  if (sizeof(T) == 2) return finite2(v.x) && finite2(v.y) && finite2(v.z) && finite2(v.w);
  return isfinite(__uint_as_float(v.x)) && isfinite(__uint_as_float(v.y)) && isfinite(__uint_as_float(v.z)) && isfinite(__uint_as_float(v.w));
}
// Gates of a window's tokens.  G is a sum in 64 bits of log2(e) log_decay, kept as a pair of floats: what counts are differences of far larger sums.
struct Gates {
  float2 sum[C];                             // G
  float beta[C], up[C], down[C];             // e^G, e^(G_C - G)
  float whole;                               // e^G_C
  int odd;                                   // something in the window's keys, values or gates is not finite
  int pad[2];
};
// 2^x for x of 0 and below, as pair: to half a step of the result and little more, where exp2f is off by two.  By a Taylor polynomial of e^(y ln 2), |y| <= 1/2.
__device__ __forceinline__ float exp2_pair(float hi, float lo) {
  if (!(hi > -150.f)) return hi == hi ? 0.f : hi;
  const float whole = rintf(hi), y = ((hi - whole) + lo) * 0.693147181f;
  float f = 1.f / 5040.f;
  f = fmaf(f, y, 1.f / 720.f);
  f = fmaf(f, y, 1.f / 120.f);
  f = fmaf(f, y, 1.f / 24.f);
  f = fmaf(f, y, 1.f / 6.f);
  f = fmaf(f, y, 0.5f);
  f = fmaf(f, y, 1.f);
  f = fmaf(f, y, 1.f);
  return scalbnf(f, (int)whole);
}
// an 8 x 8 block of pairs' terms, rows for columns
__device__ __forceinline__ uint32_t transposed(uint32_t u) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(u));
  return r;
}
__device__ __forceinline__ float fade_of(float2 to, float2 from) { return exp2_fast((to.x - from.x) + (to.y - from.y)); }

// A group's rows of a window, 16 bytes to a thread and pass
template <typename T, int ROWLEN>
struct Rows {
  static constexpr int EACH = 16 / (int)sizeof(T), ROW = ROWLEN / EACH, STEP = GROUP / ROW, PASSES = (C + STEP - 1) / STEP;
  const T* src;
  int64_t stride;
  int row, col;
  __device__ __forceinline__ Rows(const T* base, int64_t token_stride, int tid) : src(base), stride(token_stride), row(tid / ROW), col(tid % ROW * EACH) {}
  __device__ __forceinline__ void fetch(T* dst, int pitch, int first, int n) const {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = row + i * STEP;
      if (STEP * PASSES > C && r >= C) break;
      const bool there = first + r < n;
      copy16(dst + r * pitch + col, src + (there ? (int64_t)(first + r) * stride : 0) + col, there);
    }
  }
  __device__ __forceinline__ bool finite(const T* dst, int pitch) const {
    bool fine = true;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = row + i * STEP;
      if (STEP * PASSES > C && r >= C) break;
      fine &= all_finite<T>(*reinterpret_cast<const uint4*>(dst + r * pitch + col));
    }
    return fine;
  }
};

template <typename H>
__global__ void __launch_bounds__(THREADS, 1) delta_chunk_kernel(const __grid_constant__ DeltaParams p) {
  using T = typename H::T;
  constexpr int D = H::D, NS = H::NS, TERMS = H::TERMS, SEEN = H::SEEN, KS = H::KS, NT = H::NT, SK = H::SK, COLS = H::COLS, KP = H::KP,
                AP = H::AP, VP = H::VP, QP = H::QP;
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* place = smem;
  auto room = [&](int bytes) {
    uint8_t* r = place;
    place += bytes;
    return r;
  };
  float* raw = reinterpret_cast<float*>(room(H::RAW));                       // [C][D + 4]
  __nv_bfloat16* keys = reinterpret_cast<__nv_bfloat16*>(room(H::K));        // [place][term][C][KP]
  T* queries = reinterpret_cast<T*>(room(H::Q));                             // [parity][C][QP]
  T* values = reinterpret_cast<T*>(room(H::V));                              // [place][C][VP]
  float* tri = reinterpret_cast<float*>(room(H::TRI));                       // [parity][C][AP]: A, then its inverse
  uint32_t* inverse = reinterpret_cast<uint32_t*>(room(H::INV));             // [parity][tile][TK][term][lane][2]
  float* x_part = reinterpret_cast<float*>(room(H::X));                      // [run][warp][tile][lane][4]
  uint32_t* r_frag = reinterpret_cast<uint32_t*>(room(H::R));                // [run][term][TK][lane][4]
  uint32_t* u_frag = reinterpret_cast<uint32_t*>(room(H::U));                // [run][term][TK][lane][4], faded to the window's end
  uint32_t* u_seen = reinterpret_cast<uint32_t*>(room(H::SEEN_U));           // [parity][run][term][TK][lane][4]
  uint32_t* s_seen = reinterpret_cast<uint32_t*>(room(H::S));                // [parity][run][term][KS][lane][4]
  T* outs = reinterpret_cast<T*>(room(H::O));                                // [C][VP]
  Gates* gates = reinterpret_cast<Gates*>(place);                      // [place]
  static_assert(sizeof(Gates) * H::G_PLACES == H::GATES, "gates");

  const int b = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * COLS;
  const int n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int role = __shfl_sync(0xffffffffu, (int)(threadIdx.x / GROUP), 0), warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5) & 3, 0);
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, tid = threadIdx.x % GROUP;
  const int windows = (n + C - 1) / C, hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col0;
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col0;
  const int64_t gate0 = (int64_t)b * p.tokens * p.heads + h;
  const int64_t state = ((int64_t)slot * p.heads + h) * D * D + col0;
  auto keys_of = [&](int w) { return keys + (w % H::K_PLACES) * TERMS * H::TILE; };
  auto values_of = [&](int w) { return values + (w % H::V_PLACES) * C * VP; };
  auto gates_of = [&](int w) -> Gates& { return gates[w % H::G_PLACES]; };

  if (role == SYSTEM) {
    // ------------------------------------------------------------------------------- A, two windows ahead
    const Rows<T, D> k_rows(k, p.k.t, tid);
    const Rows<T, COLS> v_rows(v, p.v.t, tid);
    auto fetch = [&](int w) {
      if constexpr (TERMS == 1) k_rows.fetch(reinterpret_cast<T*>(keys_of(w)), KP, w * C, n);
      else k_rows.fetch(reinterpret_cast<T*>(raw), D + 4, w * C, n);
      v_rows.fetch(values_of(w), VP, w * C, n);
      copies_commit();
    };
    float decay = 0.f, beta = 0.f;               // of a lane's token, in the first warp
    auto fetch_gates = [&](int w) {
      const int token = w * C + lane;
      decay = beta = 0.f;
      if (token >= n) return;
      if (p.log_decay) decay = p.log_decay[gate0 + (int64_t)token * p.heads];
      beta = p.beta[gate0 + (int64_t)token * p.heads];
    };
    if (windows > 0) {
      if (warp == 0) fetch_gates(0);
      fetch(0);
    }
    for (int step = -2; step <= windows; ++step) {
      const int w = step + 2;
      if (w < windows) {
        Gates& gt = gates_of(w);
        copies_wait();
        bool odd = !v_rows.finite(values_of(w), VP);
        if constexpr (TERMS == 1) odd |= !k_rows.finite(reinterpret_cast<const T*>(keys_of(w)), KP);
        else odd |= !k_rows.finite(reinterpret_cast<const T*>(raw), D + 4);
        if (warp == 0) {
          odd |= !isfinite(beta) || !(decay < INFINITY);
          // -infinity: all of it, like -10^5
          double sum = (decay < -1e5f ? -1e5 : (double)decay) * 1.4426950408889634074;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const double other = __shfl_up_sync(0xffffffffu, sum, d);
            if (lane >= d) sum += other;
          }
          const float hi = (float)sum, lo = (float)(sum - (double)hi);
          const float2 all = make_float2(__shfl_sync(0xffffffffu, hi, 31), __shfl_sync(0xffffffffu, lo, 31));
          gt.sum[lane] = make_float2(hi, lo);
          gt.beta[lane] = beta;
          gt.up[lane] = exp2f(hi + lo);
          gt.down[lane] = exp2f((all.x - hi) + (all.y - lo));
          // the one factor that a state meets again and again: its error would add up
          if (lane == 31) gt.whole = exp2_pair(hi, lo);
        }
        odd = named_barrier_or(1 + SYSTEM, GROUP, odd);
        if (tid == 0) gt.odd = odd;
        __nv_bfloat16* ks = keys_of(w);
        if constexpr (TERMS == 3) {
          for (int i = tid; i < C * (D / 2); i += GROUP) {
            const int r = i / (D / 2), c = i % (D / 2) * 2;
            const float2 f = *reinterpret_cast<const float2*>(raw + r * (D + 4) + c);
            uint32_t terms[3];
            cut(f.x, f.y, terms);
#pragma unroll
            for (int x = 0; x < 3; ++x) *reinterpret_cast<uint32_t*>(ks + x * H::TILE + r * KP + c) = terms[x];
          }
          barrier(1 + SYSTEM);
        }
        if (w + 1 < windows) {
          fetch(w + 1);
          if (warp == 0) fetch_gates(w + 1);
        }
        // 16 rows to a warp, or to two that share their columns' tiles: those up to the diagonal's
        constexpr int SHARE = 4 / TK;
        const int strip = warp % TK, first = warp / TK;
        float acc[TT / SHARE][4];
#pragma unroll
        for (int i = 0; i < TT / SHARE; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
        for (int x = 0; x < KS; x += 2) {        // 32 elements
          uint32_t a[2][TERMS][4];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < TERMS; ++i) ldmatrix4<false>(a[e][i], smem_u32(ks + i * H::TILE + (16 * strip + (lane & 15)) * KP + (x + e) * 16 + (lane >> 4) * 8));
#pragma unroll
          for (int i = 0; i < TT / SHARE; ++i) {
            const int c = first + SHARE * i;
            if (c < 2 * strip + 2) {
              uint32_t one[TERMS][2], two[TERMS][2];
#pragma unroll
              for (int e = 0; e < TERMS; ++e) {
                uint32_t f[4];
                ldmatrix4<false>(f, smem_u32(ks + e * H::TILE + (8 * c + (lane & 7)) * KP + x * 16 + (lane >> 3) * 8));
                one[e][0] = f[0]; one[e][1] = f[1]; two[e][0] = f[2]; two[e][1] = f[3];
              }
              product(acc[i], a[0], one);
              product(acc[i], a[1], two);
            }
          }
        }
        float* A = tri + (w & 1) * C * AP;
        const int i0 = 16 * strip + g;
        const float2 sums[2] = {gt.sum[i0], gt.sum[i0 + 8]};
        const float betas[2] = {gt.beta[i0], gt.beta[i0 + 8]};
#pragma unroll
        for (int i = 0; i < TT / SHARE; ++i) {
          const int c = first + SHARE * i;
          if (c < 2 * strip + 2) {
            const int j = 8 * c + 2 * t;
            const float4 from = *reinterpret_cast<const float4*>(gt.sum + j);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float f0 = betas[r] * fade_of(sums[r], make_float2(from.x, from.y)) * acc[i][2 * r], f1 = betas[r] * fade_of(sums[r], make_float2(from.z, from.w)) * acc[i][2 * r + 1];
              *reinterpret_cast<float2*>(A + (i0 + 8 * r) * AP + j) = make_float2(j < i0 + 8 * r ? f0 : 0.f, j + 1 < i0 + 8 * r ? f1 : 0.f);
            }
          }
        }
      }
      __syncthreads();
    }
  } else if (role == INVERSE) {
    // ------------------------------------------------------------------------------- (1 + A)^-1, a window ahead
    for (int step = -2; step <= windows; ++step) {
      const int w = step + 1;
      if (w >= 0 && w < windows) {
        float* A = tri + (w & 1) * C * AP;
        uint32_t* to = inverse + (w & 1) * TT * TK * 3 * 64;
        auto put = [&](int tile, int x, int e, uint32_t b0, uint32_t b1) { *reinterpret_cast<uint2*>(to + (((tile * TK + x) * 3 + e) * 32 + lane) * 2) = make_uint2(b0, b1); };
        // the two blocks of 16 on the diagonal, a column to a lane
        float* block = A + warp * 16 * (AP + 1);
        if (warp < 2) {
          const int j = lane & 15;
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float a[16];
#pragma unroll
            for (int m = 0; m < i; m += 4) {
              const float4 f = *reinterpret_cast<const float4*>(block + i * AP + m);
              a[m] = f.x; a[m + 1] = f.y; a[m + 2] = f.z; a[m + 3] = f.w;
            }
            float sum = i == j ? 1.f : 0.f, other = 0.f;      // two chains
#pragma unroll
            for (int m = 0; m < i; ++m)
              if (m & 1) other = fmaf(-a[m], x[m], other);
              else sum = fmaf(-a[m], x[m], sum);
            x[i] = sum + other;
          }
          __syncwarp();
          if (lane < 16)
#pragma unroll
            for (int i = 0; i < 16; ++i) block[i * AP + j] = x[i];
        }
        barrier(1 + INVERSE);
        if (warp < 2) {
          // as the second operand's registers of U's product
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t terms[2][3];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 f = *reinterpret_cast<const float2*>(block + (8 * i + g) * AP + 8 * e + 2 * t);
              cut(f.x, f.y, terms[e]);
            }
#pragma unroll
            for (int e = 0; e < 3; ++e) put(2 * warp + i, warp, e, terms[0][e], terms[1][e]);
          }
        } else if (warp == 2) {
          // the block below, -T_11 A_10 T_00, transposed as the chain is: (T_00^T A_10^T) T_11^T
          uint32_t a[3][4], f[2][3][2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t terms[3];
            const float* from = A + (2 * t + 8 * (e >> 1)) * AP + g + 8 * (e & 1);
            cut(from[0], from[AP], terms);
#pragma unroll
            for (int c = 0; c < 3; ++c) a[c][e] = terms[c];
          }
          auto second = [&](const float* rows) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint32_t terms[3];
                const float2 x = *reinterpret_cast<const float2*>(rows + (8 * i + g) * AP + 8 * e + 2 * t);
                cut(x.x, x.y, terms);
#pragma unroll
                for (int c = 0; c < 3; ++c) f[i][c][e] = terms[c];
              }
          };
          float sums[2][3][4];
          auto multiply = [&](float sign) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
              for (int c = 0; c < 3; ++c) sums[i][c][0] = sums[i][c][1] = sums[i][c][2] = sums[i][c][3] = 0.f;
              product_apart(sums[i], a, f[i]);
#pragma unroll
              for (int e = 0; e < 4; ++e) sums[i][0][e] = sign * (sums[i][0][e] + (sums[i][1][e] + sums[i][2][e]));
            }
          };
          second(A + 16 * AP);
          multiply(1.f);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t terms[3];
            cut(sums[e >> 1][0][2 * (e & 1)], sums[e >> 1][0][2 * (e & 1) + 1], terms);
#pragma unroll
            for (int c = 0; c < 3; ++c) a[c][e] = terms[c];
          }
          second(A + 16 * (AP + 1));
          multiply(-1.f);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t low[3], high[3];
            cut(sums[i][0][0], sums[i][0][1], low);
            cut(sums[i][0][2], sums[i][0][3], high);
#pragma unroll
            for (int e = 0; e < 3; ++e) put(2 + i, 0, e, transposed(low[e]), transposed(high[e]));
          }
        }
      }
      __syncthreads();
    }
  } else if (role == OUT) {
    // ------------------------------------------------------------------------------- out
    // 16 tokens to a warp, or to two that share the runs of columns
    constexpr int SHARE = 4 / TK, MINE = (NS + SHARE - 1) / SHARE;
    constexpr int EACH = 16 / (int)sizeof(T);
    const int strip = warp % TK, first = warp / TK, i0 = 16 * strip;
    const Rows<T, D> q_rows(q, p.q.t, tid);
    float acc[MINE][2][4];               // columns of values 16 x g and + 8, tokens 8 e + 2 t and + 1 of the strip
    uint32_t weights[TK][2][SEEN][2];
    for (int step = -2; step <= windows; ++step) {
      // the last product of the window before
      if (step >= 1 && first < NS && !gates_of(step - 1).odd) {
        const int w = step - 1;
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
          const int i = first + SHARE * m;
          if (i >= NS) break;
#pragma unroll
          for (int x = 0; x < TK; ++x)
            if (x <= strip) {
              uint32_t a[SEEN][4];
#pragma unroll
              for (int e = 0; e < SEEN; ++e) load16(a[e], u_seen + ((((w & 1) * NS + i) * SEEN + e) * TK + x) * 128 + lane * 4);
              product(acc[m][0], a, weights[x][0]);
              product(acc[m][1], a, weights[x][1]);
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            T* to = outs + (i0 + 8 * e + 2 * t) * VP + 16 * i + g;
            to[0] = (T)acc[m][e][0];
            to[VP] = (T)acc[m][e][1];
            to[8] = (T)acc[m][e][2];
            to[VP + 8] = (T)acc[m][e][3];
          }
          __syncwarp();
          for (int e = lane; e < 16 * (16 / EACH); e += 32) {
            const int r = i0 + e / (16 / EACH), c = 16 * i + e % (16 / EACH) * EACH;
            if (w * C + r < n) *reinterpret_cast<uint4*>(o + (int64_t)(w * C + r) * p.o.t + c) = *reinterpret_cast<const uint4*>(outs + r * VP + c);
          }
        }
        __syncwarp();
      }
      if (step >= -1 && step + 1 < windows) {
        q_rows.fetch(queries + ((step + 1) & 1) * C * QP, QP, (step + 1) * C, n);
        copies_commit();
      }
      if (step >= 0 && step < windows && first < NS) {
        const int w = step;
        const T* qs = queries + (w & 1) * C * QP;
        const __nv_bfloat16* ks = keys_of(w);
        const Gates& gt = gates_of(w);
        float dots[TT][4];
#pragma unroll
        for (int i = 0; i < TT; ++i) dots[i][0] = dots[i][1] = dots[i][2] = dots[i][3] = 0.f;
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) acc[m][e][0] = acc[m][e][1] = acc[m][e][2] = acc[m][e][3] = 0.f;
#pragma unroll
        for (int x = 0; x < KS; ++x) {
          // the strip's queries as the first operand; as the second, registers 0 and 2 are its first eight tokens, 1 and 3 the others
          uint32_t a[TERMS][4];
          if constexpr (TERMS == 1) {
            ldmatrix4<false>(a[0], smem_u32(qs + (i0 + (lane & 15)) * QP + x * 16 + (lane >> 4) * 8));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 f = *reinterpret_cast<const float2*>(qs + (i0 + g + 8 * (e & 1)) * QP + x * 16 + 8 * (e >> 1) + 2 * t);
              uint32_t terms[3];
              cut(f.x, f.y, terms);
#pragma unroll
              for (int c = 0; c < 3; ++c) a[c][e] = terms[c];
            }
          }
          uint32_t one[TERMS][2], two[TERMS][2];
#pragma unroll
          for (int e = 0; e < TERMS; ++e) {
            one[e][0] = a[e][0]; one[e][1] = a[e][2];
            two[e][0] = a[e][1]; two[e][1] = a[e][3];
          }
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            const int i = first + SHARE * m;
            if (i >= NS) break;
            uint32_t f[SEEN][4];
#pragma unroll
            for (int e = 0; e < SEEN; ++e) load16(f[e], s_seen + ((((w & 1) * NS + i) * SEEN + e) * KS + x) * 128 + lane * 4);
            product(acc[m][0], f, one);
            product(acc[m][1], f, two);
          }
#pragma unroll
          for (int c = 0; c < TT; c += 2)
            if (c <= 2 * strip) {
              uint32_t left[TERMS][2], right[TERMS][2];
#pragma unroll
              for (int e = 0; e < TERMS; ++e) {
                uint32_t f[4];
                ldmatrix4<false>(f, smem_u32(ks + e * H::TILE + (8 * c + (lane & 7) + 8 * (lane >> 4)) * KP + x * 16 + ((lane >> 3) & 1) * 8));
                left[e][0] = f[0]; left[e][1] = f[1]; right[e][0] = f[2]; right[e][1] = f[3];
              }
              product(dots[c], a, left);
              product(dots[c + 1], a, right);
            }
        }
        // P, and the part of the state
        const int at = i0 + g;
        const float2 sums[2] = {gt.sum[at], gt.sum[at + 8]};
#pragma unroll
        for (int c = 0; c < TT; ++c)
          if (c < 2 * strip + 2) {
            const int j = 8 * c + 2 * t;
            const float4 from = *reinterpret_cast<const float4*>(gt.sum + j);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float f0 = p.scale * fade_of(sums[r], make_float2(from.x, from.y)) * dots[c][2 * r], f1 = p.scale * fade_of(sums[r], make_float2(from.z, from.w)) * dots[c][2 * r + 1];
              uint32_t terms[3];
              cut(j <= at + 8 * r ? f0 : 0.f, j + 1 <= at + 8 * r ? f1 : 0.f, terms);
#pragma unroll
              for (int e = 0; e < SEEN; ++e) weights[c >> 1][r][e][c & 1] = terms[e];
            }
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 up = *reinterpret_cast<const float2*>(gt.up + i0 + 8 * e + 2 * t);
#pragma unroll
          for (int m = 0; m < MINE; ++m) {
            acc[m][e][0] *= p.scale * up.x; acc[m][e][1] *= p.scale * up.y;
            acc[m][e][2] *= p.scale * up.x; acc[m][e][3] *= p.scale * up.y;
          }
        }
      }
      copies_wait();
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
    auto advance = [&](int w) {
      const __nv_bfloat16* ks = keys_of(w);
      const T* vs = values_of(w);
      const Gates& gt = gates_of(w);
      // R, U: of tokens 8 warp .. 8 warp + 7, whose sums over tokens reach up to them
      const int token = 8 * warp + 2 * t;
      const bool both = warp >= 2;
      uint32_t inv[2][3][2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x == 0 || both)
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            const uint2 z = *reinterpret_cast<const uint2*>(inverse + ((((w & 1) * TT + warp) * TK + x) * 3 + e) * 64 + lane * 2);
            inv[x][e][0] = z.x; inv[x][e][1] = z.y;
          }
      const float2 beta = *reinterpret_cast<const float2*>(gt.beta + token), up = *reinterpret_cast<const float2*>(gt.up + token),
                   down = *reinterpret_cast<const float2*>(gt.down + token);
      const float whole = gt.whole;
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
      }
      barrier(1 + CHAIN);
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
        for (int i = w * C; i < min(n, w * C + C); ++i) {
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
    for (int step = -2; step <= windows; ++step) {
      if (step >= 0 && step < windows) {
        if (gates_of(step).odd) advance_slowly(step);
        else advance(step);
      }
      if (step >= -1 && step + 1 < windows) ask(step + 1);
      __syncthreads();
    }
    if (windows > 0 || p.state_out != p.state)
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
  if constexpr (Shape<T, D, 2>::FITS)
    if (runs > 2 * PLAN_SMS) return launch_shape<Shape<T, D, 2>>(p, s);
  return launch_shape<Shape<T, D, 1>>(p, s);
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

cudaError_t launch_delta_chunk(const DeltaParams& p, bool bf16, int D, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
}

}  // namespace tok
}  // namespace tt

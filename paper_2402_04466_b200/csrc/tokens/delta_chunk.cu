// The gated delta rule over several tokens (tt_delta_rule), a window of C tokens at a time.
//
// Within a window let G_i be the sum of log_decay up to and including token i.  The corrections u_i then solve a triangular system,
//   u_i + sum_{j<i} beta_i e^(G_i - G_j) (k_i . k_j) u_j = beta_i (v_i - e^G_i S^T k_i)   or   (1 + A) U = R,
//   out_i = scale (e^G_i S^T q_i + sum_{j<=i} e^(G_i - G_j) (q_i . k_j) u_j),   S' = e^G_C S + sum_j e^(G_C - G_j) k_j u_j^T.
// T = (1 + A)^-1 and the weights P of U in out depend on no state: half of the block's warps work them out for the next window while the other half takes this one's
// state along, which is the chain that bounds a sequence:  S -> R -> U = T R -> S'.
//
// A block owns NS runs of 16 value columns of one head's state (the columns are independent of each other).  Everything on the chain is kept transposed, columns of
// values along M: the accumulators of one m16n8k16 product are then the other operand's registers of the next, X^T = S^T K^T, U^T = R^T T^T,
// S'^T = U'^T K, and what warps exchange lies in shared memory as those registers, 16 bytes to a lane.  (A tcgen05 product of 16 columns takes 40 cycles however few
// its columns are, and its way through tensor memory twice that: the chain would be longer, not shorter.)
//
// The state is fp32, and so is everything between two products: an operand that is not bf16 to begin with is cut into three bf16 terms (8 + 8 + 8 bits), of whose
// products those of 2^-16 and more count.  Only what out alone reads is rounded further: in bf16 calls S, U and P count with 16 bits.  (P rounded to bf16 once
// is not enough: of keys that repeat the corrections are many times larger than what is left of their sum.)
#include "linear_common.cuh"

#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = 32;                        // tokens of a window
constexpr int GROUP = 128;                   // threads of the chain, and of the preparation
constexpr int THREADS = 2 * GROUP;

template <typename T, int D, int NS>
struct Shape {
  static constexpr int TERMS = sizeof(T) == 2 ? 1 : 3;       // of queries and keys
  static constexpr int SEEN = sizeof(T) == 2 ? 2 : 3;        // of S, U and P in out
  static constexpr int KS = D / 16;                          // products along a key
  static constexpr int NT = D / 8 / 4;                       // tiles of 8 keys' elements of the state to a warp
  static constexpr int COLS = 16 * NS;
  static constexpr int KP = D + 8, PP = C + 8, TP = C + 4, VP = COLS + 16 / (int)sizeof(T);   // pitches
  static constexpr int TILE = C * KP;                        // bf16 elements of one term of keys or queries
  static constexpr int STAGES = 3;
  // bf16 tiles are copied where they are used; fp32 ones wait in `raw` to be cut, and their terms have two places
  static constexpr int PLACES = TERMS == 1 ? STAGES : 2;
  static constexpr int RAW = TERMS == 1 ? 0 : 2 * C * (D + 4) * 4;
  static constexpr int KQ = PLACES * 2 * TERMS * TILE * 2;
  static constexpr int V = STAGES * C * VP * (int)sizeof(T);
  static constexpr int TRI = 2 * C * TP * 4, Y = 16 * 20 * 4, P = 2 * SEEN * C * PP * 2;
  static constexpr int S = NS * 3 * KS * 512, R = NS * 3 * (C / 16) * 512, U = NS * (3 + SEEN) * (C / 16) * 512;
  static constexpr int OUT = C * VP * (int)sizeof(T);
  static constexpr int GATES = 2 * (4 * C + 4) * 4;
  static constexpr int SMEM = RAW + KQ + V + TRI + Y + P + S + R + U + OUT + GATES;
  static_assert(SMEM + 1024 <= 227 * 1024, "shared memory");
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
// acc += A B, A of TA terms and B of TB: what is below the last term of the longer of the two is left out, and the products of the largest terms add up apart
template <int TA, int TB>
__device__ __forceinline__ void product(float (&most)[4], float (&rest)[4], const uint32_t (&a)[TA][4], const uint32_t (&b)[TB][2]) {
#pragma unroll
  for (int i = 0; i < TA; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j)
      if (i + j < (TA > TB ? TA : TB)) mma16816(i + j == 0 ? most : rest, a[i], b[j][0], b[j][1]);
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
__device__ __forceinline__ bool finite2(uint32_t u) { return (u & 0x7F800000u) != 0x7F800000u && (u & 0x7F80u) != 0x7F80u; }
template <typename T>
__device__ __forceinline__ bool all_finite(uint4 v) {
  if (sizeof(T) == 2) return finite2(v.x) && finite2(v.y) && finite2(v.z) && finite2(v.w);
  return isfinite(__uint_as_float(v.x)) && isfinite(__uint_as_float(v.y)) && isfinite(__uint_as_float(v.z)) && isfinite(__uint_as_float(v.w));
}
// gates of a window's tokens; `odd`: something in its keys, values or gates is not finite
struct Gates {
  float beta[C], up[C], down[C], sum[C];     // e^G, e^(G_C - G)
  float whole, low;                          // e^G_C
  int odd, pad;
};

template <typename T, int D, int NS>
__global__ void __launch_bounds__(THREADS) delta_chunk_kernel(const __grid_constant__ DeltaParams p) {
  using H = Shape<T, D, NS>;
  constexpr int TERMS = H::TERMS, SEEN = H::SEEN, KS = H::KS, NT = H::NT, COLS = H::COLS, KP = H::KP, PP = H::PP, TP = H::TP, VP = H::VP;
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* at = smem;
  auto room = [&](int bytes) {
    uint8_t* r = at;
    at += bytes;
    return r;
  };
  float* raw = reinterpret_cast<float*>(room(H::RAW));                       // [keys, queries][C][D + 4]
  __nv_bfloat16* kq = reinterpret_cast<__nv_bfloat16*>(room(H::KQ));         // [place][keys, queries][term][C][KP]
  T* vs = reinterpret_cast<T*>(room(H::V));                                  // [stage][C][VP]
  float* tri = reinterpret_cast<float*>(room(H::TRI));                       // [parity][C][TP]: A, then T
  float* y = reinterpret_cast<float*>(room(H::Y));                           // [16][20]
  __nv_bfloat16* ps = reinterpret_cast<__nv_bfloat16*>(room(H::P));          // [parity][SEEN terms][C][PP]
  uint32_t* s_frag = reinterpret_cast<uint32_t*>(room(H::S));                // [run][term][KS][lane][4]
  uint32_t* r_frag = reinterpret_cast<uint32_t*>(room(H::R));                // [run][term][C / 16][lane][4]
  uint32_t* u_frag = reinterpret_cast<uint32_t*>(room(H::U));                // [run][3 faded terms, SEEN plain ones][C / 16][lane][4]
  T* outs = reinterpret_cast<T*>(room(H::OUT));                              // [C][VP]
  Gates* gates = reinterpret_cast<Gates*>(at);                               // [parity]
  static_assert(sizeof(Gates) * 2 == H::GATES, "gates");

  const int b = blockIdx.z, h = blockIdx.y, col0 = (int)blockIdx.x * COLS;
  const int n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int tid = threadIdx.x % GROUP, windows = (n + C - 1) / C;
  const int hk = h / p.group;
  const int64_t state = ((int64_t)slot * p.heads + h) * D * D + col0;

  // ------------------------------------------------------------------------------- preparation
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col0;
  const int64_t gate0 = (int64_t)b * p.tokens * p.heads + h;
  constexpr int EACH = 16 / (int)sizeof(T), ROW = D / EACH, VROW = COLS / EACH;      // elements of a copy, copies of a row
  auto fetch = [&](int w) {
    T* kd;
    int pitch;
    if constexpr (TERMS == 1) {
      kd = reinterpret_cast<T*>(kq) + (w % H::PLACES) * 2 * H::TILE;
      pitch = KP;
    } else {
      kd = reinterpret_cast<T*>(raw);
      pitch = D + 4;
    }
    for (int i = tid; i < 2 * C * ROW; i += GROUP) {
      const int side = i / (C * ROW), r = i / ROW % C, c = i % ROW * EACH;
      const bool there = w * C + r < n;
      const int64_t token = there ? w * C + r : 0;
      copy16(kd + (side * C + r) * pitch + c, side ? q + token * p.q.t + c : k + token * p.k.t + c, there);
    }
    for (int i = tid; i < C * VROW; i += GROUP) {
      const int r = i / VROW, c = i % VROW * EACH;
      const bool there = w * C + r < n;
      copy16(vs + ((w % H::STAGES) * C + r) * VP + c, v + (int64_t)(there ? w * C + r : 0) * p.v.t + c, there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float next_decay = 0.f, next_beta = 0.f;     // of the first warp's tokens of the window that is prepared next
  auto fetch_gates = [&](int w) {
    const int token = w * C + lane;
    next_decay = next_beta = 0.f;
    if (warp != 4 || token >= n) return;
    if (p.log_decay) next_decay = p.log_decay[gate0 + (int64_t)token * p.heads];
    next_beta = p.beta[gate0 + (int64_t)token * p.heads];
  };
  auto prepare = [&](int w) {
    const int parity = w & 1;
    Gates& gt = gates[parity];
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    bool odd = false;
    // its own copies
    for (int i = tid; i < C * ROW; i += GROUP) {
      const int r = i / ROW, c = i % ROW * EACH;
      const T* from = TERMS == 1 ? reinterpret_cast<const T*>(kq) + (w % H::PLACES) * 2 * H::TILE + r * KP + c : reinterpret_cast<const T*>(raw) + r * (D + 4) + c;
      odd |= !all_finite<T>(*reinterpret_cast<const uint4*>(from));
    }
    for (int i = tid; i < C * VROW; i += GROUP)
      odd |= !all_finite<T>(*reinterpret_cast<const uint4*>(vs + ((w % H::STAGES) * C + i / VROW) * VP + i % VROW * EACH));
    if (warp == 4) {
      // sums in 64 bits: what counts are differences of them, and a token may fade by any factor.  -infinity: all of it, like -10^5.
      odd |= !isfinite(next_beta) || !(next_decay < INFINITY);
      const double mine = next_decay < -1e5f ? -1e5 : (double)next_decay;
      double sum = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double other = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += other;
      }
      const double all = __shfl_sync(0xffffffffu, sum, 31);
      gt.beta[lane] = next_beta;
      gt.up[lane] = expf((float)sum);
      gt.down[lane] = expf((float)(all - sum));
      // differences are taken from this and, for what it lacks, `low`, which is the same for all of them: sums are counted from the window's middle
      gt.sum[lane] = (float)sum;
      reinterpret_cast<float*>(y)[lane] = (float)(sum - (double)(float)sum);
      if (lane == 0) gt.whole = expf((float)all);
    }
    odd = named_barrier_or(2, GROUP, odd);
    if (tid == 0) gt.odd = odd;
    __nv_bfloat16* ks = kq + (w % H::PLACES) * 2 * TERMS * H::TILE;
    __nv_bfloat16* qs = ks + TERMS * H::TILE;
    if constexpr (TERMS == 3) {
      for (int i = tid; i < 2 * C * (D / 2); i += GROUP) {
        const int side = i / (C * (D / 2)), r = i / (D / 2) % C, c = i % (D / 2) * 2;
        const float2 f = *reinterpret_cast<const float2*>(raw + (side * C + r) * (D + 4) + c);
        uint32_t terms[3];
        cut(f.x, f.y, terms);
#pragma unroll
        for (int x = 0; x < 3; ++x) *reinterpret_cast<uint32_t*>(ks + (side * 3 + x) * H::TILE + r * KP + c) = terms[x];
      }
      barrier(2);
    }
    if (w + 1 < windows) {
      fetch(w + 1);
      fetch_gates(w + 1);
    }
    // A and P: 16 rows to a warp, their columns up to the diagonal's
    const int job = warp - 4, strip = job < 2 ? 1 : 0, rows = 16 * strip;
    const bool keys = (job & 1) == 0;
    const __nv_bfloat16* left = keys ? ks : qs;
    float acc[4][4], rest[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) acc[i][x] = rest[i][x] = 0.f;
#pragma unroll
    for (int x = 0; x < KS; x += 2) {          // 32 elements
      uint32_t a[2][TERMS][4];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < TERMS; ++i) ldmatrix4<false>(a[e][i], smem_u32(left + i * H::TILE + (rows + (lane & 15)) * KP + (x + e) * 16 + (lane >> 4) * 8));
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (c < 2 * strip + 2) {
          uint32_t one[TERMS][2], two[TERMS][2];
#pragma unroll
          for (int i = 0; i < TERMS; ++i) {
            uint32_t f[4];
            ldmatrix4<false>(f, smem_u32(ks + i * H::TILE + (8 * c + (lane & 7)) * KP + x * 16 + (lane >> 3) * 8));
            one[i][0] = f[0]; one[i][1] = f[1]; two[i][0] = f[2]; two[i][1] = f[3];
          }
          product(acc[c], rest[c], a[0], one);
          product(acc[c], rest[c], a[1], two);
        }
    }
    float* A = tri + parity * C * TP;
    const float* low = y;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (c < 2 * strip + 2)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int i = rows + g + 8 * r, j = 8 * c + 2 * t;
          const float si = gt.sum[i], li = low[i];
          float f[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const bool there = keys ? j + x < i : j + x <= i;
            const float fade = expf((si - gt.sum[j + x]) + (li - low[j + x]));
            f[x] = there ? (keys ? gt.beta[i] : p.scale) * fade * (acc[c][2 * r + x] + rest[c][2 * r + x]) : 0.f;
          }
          if (keys) {
            *reinterpret_cast<float2*>(A + i * TP + j) = make_float2(f[0], f[1]);
          } else {
            uint32_t terms[3];
            cut(f[0], f[1], terms);
#pragma unroll
            for (int x = 0; x < SEEN; ++x) *reinterpret_cast<uint32_t*>(ps + (parity * SEEN + x) * C * PP + i * PP + j) = terms[x];
          }
        }
    barrier(2);
    // the inverses of both diagonal blocks, a column to a lane
    if (job < 2) {
      float* at = A + job * 16 * (TP + 1);
      const int j = lane & 15;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float sum = i == j ? 1.f : 0.f;
#pragma unroll
        for (int m = 0; m < i; ++m) sum = fmaf(-at[i * TP + m], x[m], sum);
        x[i] = sum;
      }
      __syncwarp();
      if (lane < 16)
#pragma unroll
        for (int i = 0; i < 16; ++i) at[i * TP + j] = x[i];
    }
    barrier(2);
    // the block below: -T_11 (A_10 T_00)
    const int r = tid / 8, c = tid % 8 * 2;
    {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int m = 0; m < 16; ++m) {
        const float a = A[(16 + r) * TP + m];
        const float2 x = *reinterpret_cast<const float2*>(A + m * TP + c);
        sum = make_float2(fmaf(a, x.x, sum.x), fmaf(a, x.y, sum.y));
      }
      *reinterpret_cast<float2*>(y + r * 20 + c) = sum;
    }
    barrier(2);
    {
      float2 sum = make_float2(0.f, 0.f);
#pragma unroll
      for (int m = 0; m < 16; ++m) {
        const float a = A[(16 + r) * TP + 16 + m];
        const float2 x = *reinterpret_cast<const float2*>(y + m * 20 + c);
        sum = make_float2(fmaf(-a, x.x, sum.x), fmaf(-a, x.y, sum.y));
      }
      *reinterpret_cast<float2*>(A + (16 + r) * TP + c) = sum;
    }
  };

  // ------------------------------------------------------------------------------- the chain
  // rows: value columns 16 s + g and + 8; columns: elements 2t and 2t + 1 of the warp's tiles of 8
  float s[NS][NT][4];
  auto keep_state = [&]() {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < NT; ++x) keep<3>(s_frag + i * 3 * KS * 128, KS * 128, lane, warp * NT + x, s[i][x]);
  };
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col0;
  auto advance = [&](int w) {
    const int parity = w & 1;
    const Gates& gt = gates[parity];
    const float* T_ = tri + parity * C * TP;
    const __nv_bfloat16* ks = kq + (w % H::PLACES) * 2 * TERMS * H::TILE;
    const __nv_bfloat16* qs = ks + TERMS * H::TILE;
    // this warp's tokens: 8 warp .. 8 warp + 7, products along tokens up to theirs
    const int steps = warp / 2 + 1;
    uint32_t tf[2][3][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 f = x < steps ? *reinterpret_cast<const float2*>(T_ + (8 * warp + g) * TP + 16 * x + 8 * e + 2 * t) : make_float2(0.f, 0.f);
        uint32_t terms[3];
        cut(f.x, f.y, terms);
#pragma unroll
        for (int i = 0; i < 3; ++i) tf[x][i][e] = terms[i];
      }
    }
    const int token = 8 * warp + 2 * t;
    const float2 beta = *reinterpret_cast<const float2*>(gt.beta + token), up = *reinterpret_cast<const float2*>(gt.up + token),
                 down = *reinterpret_cast<const float2*>(gt.down + token);
    // S^T K^T and S^T Q^T
    float x0[NS][4], x1[NS][4], o0[NS][4], o1[NS][4];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) x0[i][x] = x1[i][x] = o0[i][x] = o1[i][x] = 0.f;
#pragma unroll
    for (int x = 0; x < KS; x += 2) {
      uint32_t kf[2][TERMS][2], qf[2][TERMS][2];
#pragma unroll
      for (int i = 0; i < TERMS; ++i) {
        uint32_t f[4];
        const int at = i * H::TILE + (8 * warp + (lane & 7)) * KP + x * 16 + (lane >> 3) * 8;
        ldmatrix4<false>(f, smem_u32(ks + at));
        kf[0][i][0] = f[0]; kf[0][i][1] = f[1]; kf[1][i][0] = f[2]; kf[1][i][1] = f[3];
        ldmatrix4<false>(f, smem_u32(qs + at));
        qf[0][i][0] = f[0]; qf[0][i][1] = f[1]; qf[1][i][0] = f[2]; qf[1][i][1] = f[3];
      }
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t a[3][4];
#pragma unroll
          for (int c = 0; c < 3; ++c) load16(a[c], s_frag + ((i * 3 + c) * KS + x + e) * 128 + lane * 4);
          product(x0[i], x1[i], a, kf[e]);
          product(o0[i], o1[i], reinterpret_cast<const uint32_t(&)[SEEN][4]>(a), qf[e]);
        }
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const T* vv = vs + ((w % H::STAGES) * C + token) * VP + 16 * i + g;
      float r[4];
      r[0] = beta.x * fmaf(-up.x, x0[i][0] + x1[i][0], to_float(vv[0]));
      r[1] = beta.y * fmaf(-up.y, x0[i][1] + x1[i][1], to_float(vv[VP]));
      r[2] = beta.x * fmaf(-up.x, x0[i][2] + x1[i][2], to_float(vv[8]));
      r[3] = beta.y * fmaf(-up.y, x0[i][3] + x1[i][3], to_float(vv[VP + 8]));
      keep<3>(r_frag + i * 3 * (C / 16) * 128, (C / 16) * 128, lane, warp, r);
#pragma unroll
      for (int x = 0; x < 4; ++x) o0[i][x] = (o0[i][x] + o1[i][x]) * (p.scale * (x & 1 ? up.y : up.x));
    }
    barrier(1);
    // U^T = R^T T^T
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      float u0[4] = {}, u1[4] = {};
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x < steps) {
          uint32_t a[3][4];
#pragma unroll
          for (int c = 0; c < 3; ++c) load16(a[c], r_frag + ((i * 3 + c) * (C / 16) + x) * 128 + lane * 4);
          product(u0, u1, a, tf[x]);
        }
#pragma unroll
      for (int x = 0; x < 4; ++x) u0[x] += u1[x];
      uint32_t* to = u_frag + i * (3 + SEEN) * (C / 16) * 128;
      keep<SEEN>(to + 3 * (C / 16) * 128, (C / 16) * 128, lane, warp, u0);
      u0[0] *= down.x; u0[1] *= down.y; u0[2] *= down.x; u0[3] *= down.y;
      keep<3>(to, (C / 16) * 128, lane, warp, u0);
    }
    barrier(1);
    // S'^T = e^G_C S^T + U'^T K
    uint32_t pf[2][SEEN][2];
#pragma unroll
    for (int i = 0; i < SEEN; ++i) {
      uint32_t f[4];
      ldmatrix4<false>(f, smem_u32(ps + (parity * SEEN + i) * C * PP + (8 * warp + (lane & 7)) * PP + (lane >> 3) * 8));
      pf[0][i][0] = f[0]; pf[0][i][1] = f[1]; pf[1][i][0] = f[2]; pf[1][i][1] = f[3];
    }
    const float whole = gt.whole;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      uint32_t a[2][3][4];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int c = 0; c < 3; ++c) load16(a[x][c], u_frag + ((i * (3 + SEEN) + c) * (C / 16) + x) * 128 + lane * 4);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        float d0[4] = {}, d1[4] = {};
        uint32_t one[TERMS][2], two[TERMS][2];
#pragma unroll
        for (int c = 0; c < TERMS; ++c) {
          uint32_t f[4];
          ldmatrix4<true>(f, smem_u32(ks + c * H::TILE + lane * KP + (warp * NT + m) * 8));
          one[c][0] = f[0]; one[c][1] = f[1]; two[c][0] = f[2]; two[c][1] = f[3];
        }
        product(d0, d1, a[0], one);
        product(d0, d1, a[1], two);
#pragma unroll
        for (int x = 0; x < 4; ++x) s[i][m][x] = fmaf(whole, s[i][m][x], d0[x] + d1[x]);
      }
    }
    keep_state();
    // out: behind the state, which the others wait for
#pragma unroll
    for (int i = 0; i < NS; ++i) {
#pragma unroll
      for (int x = 0; x < 4; ++x) o1[i][x] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (x < steps) {
          uint32_t a[SEEN][4];
#pragma unroll
          for (int c = 0; c < SEEN; ++c) load16(a[c], u_frag + ((i * (3 + SEEN) + 3 + c) * (C / 16) + x) * 128 + lane * 4);
          product(o0[i], o1[i], a, pf[x]);
        }
      T* to = outs + token * VP + 16 * i + g;
      to[0] = (T)(o0[i][0] + o1[i][0]);
      to[VP] = (T)(o0[i][1] + o1[i][1]);
      to[8] = (T)(o0[i][2] + o1[i][2]);
      to[VP + 8] = (T)(o0[i][3] + o1[i][3]);
    }
    __syncwarp();
    for (int i = lane; i < 8 * VROW; i += 32) {
      const int r = 8 * warp + i / VROW, c = i % VROW * EACH;
      if (w * C + r < n) *reinterpret_cast<uint4*>(o + (int64_t)(w * C + r) * p.o.t + c) = *reinterpret_cast<const uint4*>(outs + r * VP + c);
    }
    __syncwarp();
  };
  // A window with something in it that is not finite, token by token, a value column to a thread: the weights of 0 that a window's products give earlier tokens would
  // make NaN of it.
  auto advance_slowly = [&](int w) {
    float* st = reinterpret_cast<float*>(s_frag);      // [COLS][D + 1]
    static_assert(COLS * (D + 1) * 4 <= H::S + H::R, "the state takes its operands' place");
    auto each = [&](auto f) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int x = 0; x < NT; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) f(s[i][x][e], st[(16 * i + g + 8 * (e >> 1)) * (D + 1) + (warp * NT + x) * 8 + 2 * t + (e & 1)]);
    };
    each([](float& mine, float& there) { there = mine; });
    barrier(1);
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
    barrier(1);
    each([](float& mine, float& there) { mine = there; });
    barrier(1);                        // the state's operands take the place back
    keep_state();
  };

  if (warp < 4) {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][x][e] = p.state[state + (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + 16 * i + g + 8 * (e >> 1)];
    keep_state();
  } else if (windows > 0) {
    fetch_gates(0);
    fetch(0);
    prepare(0);
  }
  __syncthreads();
  for (int w = 0; w < windows; ++w) {
    if (warp >= 4) {
      if (w + 1 < windows) prepare(w + 1);
    } else if (gates[w & 1].odd) {
      advance_slowly(w);
    } else {
      advance(w);
    }
    __syncthreads();                   // the next window is prepared, this one's places are free
  }
  if (warp < 4 && (windows > 0 || p.state_out != p.state))
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) p.state_out[state + (int64_t)((warp * NT + x) * 8 + 2 * t + (e & 1)) * D + 16 * i + g + 8 * (e >> 1)] = s[i][x][e];
}

template <typename T, int D, int NS>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  using H = Shape<T, D, NS>;
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(delta_chunk_kernel<T, D, NS>, cudaFuncAttributeMaxDynamicSharedMemorySize, H::SMEM); });
  if (e != cudaSuccess) return e;
  delta_chunk_kernel<T, D, NS><<<dim3(D / H::COLS, (unsigned)p.heads, (unsigned)p.batch), THREADS, H::SMEM, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  return (int64_t)p.batch * p.heads * (D / 16) < 4 * PLAN_SMS ? launch<T, D, 1>(p, s) : launch<T, D, 2>(p, s);
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

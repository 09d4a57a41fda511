// The gated delta rule, token by token (tt_delta_rule).  With S a head's state [key][value], a = exp(log_decay):
//   F = a S,  u = beta (v - F^T k),  S' = F + k u^T,  out = scale S'^T q = scale (F^T q + (k . q) u).
// The second form of out lets one pass over the state give both sums, F^T k and F^T q, so that a single meeting of the block's threads lies
// between reading a state and writing it.  A block owns a run of W value columns of one head's state (the columns are
// independent of each other), LANES = W / 4 threads to a row, in registers for the whole call: a token by itself reads and writes each state once, and that bounds
// many states (256 sessions of 8 heads of 128, 268 MB: 47 us, 88 % of the rate of a copy; 48 call by call).  Few states are bound by the launch (2.2 us); a further token takes 0.8 us.
#include "linear_common.cuh"

namespace tt {
namespace tok {
namespace {

template <int D, int W>
struct DeltaStep {
  static constexpr int LANES = W / 4;                                   // threads to a row
  static constexpr int THREADS = LANES * D < 256 ? LANES * D : 256;
  static constexpr int ROWS = D * LANES / THREADS;                      // rows to a thread
};

// SEVERAL: the next token's operands are fetched while this one is worked on.  (Bounds on registers: without them the path of products that overflow costs 24 fp32 tokens of 256 x 8 heads
// of 128 100 us of the 397 that they take.)
template <typename T, int D, int W, bool SEVERAL>
__global__ void __launch_bounds__(256, !SEVERAL ? 0 : D == 128 ? 2 : 3) delta_step_kernel(const __grid_constant__ DeltaParams p) {
  using Shape = DeltaStep<D, W>;
  constexpr int LANES = Shape::LANES, ROWS = Shape::ROWS, STEP = Shape::THREADS / LANES, WARPS = Shape::THREADS / 32;
  // of either parity of tokens: a warp may be at the next one while another still reads these
  __shared__ float4 said[2][WARPS][LANES], asked[2][WARPS][LANES];
  __shared__ float dots[2][WARPS];
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x % LANES, col = (int)blockIdx.x * W + lane * 4, row = threadIdx.x / LANES, warp = threadIdx.x / 32;
  const int n = clamp_length(p.lengths, b, p.tokens);
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int64_t base = ((int64_t)slot * p.heads + h) * D * D + (int64_t)row * D + col;
  float4 s[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) s[i] = *reinterpret_cast<const float4*>(p.state + base + (int64_t)i * STEP * D);
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h + row;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h + row;
  const T* v = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + h * p.v.h + col;
  T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col;
  const int64_t gates = (int64_t)b * p.tokens * p.heads + h;
  struct Token {
    T k[ROWS], q[ROWS], v[4];
    float decay = 0.f, beta;
  };
  auto fetch = [&](Token& to, int t) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      to.k[i] = k[t * p.k.t + i * STEP];
      to.q[i] = q[t * p.q.t + i * STEP];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) to.v[j] = v[t * p.v.t + j];
    if (p.log_decay) to.decay = p.log_decay[gates + (int64_t)t * p.heads];
    to.beta = p.beta[gates + (int64_t)t * p.heads];
  };
  Token next;
  if (n > 0) fetch(next, 0);
  for (int t = 0; t < (SEVERAL ? n : min(n, 1)); ++t) {
    float kk[ROWS], qq[ROWS], vv[4];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) { kk[i] = to_float(next.k[i]); qq[i] = to_float(next.q[i]); }
#pragma unroll
    for (int j = 0; j < 4; ++j) vv[j] = to_float(next.v[j]);
    const float fade = expf(next.decay), beta = next.beta;
    if (SEVERAL && t + 1 < n) fetch(next, t + 1);
    float x[4] = {}, y[4] = {}, kq = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      kq = fmaf(kk[i], qq[i], kq);
      // before the sums: those of a state that the decay takes back may pass what 32 bits hold
      s[i].x *= fade; s[i].y *= fade; s[i].z *= fade; s[i].w *= fade;
      x[0] = fmaf(kk[i], s[i].x, x[0]); x[1] = fmaf(kk[i], s[i].y, x[1]); x[2] = fmaf(kk[i], s[i].z, x[2]); x[3] = fmaf(kk[i], s[i].w, x[3]);
      y[0] = fmaf(qq[i], s[i].x, y[0]); y[1] = fmaf(qq[i], s[i].y, y[1]); y[2] = fmaf(qq[i], s[i].z, y[2]); y[3] = fmaf(qq[i], s[i].w, y[3]);
    }
#pragma unroll
    for (int d = 16; d >= LANES; d >>= 1) {
      kq += __shfl_xor_sync(0xFFFFFFFFu, kq, d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] += __shfl_xor_sync(0xFFFFFFFFu, x[j], d);
        y[j] += __shfl_xor_sync(0xFFFFFFFFu, y[j], d);
      }
    }
    if (threadIdx.x % 32 < LANES) {
      said[t & 1][warp][lane] = make_float4(x[0], x[1], x[2], x[3]);
      asked[t & 1][warp][lane] = make_float4(y[0], y[1], y[2], y[3]);
    }
    if (threadIdx.x % 32 == 0) dots[t & 1][warp] = kq;
    __syncthreads();
    float4 sx = said[t & 1][0][lane];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) {
      const float4 f = said[t & 1][w][lane];
      sx.x += f.x; sx.y += f.y; sx.z += f.z; sx.w += f.w;
    }
    const float u[4] = {beta * (vv[0] - sx.x), beta * (vv[1] - sx.y), beta * (vv[2] - sx.z), beta * (vv[3] - sx.w)};
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      s[i].x = fmaf(kk[i], u[0], s[i].x);
      s[i].y = fmaf(kk[i], u[1], s[i].y);
      s[i].z = fmaf(kk[i], u[2], s[i].z);
      s[i].w = fmaf(kk[i], u[3], s[i].w);
    }
    if (threadIdx.x < LANES) {
      float4 sy = asked[t & 1][0][lane];
      float dot = dots[t & 1][0];
#pragma unroll
      for (int w = 1; w < WARPS; ++w) {
        const float4 f = asked[t & 1][w][lane];
        sy.x += f.x; sy.y += f.y; sy.z += f.z; sy.w += f.w;
        dot += dots[t & 1][w];
      }
      float sum[4] = {fmaf(dot, u[0], sy.x), fmaf(dot, u[1], sy.y), fmaf(dot, u[2], sy.z), fmaf(dot, u[3], sy.w)};
      if (__builtin_expect(!isfinite(dot), 0)) {
        // k . q passes what 32 bits hold, or an element is not finite: q (k u) then, as the state has it
        sum[0] = sy.x; sum[1] = sy.y; sum[2] = sy.z; sum[3] = sy.w;
#pragma unroll 1
        for (int i = 0; i < D; ++i) {
          const float ki = to_float(k[t * p.k.t - row + i]), qi = to_float(q[t * p.q.t - row + i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) sum[j] = fmaf(qi, ki * u[j], sum[j]);
        }
      }
      T* to = o + t * p.o.t;
#pragma unroll
      for (int j = 0; j < 4; ++j) to[j] = (T)(p.scale * sum[j]);
    }
  }
  if (n == 0 && p.state_out == p.state) return;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) *reinterpret_cast<float4*>(p.state_out + base + (int64_t)i * STEP * D) = s[i];
}

template <typename T, int D, int W, bool SEVERAL>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  delta_step_kernel<T, D, W, SEVERAL><<<dim3(D / W, (unsigned)p.heads, (unsigned)p.batch), DeltaStep<D, W>::THREADS, 0, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  // Columns to a block: the fewer, the more multiprocessors fetch a state and the more threads share a row's sums, which is what a token takes.  Whole, halves and quarters, us:
  // 256 sessions of 8 heads of 128, a token 60.1 46.6 53.0, six tokens 125 126 185; of 64 16.8 20.8 33.5, 46 77 135; of 32 9.7 9.6 10.4, 33 30 31;
  // five sessions, six tokens of heads of 128 11.7 7.6 6.3, of 64 6.3 6.3 5.6.
  const auto run = [&](auto several) {
    constexpr bool S = decltype(several)::value;
    if constexpr (D == 64)
      if ((int64_t)p.batch * p.heads >= PLAN_SMS) return launch<T, D, 64, S>(p, s);
    return launch<T, D, D / 2, S>(p, s);
  };
  return p.tokens > 1 ? run(std::true_type()) : run(std::false_type());
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

cudaError_t launch_delta_step(const DeltaParams& p, bool bf16, int D, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
}

}  // namespace tok
}  // namespace tt

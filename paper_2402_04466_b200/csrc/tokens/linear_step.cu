// Linear attention, a single token per entry (tt_linear_attention with tokens == 1):
//   S' = exp(log_decay) S + k v^T,  out = scale * q S'.
// Bound by memory: the fp32 state is read and written once and everything else is small beside it.  A block owns a run of W value columns of
// one head's state (the columns are independent of each other), LANES = W / 4 threads to a row, all of its loads in flight
// together (256 streams of 8 heads of 128: 45.4 us, 6.0 TB/s, 91 % of a plain copy's rate; five of 2 heads of 64: 2.9 us, a launch).  The sum over the rows goes through shuffles and then shared memory, always in the same order.
#include "linear_common.cuh"

namespace tt {
namespace tok {
namespace {

template <int D, int W>
struct StepShape {
  static constexpr int LANES = W / 4;                                   // threads to a row
  static constexpr int THREADS = LANES * D < 256 ? LANES * D : 256;
  static constexpr int ROWS = D * LANES / THREADS;                      // rows to a thread
};

template <typename T, int D, int W>
__global__ void __launch_bounds__(256) linear_step_kernel(const __grid_constant__ LinearParams p) {
  using Shape = StepShape<D, W>;
  constexpr int LANES = Shape::LANES, ROWS = Shape::ROWS, STEP = Shape::THREADS / LANES, WARPS = Shape::THREADS / 32;
  __shared__ float4 sums[WARPS][LANES];
  const int b = blockIdx.z, h = blockIdx.y, col = (int)blockIdx.x * W + (int)(threadIdx.x % LANES) * 4, row = threadIdx.x / LANES;
  const bool has = clamp_length(p.lengths, b, 1) == 1;
  // before any of its data is touched: the slot of an entry that is passed over may be one that an earlier entry is writing
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;                // the whole block
  const int64_t base = ((int64_t)slot * p.heads + h) * D * D + (int64_t)row * D + col;
  float4 s[ROWS];
  float kk[ROWS], qq[ROWS], v[4];
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + h * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const T* vv = reinterpret_cast<const T*>(p.v.p) + b * p.v.b + hk * p.v.h;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) s[i] = *reinterpret_cast<const float4*>(p.state + base + (int64_t)i * STEP * D);
  if (has) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      kk[i] = to_float(k[row + i * STEP]);
      qq[i] = to_float(q[row + i * STEP]) * p.scale;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = to_float(vv[col + j]);
  }
  float* out_state = p.state_out + base;
  if (!has) {
    if (p.state_out != p.state)
#pragma unroll
      for (int i = 0; i < ROWS; ++i) *reinterpret_cast<float4*>(out_state + (int64_t)i * STEP * D) = s[i];
    return;
  }
  const float decay = decay_power(p.log_decay[h], 1);
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    s[i].x = fmaf(decay, s[i].x, kk[i] * v[0]);
    s[i].y = fmaf(decay, s[i].y, kk[i] * v[1]);
    s[i].z = fmaf(decay, s[i].z, kk[i] * v[2]);
    s[i].w = fmaf(decay, s[i].w, kk[i] * v[3]);
    *reinterpret_cast<float4*>(out_state + (int64_t)i * STEP * D) = s[i];
    sum.x = fmaf(qq[i], s[i].x, sum.x);
    sum.y = fmaf(qq[i], s[i].y, sum.y);
    sum.z = fmaf(qq[i], s[i].z, sum.z);
    sum.w = fmaf(qq[i], s[i].w, sum.w);
  }
#pragma unroll
  for (int o = 16; o >= LANES; o >>= 1) {
    sum.x += __shfl_xor_sync(0xFFFFFFFFu, sum.x, o);
    sum.y += __shfl_xor_sync(0xFFFFFFFFu, sum.y, o);
    sum.z += __shfl_xor_sync(0xFFFFFFFFu, sum.z, o);
    sum.w += __shfl_xor_sync(0xFFFFFFFFu, sum.w, o);
  }
  if (threadIdx.x % 32 < LANES) sums[threadIdx.x / 32][threadIdx.x % 32] = sum;
  __syncthreads();
  if (threadIdx.x < LANES) {
    float4 t = sums[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) {
      const float4 u = sums[w][threadIdx.x];
      t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
    }
    T* o = reinterpret_cast<T*>(p.o.p) + b * p.o.b + h * p.o.h + col;
    o[0] = (T)t.x; o[1] = (T)t.y; o[2] = (T)t.z; o[3] = (T)t.w;
  }
}

template <typename T, int D, int W>
cudaError_t launch(const LinearParams& p, cudaStream_t s) {
  linear_step_kernel<T, D, W><<<dim3(D / W, (unsigned)p.heads, (unsigned)p.batch), StepShape<D, W>::THREADS, 0, s>>>(p);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch(const LinearParams& p, cudaStream_t s) {
  // few states: cut each into four runs of columns, so that more multiprocessors fetch
  return (int64_t)p.batch * p.heads < 2 * PLAN_SMS ? launch<T, D, D / 4>(p, s) : launch<T, D, D>(p, s);
}
template <typename T>
cudaError_t launch(const LinearParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

cudaError_t launch_linear_step(const LinearParams& p, bool bf16, int D, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
}

}  // namespace tok
}  // namespace tt

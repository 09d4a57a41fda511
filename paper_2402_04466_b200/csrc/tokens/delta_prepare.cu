// The gated delta rule over several tokens, first part (tt_delta_rule): of every window of 32 tokens and head, what depends on no state.
// A block takes a window as delta_window.cuh says.  The windows of all sequences run at once; the chain of states, delta_chunk.cu, reads what is left here as the registers
// it needs.  150 windows of 32 heads of 64, a third of eight maps: 26.6 us, bound by the substitutions' and products' latencies at five blocks to a multiprocessor.
#include "delta_window.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int C = DELTA_C;

template <typename T, int D>
__global__ void __launch_bounds__(DELTA_GROUP, sizeof(T) == 2 ? 5 : 3) delta_prepare_kernel(const __grid_constant__ DeltaParams p) {
  using W = DeltaWindow<T, D>;
  constexpr int TERMS = W::TERMS, SEEN = W::SEEN, KP = W::KP;
  extern __shared__ __align__(16) uint8_t smem[];
  __nv_bfloat16* ks = reinterpret_cast<__nv_bfloat16*>(smem);                // [keys, queries][term][C][KP]
  __nv_bfloat16* qs = ks + TERMS * W::TILE;
  typename W::Room& room = *reinterpret_cast<typename W::Room*>(qs + TERMS * W::TILE);
  pdl_launch_dependents();
  const int b = blockIdx.z, h = blockIdx.y, w = p.first_window + blockIdx.x;
  const int n = clamp_length(p.lengths, b, p.tokens);
  // Behind the chain of the range before, which it runs beside, it ends behind that, so that what waits for the one has waited for the other: one block sees to it.
  const bool holds = p.first_window > 0 && (blockIdx.x | blockIdx.y | blockIdx.z) == 0;
  if (w * C >= n || slot_of(p.slots, p.num_slots, b) < 0) {
    if (holds) pdl_wait();
    return;                                                                  // the whole block
  }
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, tid = threadIdx.x;
  const int hk = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q.p) + b * p.q.b + hk * p.q.h;
  const T* k = reinterpret_cast<const T*>(p.k.p) + b * p.k.b + hk * p.k.h;
  DeltaRecord<SEEN>& record = reinterpret_cast<DeltaRecord<SEEN>*>(p.records)[((int64_t)b * p.heads + h) * p.windows + blockIdx.x];
  float decay = 0.f, beta = 0.f;
  if (warp == 0) {
    const int token = w * C + lane;
    const int64_t gate = ((int64_t)b * p.tokens + token) * p.heads + h;
    if (token < n) {
      if (p.log_decay) decay = p.log_decay[gate];
      beta = p.beta[gate];
    }
  }
  const Rows<T, D> k_rows(k, p.k.t, tid), q_rows(q, p.q.t, tid);
  if constexpr (TERMS == 1) {
    k_rows.fetch(reinterpret_cast<T*>(ks), KP, w * C, n);
    q_rows.fetch(reinterpret_cast<T*>(qs), KP, w * C, n);
    copies_commit();
  } else {
    for (int i = tid; i < 2 * C * (D / 4); i += DELTA_GROUP) {
      const int side = i / (C * (D / 4)), r = i / (D / 4) % C, c = i % (D / 4) * 4;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (w * C + r < n) f = *reinterpret_cast<const float4*>((side ? q + (int64_t)(w * C + r) * p.q.t : k + (int64_t)(w * C + r) * p.k.t) + c);
      uint32_t low[3], high[3];
      cut(f.x, f.y, low);
      cut(f.z, f.w, high);
#pragma unroll
      for (int x = 0; x < 3; ++x) *reinterpret_cast<uint2*>(ks + (side * 3 + x) * W::TILE + r * KP + c) = make_uint2(low[x], high[x]);
    }
  }
  const auto ready = [] {
    if constexpr (TERMS == 1) copies_wait<0>();
    __syncthreads();
  };
  W::prepare(record, room, ks, qs, decay, beta, p.scale, warp, lane, ready, [] { __syncthreads(); });
  if (holds) pdl_wait();
}

template <typename T, int D>
cudaError_t launch(const DeltaParams& p, cudaStream_t s) {
  using W = DeltaWindow<T, D>;
  constexpr int SMEM = 2 * W::TERMS * W::TILE * 2 + (int)sizeof(typename W::Room);
  static OncePerContext once;
  const cudaError_t e = once([] { return cudaFuncSetAttribute(delta_prepare_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); });
  if (e != cudaSuccess) return e;
  return launch_kernel(delta_prepare_kernel<T, D>, dim3((unsigned)p.windows, (unsigned)p.heads, (unsigned)p.batch), DELTA_GROUP, SMEM, s, p, p.first_window > 0);
}
template <typename T>
cudaError_t launch(const DeltaParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<T, 32>(p, s) : D == 64 ? launch<T, 64>(p, s) : launch<T, 128>(p, s);
}

}  // namespace

cudaError_t launch_delta_prepare(const DeltaParams& p, bool bf16, int D, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(p, D, s) : launch<float>(p, D, s);
}

}  // namespace tok
}  // namespace tt

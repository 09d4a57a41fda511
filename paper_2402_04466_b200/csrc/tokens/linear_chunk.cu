// Linear attention over several fp32 tokens (tt_linear_attention): chunks of C tokens, on the fp32 units.
//
// With the state S before a chunk, l the head's decay, tokens i, j of the chunk counted from 0 and m their number:
//   out_i = scale * ( l^(i+1) q_i S + sum_{j <= i} l^(i-j) (q_i k_j) v_j ),     S' = l^m S + sum_j l^(m-1-j) k_j v_j^T.
// Every exponent is 0 or more, so nothing overflows however strong the decay.
//
// A sequence (entry and head) is sequential over its chunks.  Where there are too few sequences to fill the device the tokens are cut into
// segments: linear_segment_kernel forms what each segment adds to the state, linear_scan_kernel turns that into the state
// before each segment, and linear_chunk_kernel then runs all segments at once.  K and V are read twice then.
//
// Bound by the fp32 units and what feeds them from shared memory, with eight warps to a multiprocessor.  Two sequences of 4801 tokens, 2 heads of 64 over
// one of keys and values: 43 us, a third of it the segments' sums; a block has a chain of three chunks.
#include "linear_common.cuh"
#include "token_ptx.cuh"

namespace tt {
namespace tok {
namespace {

constexpr int THREADS = 256;           // 16 x 16

template <int D>
struct ChunkShape {
  static constexpr int C = D == 128 ? 32 : 64;          // tokens of a chunk
  static constexpr int A = C / 16;                      // rows of the chunk to a thread
  static constexpr int E = D / 16;                      // rows of the state, and columns, to a thread
  static constexpr int QP = D + 4;                      // pitch of rows that 16 threads read side by side
  static constexpr int PP = C + 4;
  static constexpr size_t smem = sizeof(float) * (2 * C * QP + C * D + D * D + C * PP + C + 1);
};

// columns of a thread: four neighbours at 4 tx (and 64 + 4 tx), two at 2 tx where D is 32
template <int D>
__device__ __forceinline__ int column(int tx, int j) { return D == 32 ? 2 * tx + j : 4 * tx + (j & 3) + (j >> 2) * 64; }

template <int D>
__device__ __forceinline__ void load_columns(const float* row, int tx, float (&f)[D / 16]) {
  if constexpr (D == 32) {
    const float2 v = *reinterpret_cast<const float2*>(row + 2 * tx);
    f[0] = v.x; f[1] = v.y;
  } else {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const float4 v = *reinterpret_cast<const float4*>(row + 4 * tx + 64 * j);
      f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
    }
  }
}

// o += x y for rows ty + 16 a of x and this thread's columns of y; `n` inner steps, four at a time: a row's factors in one load
template <int D, int A>
__device__ __forceinline__ void multiply(Two (&o)[A][D / 32], const float* x, int pitch, const float* y, int n, int ty, int tx) {
#pragma unroll 2
  for (int e = 0; e < n; e += 4) {
    float4 f[A];
#pragma unroll
    for (int a = 0; a < A; ++a) f[a] = *reinterpret_cast<const float4*>(x + (ty + 16 * a) * pitch + e);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      Two g[D / 32];
      load_pairs<D>(y + (e + k) * D, tx, g);
#pragma unroll
      for (int a = 0; a < A; ++a) {
        const float w = k == 0 ? f[a].x : k == 1 ? f[a].y : k == 2 ? f[a].z : f[a].w;
        const Two w2 = pack2(w, w);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[a][c] = fma2_of(w2, g[c], o[a][c]);
      }
    }
  }
}

// a thread's columns of a row's out once more, terms of later tokens left out
template <int D>
__device__ __noinline__ void own_sums(float* out, const float* q, const float* S, const float* P, const float* v, int i, float decay, float scale, int tx) {
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    const int at = column<D>(tx, c);
    float sum = 0.f;
    for (int e = 0; e < D; ++e) sum = fmaf(q[e], S[e * D + at], sum);
    sum *= decay;
    for (int j = 0; j <= i; ++j) sum = fmaf(P[j], v[j * D + at], sum);
    out[at] = sum * scale;
  }
}

// Rows of D elements on their way into shared memory, zeros behind the m-th.  All loads come before the first store, which might, for all the
// compiler knows, change what a later load finds: one latency for a tile, not one for each of a thread's loads.
template <int D, int ROWS>
struct Tile {
  static constexpr int N = ROWS * (D / 4) / THREADS;
  static_assert(ROWS * (D / 4) % THREADS == 0, "whole rounds");
  float4 f[N];
  __device__ __forceinline__ void load(const float* src, int64_t stride, int m) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = threadIdx.x + n * THREADS, r = i / (D / 4);
      f[n] = r < m ? *reinterpret_cast<const float4*>(src + r * stride + i % (D / 4) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ void store(float* dst, int pitch) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = threadIdx.x + n * THREADS;
      *reinterpret_cast<float4*>(dst + i / (D / 4) * pitch + i % (D / 4) * 4) = f[n];
    }
  }
};

template <int D, bool WITH_OUT>
__device__ __forceinline__ void run_chunks(const LinearParams& p, int b, int h, int t0, int t1, float* S, float* smem) {
  using Shape = ChunkShape<D>;
  constexpr int C = Shape::C, A = Shape::A, E = Shape::E, QP = Shape::QP, PP = Shape::PP;
  float* q = smem;
  float* k = q + C * QP;
  float* v = k + C * QP;
  float* P = v + C * D + D * D;        // S lies between
  float* pw = P + C * PP;              // decay^0 .. decay^C
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16, hk = h / p.group;
  const float* gq = reinterpret_cast<const float*>(p.q.p) + b * p.q.b + h * p.q.h;
  const float* gk = reinterpret_cast<const float*>(p.k.p) + b * p.k.b + hk * p.k.h;
  const float* gv = reinterpret_cast<const float*>(p.v.p) + b * p.v.b + hk * p.v.h;
  float* go = reinterpret_cast<float*>(p.o.p) + b * p.o.b + h * p.o.h;
  if (threadIdx.x <= C) pw[threadIdx.x] = decay_power(p.log_decay[h], threadIdx.x);
  for (int t = t0; t < t1; t += C) {
    const int m = min(C, t1 - t);
    Tile<D, C> tq, tk, tv;
    if (WITH_OUT) tq.load(gq + t * p.q.t, p.q.t, m);
    tk.load(gk + t * p.k.t, p.k.t, m);
    tv.load(gv + t * p.v.t, p.v.t, m);
    __syncthreads();                   // the state, and the last chunk's reads
    if (WITH_OUT) tq.store(q, QP);
    tk.store(k, QP);
    tv.store(v, D);
    __syncthreads();
    if (WITH_OUT) {
      Two acc[A][A];                   // even and odd elements
#pragma unroll
      for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < A; ++c) acc[a][c] = pack2(0.f, 0.f);
#pragma unroll 4
      for (int e = 0; e < D; e += 4) {
        ulonglong2 x[A], y[A];
#pragma unroll
        for (int a = 0; a < A; ++a) {
          x[a] = *reinterpret_cast<const ulonglong2*>(q + (ty + 16 * a) * QP + e);
          y[a] = *reinterpret_cast<const ulonglong2*>(k + (tx + 16 * a) * QP + e);
        }
#pragma unroll
        for (int a = 0; a < A; ++a)
#pragma unroll
          for (int c = 0; c < A; ++c) acc[a][c] = fma2_of(x[a].y, y[c].y, fma2_of(x[a].x, y[c].x, acc[a][c]));
      }
#pragma unroll
      for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < A; ++c) {
          const int i = ty + 16 * a, j = tx + 16 * c;
          float lo, hi;
          unpack2(acc[a][c], lo, hi);
          P[i * PP + j] = i >= j ? (lo + hi) * pw[i - j] : 0.f;
        }
      Two o[A][E / 2];                 // pairs of neighbouring columns
#pragma unroll
      for (int a = 0; a < A; ++a)
#pragma unroll
        for (int c = 0; c < E / 2; ++c) o[a][c] = pack2(0.f, 0.f);
      multiply<D, A>(o, q, QP, S, D, ty, tx);
#pragma unroll
      for (int a = 0; a < A; ++a) {
        const float f = pw[ty + 16 * a + 1];
        const Two f2 = pack2(f, f);
#pragma unroll
        for (int c = 0; c < E / 2; ++c) o[a][c] = mul2_of(o[a][c], f2);
      }
      __syncthreads();                 // P
      multiply<D, A>(o, P, PP, v, (m + 3) & ~3, ty, tx);
#pragma unroll
      for (int a = 0; a < A; ++a) {
        const int i = ty + 16 * a;
        if (i < m) {
          float* dst = go + (int64_t)(t + i) * p.o.t;
          const Two s2 = pack2(p.scale, p.scale);
#pragma unroll
          for (int c = 0; c < E / 2; ++c) *reinterpret_cast<Two*>(dst + column<D>(tx, 2 * c)) = mul2_of(o[a][c], s2);
          // the weights of 0 behind a token make NaN of what is not finite in a later token's values: sums of its own and earlier tokens only
          Two bad = pack2(0.f, 0.f);
#pragma unroll
          for (int c = 0; c < E / 2; ++c) bad = fma2_of(o[a][c], pack2(0.f, 0.f), bad);
          float b0, b1;
          unpack2(bad, b0, b1);
          if (__builtin_expect(b0 + b1 != 0.f, 0)) own_sums<D>(dst, q + i * QP, S, P + i * PP, v, i, pw[i + 1], p.scale, tx);
        }
      }
    }
    // own rows and columns of the state: read by the block above, written here behind a barrier
    Two s[E][E / 2];
#pragma unroll
    for (int a = 0; a < E; ++a)
#pragma unroll
      for (int c = 0; c < E / 2; ++c) s[a][c] = pack2(0.f, 0.f);
#pragma unroll 2
    for (int j = 0; j < m; ++j) {
      float x[E];
      Two y[E / 2];
      load_columns<D>(k + j * QP, ty, x);
      load_pairs<D>(v + j * D, tx, y);
      const float d = pw[m - 1 - j];
#pragma unroll
      for (int a = 0; a < E; ++a) {
        const Two x2 = pack2(x[a] * d, x[a] * d);
#pragma unroll
        for (int c = 0; c < E / 2; ++c) s[a][c] = fma2_of(x2, y[c], s[a][c]);
      }
    }
    __syncthreads();
    const Two d2 = pack2(pw[m], pw[m]);
#pragma unroll
    for (int a = 0; a < E; ++a)
#pragma unroll
      for (int c = 0; c < E / 2; ++c) {
        Two* at = reinterpret_cast<Two*>(S + column<D>(ty, a) * D + column<D>(tx, 2 * c));
        *at = fma2_of(d2, *at, s[a][c]);
      }
  }
  __syncthreads();
}

template <int D>
__device__ __forceinline__ float* state_in_shared(float* smem) { return smem + ChunkShape<D>::C * (2 * ChunkShape<D>::QP + D); }

// What segment s of a sequence leaves behind when it starts from nothing.
template <int D>
__global__ void __launch_bounds__(THREADS) linear_segment_kernel(const __grid_constant__ LinearParams p) {
  extern __shared__ float4 raw[];
  float* smem = reinterpret_cast<float*>(raw);
  float* S = state_in_shared<D>(smem);
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x;
  pdl_launch_dependents();
  if (slot_of(p.slots, p.num_slots, b) < 0) return;
  const int n = clamp_length(p.lengths, b, p.tokens), t0 = seg * p.seg_tokens;
  if (t0 + p.seg_tokens >= n) return;      // the last one's is not needed
  for (int i = threadIdx.x; i < D * D; i += THREADS) S[i] = 0.f;
  run_chunks<D, false>(p, b, h, t0, t0 + p.seg_tokens, S, smem);
  float* dst = p.seg_state + (((int64_t)b * p.heads + h) * p.segments + seg) * D * D;
  for (int i = threadIdx.x; i < D * D; i += THREADS) dst[i] = S[i];
}

// In place: what each segment adds becomes the state before it.  (bf16's segments as well.)
template <int D>
__global__ void __launch_bounds__(THREADS) linear_scan_kernel(const __grid_constant__ LinearParams p) {
  const int b = blockIdx.z, h = blockIdx.y, i = (int)blockIdx.x * THREADS + (int)threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();             // (fp32 only: bf16's next grid, launched ahead of this one's end, made eight maps 112 us of 104)
  const int slot = slot_of(p.slots, p.num_slots, b);
  if (slot < 0) return;
  const int n = clamp_length(p.lengths, b, p.tokens);
  const float decay = decay_power(p.log_decay[h], p.seg_tokens);
  float* seg = p.seg_state + ((int64_t)b * p.heads + h) * p.segments * D * D + i;
  const int segments = max(1, (n + p.seg_tokens - 1) / p.seg_tokens);
  float cur = p.state[((int64_t)slot * p.heads + h) * D * D + i];
  // eight segments' loads are in flight together
  for (int s0 = 0; s0 < segments; s0 += 8) {
    float add[8];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s0 + s + 1 < segments) add[s] = seg[(int64_t)(s0 + s) * D * D];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s0 + s < segments) {
        seg[(int64_t)(s0 + s) * D * D] = cur;
        if (s0 + s + 1 < segments) cur = fmaf(decay, cur, add[s]);
      }
  }
}

template <int D>
__global__ void __launch_bounds__(THREADS) linear_chunk_kernel(const __grid_constant__ LinearParams p) {
  extern __shared__ float4 raw[];
  float* smem = reinterpret_cast<float*>(raw);
  float* S = state_in_shared<D>(smem);
  const int b = blockIdx.z, h = blockIdx.y, seg = blockIdx.x;
  const int slot = slot_of(p.slots, p.num_slots, b);
  pdl_wait();
  if (slot < 0) return;
  const int n = clamp_length(p.lengths, b, p.tokens), t0 = seg * p.seg_tokens, t1 = min(n, t0 + p.seg_tokens);
  if (seg > 0 && t0 >= n) return;
  const int64_t at = ((int64_t)slot * p.heads + h) * D * D;
  const float* src = p.segments > 1 ? p.seg_state + (((int64_t)b * p.heads + h) * p.segments + seg) * D * D : p.state + at;
  Tile<D, D> first;
  first.load(src, D, D);
  first.store(S, D);
  run_chunks<D, true>(p, b, h, t0, t1, S, smem);
  if (t1 == n)
    for (int i = threadIdx.x; i < D * D; i += THREADS) p.state_out[at + i] = S[i];
}

template <int D>
cudaError_t launch(const LinearParams& p, cudaStream_t s) {
  const size_t smem = ChunkShape<D>::smem;
  static OncePerContext once;
  cudaError_t e = once([&] {
    cudaError_t r = cudaFuncSetAttribute(linear_segment_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return r != cudaSuccess ? r : cudaFuncSetAttribute(linear_chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  });
  if (e != cudaSuccess) return e;
  if (p.segments > 1) {
    linear_segment_kernel<D><<<dim3((unsigned)p.segments - 1, (unsigned)p.heads, (unsigned)p.batch), THREADS, smem, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if ((e = launch_linear_scan(p, D, s)) != cudaSuccess) return e;
  }
  return launch_kernel(linear_chunk_kernel<D>, dim3((unsigned)p.segments, (unsigned)p.heads, (unsigned)p.batch), THREADS, smem, s, p, p.segments > 1);
}
}  // namespace

// One block to a multiprocessor: a few with two would be what the rest waits for (fp32, 2 x 2 heads of 64 on 4801 tokens: 152 segments of 128
// tokens 49 us, 124 of 160 tokens 43).  bf16 segments are whole chunks; three launches are not worth it for less than 128 tokens more.
void linear_plan(int batch, int tokens, int heads, bool bf16, int* segments, int* seg_tokens) {
  const int64_t sequences = (int64_t)batch * heads;
  const int step = bf16 ? 128 : 32;
  const int64_t most = ((int64_t)tokens + 127) / 128, want = PLAN_SMS / sequences;
  int64_t n = want < most ? want : most;
  if (n < 1) n = 1;
  const int64_t each = tokens > 0 ? ((tokens + n - 1) / n + step - 1) / step * step : step;
  *seg_tokens = (int)each;
  *segments = tokens > 0 ? (int)((tokens + each - 1) / each) : 1;
}

cudaError_t launch_linear_scan(const LinearParams& p, int D, cudaStream_t s) {
  const dim3 grid((unsigned)(D * D / THREADS), (unsigned)p.heads, (unsigned)p.batch);
  return launch_kernel(D == 32 ? linear_scan_kernel<32> : D == 64 ? linear_scan_kernel<64> : linear_scan_kernel<128>, grid, THREADS, 0, s, p, true);
}

cudaError_t launch_linear_chunk(const LinearParams& p, int D, cudaStream_t s) {
  return D == 32 ? launch<32>(p, s) : D == 64 ? launch<64>(p, s) : launch<128>(p, s);
}

}  // namespace tok
}  // namespace tt

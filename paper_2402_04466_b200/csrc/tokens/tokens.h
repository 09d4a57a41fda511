// Launch interfaces of the operators over tokens (tt.h: tt_qk_norm_rope, tt_linear_attention, tt_delta_rule, tt_cross_attention,
// tt_differential_attention).
#pragma once

#include <type_traits>

#include "../tt_internal.h"

namespace tt {
namespace tok {

// Grids and splits are planned for this many multiprocessors, whatever the device has, so that scratch sizes and the order of
// every sum are the same wherever the call is planned.
constexpr int PLAN_SMS = 148;

// [batch][token][head][head_dim] view, strides in elements
struct View {
  void* p;
  int64_t b, t, h;
};

struct alignas(32) RopeParams {
  View x[2], y[2];              // queries, keys
  const float* weight[2];       // or null
  const int64_t* positions;
  const double* inv_freq;
  const int32_t* lengths;
  int64_t pos_stride;
  int32_t tokens, heads[2], rot, norm;
  float eps, rot_scale;
  int32_t batch;
};
cudaError_t launch_qk_norm_rope(const RopeParams& p, bool bf16, int D, bool interleaved, cudaStream_t s);

struct alignas(32) LinearParams {
  View q, k, v, o;
  const float* log_decay;
  const float* state;
  float* state_out;
  const int32_t* slots;
  const int32_t* lengths;
  float* seg_state;             // [batch][heads][segments][D][D], where segments > 1
  int32_t* status;
  int32_t batch, tokens, heads, group;     // group: query heads to a key and value head
  int32_t num_slots, segments, seg_tokens; // tokens to a segment
  float scale;
};
// How many segments the tokens are cut into, and of how many tokens.
void linear_plan(int batch, int tokens, int heads, bool bf16, int* segments, int* seg_tokens);
cudaError_t launch_linear_step(const LinearParams& p, bool bf16, int D, cudaStream_t s);
cudaError_t launch_linear_chunk(const LinearParams& p, int D, cudaStream_t s);    // fp32, and calls without tokens
cudaError_t launch_linear_tc(const LinearParams& p, int D, cudaStream_t s);       // bf16
cudaError_t launch_linear_scan(const LinearParams& p, int D, cudaStream_t s);     // what segments add -> the states before them

struct alignas(32) DeltaParams {
  View q, k, v, o;
  const float* log_decay;       // or null
  const float* beta;
  const float* state;
  float* state_out;
  const int32_t* slots;
  const int32_t* lengths;
  int32_t batch, tokens, heads, group;     // group: heads to a query and key head
  int32_t num_slots;
  float scale;
  int32_t first_window, windows;           // of several tokens: windows first_window .. + windows - 1 of every sequence, in order
  void* records;                           // [batch][heads][windows]: DeltaRecord
  int32_t more;                            // windows follow, whose preparation may begin
};
cudaError_t launch_delta_step(const DeltaParams& p, bool bf16, int D, cudaStream_t s);      // token by token
cudaError_t launch_delta_prepare(const DeltaParams& p, bool bf16, int D, cudaStream_t s);   // of every window, what depends on no state
cudaError_t launch_delta_chunk(DeltaParams p, bool bf16, int D, cudaStream_t s);            // a window of tokens at a time, prepared range by range or on the way
uint64_t delta_scratch(int batch, int tokens, int heads, int D, bool bf16);
// Few tokens are taken one by one: a window takes its way through the products whatever it holds.  Both measured, us one by one and by window.  bf16, 8 and 12 tokens, heads of 32, 64, 128: five
// entries of 2 heads 5.1 5.6, 7.0 6.3; 7.6 6.3, 9.8 6.3; 9.1 6.4, 11.9 7.0; 256 of 8 heads 37 50, 53 52; 56 72, 78 72; 156 191, 218 191.  fp32, 12 and 16 tokens, heads of 32 and 64: five entries
// 6.4 7.8, 8.3 7.7; 9.7 9.0, 11.9 9.0; 256 53 66, 70 67; 78 102, 100 103.  fp32 windows of heads of 128 take longest and have a block to a multiprocessor: five entries, 12 tokens 12.0 11.1; 160
// states (few more than multiprocessors, which is two rounds of blocks one by one) 24 tokens 49 51, 28 56 53; 296 states 32 tokens 79 89, 33 82 125, 48 115 127, 56 132 129; 2048 states 24 tokens
// 396 561, 33 532 836, 48 760 853.
inline bool delta_by_window(int batch, int tokens, int heads, int D, bool bf16) {
  const int64_t states = (int64_t)batch * heads;
  return tokens > (bf16 ? 8 : D < 128 || states < PLAN_SMS ? 12 : states < 2 * PLAN_SMS ? 24 : 48);
}

struct alignas(32) CrossParams {
  View q, k, v, o;
  const int32_t* q_lengths;
  const int32_t* kv_lengths;
  const uint8_t* mask;          // or null
  int64_t mask_b, mask_q;
  float* part;                  // partial results where splits > 1: see cross_attention.cu
  int32_t* status;
  int32_t batch, q_tokens, kv_tokens, heads, group;
  int32_t splits, split_keys;   // keys to a split; 0: an entry's keys in `splits` equal pieces
  int32_t cluster;              // blocks that share a piece
  float scale_log2;             // scale * log2(e)
};
// Differential attention is cross attention with two maps, each of one half of a head's queries and keys, over the same values, and an end of its own.
struct DiffEnd {
  const float* lambda;          // four vectors of head_dim / 2
  int64_t lambda_h;             // from one head's to the next's, 0: shared
  const float* weight;          // of the norm, or null
  float lambda_init, eps, out_scale;
  int32_t norm;
};
struct alignas(32) DiffParams : CrossParams {
  DiffEnd end;
};
template <int MAPS>
using ParamsOf = std::conditional_t<MAPS == 2, DiffParams, CrossParams>;
enum { CROSS_SCALAR = 0, CROSS_TC = 1, CROSS_FEW = 2 };
struct CrossPlan {
  int32_t kernel;               // one of CROSS_...
  int32_t rows;                 // CROSS_SCALAR: rows (queries x heads of a group) of a block's tile
  int32_t warps;                // CROSS_FEW: of a block
  int32_t splits, split_keys, cluster;
  uint64_t scratch;
};
CrossPlan cross_plan(int batch, int q_tokens, int kv_tokens, int heads, int group, int D, bool bf16, bool mask, int maps);
template <int MAPS>
cudaError_t launch_cross(const ParamsOf<MAPS>& p, const CrossPlan& plan, bool bf16, int D, cudaStream_t s);

template <int MAPS>
cudaError_t launch_cross_few(const ParamsOf<MAPS>& p, int D, int warps, cudaStream_t s);   // splits > 1: the join is the caller's
template <int MAPS>
cudaError_t launch_cross_tc(const ParamsOf<MAPS>& p, int D, cudaStream_t s);      // kv_tokens > 0
uint64_t cross_tc_scratch(int batch, int q_tokens, int kv_tokens, int heads, int D, int maps);

// Tensor map of a bf16 view, boxes of `box` tokens of one head.  An axis of stride 0 has one place.
bool token_map(TensorMap128* map, const View& v, int D, int tokens, int heads, int batch, int box = 128);

// ------------------------------------------------------------------------------- device helpers
__device__ __forceinline__ int clamp_length(const int32_t* lengths, int b, int extent) {
  if (!lengths) return extent;
  const int n = lengths[b];
  return n < 0 ? 0 : n > extent ? extent : n;
}

// Where a row's partial results lie: [batch][kv head][row][map][split], maximum and total first, then the sums.
struct Part {
  float2* stat;
  float* sum;
};
template <int MAPS>
__device__ __forceinline__ Part part_of(const CrossParams& p, int D, int b, int hk, int row, int map) {
  const int64_t rows = (int64_t)p.q_tokens * p.group * MAPS, all = rows * p.batch * (p.heads / p.group);
  const int64_t at = (((int64_t)b * (p.heads / p.group) + hk) * rows + (int64_t)row * MAPS + map) * p.splits;
  return {reinterpret_cast<float2*>(p.part + all * p.splits * D) + at, p.part + at * D};
}

// lambda of head h; a whole warp calls it.
__device__ __forceinline__ float lambda_of(const DiffEnd& e, int half, int h) {
  const float* v = e.lambda + h * e.lambda_h;
  float a = 0.f, c = 0.f;
  for (int i = threadIdx.x % 32; i < half; i += 32) {
    a = fmaf(v[i], v[half + i], a);
    c = fmaf(v[2 * half + i], v[3 * half + i], c);
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, x);
    c += __shfl_xor_sync(0xFFFFFFFFu, c, x);
  }
  return expf(a) - expf(c) + e.lambda_init;
}
// What a row's difference is multiplied by, from the sum of its squares: a row of zeros stays one, whatever eps is.
template <int D>
__device__ __forceinline__ float row_gain(const DiffEnd& e, float squares) {
  if (!e.norm) return e.out_scale;
  const float mean = fmaf(squares, 1.f / D, e.eps);
  return mean == 0.f ? 0.f : e.out_scale * rsqrtf(mean);
}
__device__ __forceinline__ float norm_weight(const DiffEnd& e, int d) { return e.norm && e.weight ? __ldg(e.weight + d) : 1.f; }

}  // namespace tok
}  // namespace tt

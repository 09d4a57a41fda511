// Launch interfaces of the operators over tokens (tt.h: tt_qk_norm_rope, tt_linear_attention, tt_cross_attention).
#pragma once

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
enum { CROSS_SCALAR = 0, CROSS_TC = 1, CROSS_FEW = 2 };
struct CrossPlan {
  int32_t kernel;               // one of CROSS_...
  int32_t rows;                 // CROSS_SCALAR: rows (queries x heads of a group) of a block's tile
  int32_t warps;                // CROSS_FEW: of a block
  int32_t splits, split_keys, cluster;
  uint64_t scratch;
};
CrossPlan cross_plan(int batch, int q_tokens, int kv_tokens, int heads, int group, int D, bool bf16, bool mask);
cudaError_t launch_cross(const CrossParams& p, const CrossPlan& plan, bool bf16, int D, cudaStream_t s);

cudaError_t launch_cross_few(const CrossParams& p, int D, int warps, cudaStream_t s);   // splits > 1: the join is the caller's
cudaError_t launch_cross_tc(const CrossParams& p, int D, cudaStream_t s);         // kv_tokens > 0
uint64_t cross_tc_scratch(int batch, int q_tokens, int kv_tokens, int heads, int D);

// Tensor map of a bf16 view, boxes of `box` tokens of one head.  An axis of stride 0 has one place.
bool token_map(TensorMap128* map, const View& v, int D, int tokens, int heads, int batch, int box = 128);

// ------------------------------------------------------------------------------- device helpers
__device__ __forceinline__ int clamp_length(const int32_t* lengths, int b, int extent) {
  if (!lengths) return extent;
  const int n = lengths[b];
  return n < 0 ? 0 : n > extent ? extent : n;
}

// Where a row's partial results lie: [batch][kv head][row][split], maximum and total first, then the sums.
struct Part {
  float2* stat;
  float* sum;
};
__device__ __forceinline__ Part part_of(const CrossParams& p, int D, int b, int hk, int row) {
  const int64_t rows = (int64_t)p.q_tokens * p.group, all = rows * p.batch * (p.heads / p.group);
  const int64_t at = (((int64_t)b * (p.heads / p.group) + hk) * rows + row) * p.splits;
  return {reinterpret_cast<float2*>(p.part + all * p.splits * D) + at, p.part + at * D};
}

}  // namespace tok
}  // namespace tt

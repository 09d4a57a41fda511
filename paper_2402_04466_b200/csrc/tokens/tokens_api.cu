// Entry points of the operators over tokens: argument checks, plans and launches.  Everything the kernels assume about sizes,
// strides and alignment is checked here, so that a bad argument is a status and never a device fault.
#include <cmath>
#include <utility>

#include "tokens.h"

using namespace tt;
using namespace tt::tok;

namespace {

constexpr int64_t MAX_EXTENT = 1 << 28;      // tokens of an entry
constexpr int64_t MAX_STRIDE = 1ll << 38;    // elements: what a tensor map holds, in bytes of either type
constexpr int64_t MAX_REACH = 1ll << 46;     // elements between a view's first and last

bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// `size`: bytes of an element.  An empty view (no tokens) needs no pointer.
bool bad_view(const char* who, const char* name, const tt_tokens& v, int64_t batch, int64_t tokens, int64_t heads, int size) {
  if (batch * tokens * heads == 0) return false;
  if (!v.data) return set_error(TT_ERR_INVALID_ARG, "%s: %s is null", who, name), true;
  const int64_t unit = 16 / size, limit = MAX_REACH;
  if (misaligned(v.data, 16)) return set_error(TT_ERR_INVALID_ARG, "%s: %s must start on 16 bytes", who, name), true;
  if (tokens > 1 && v.token_stride == 0) return set_error(TT_ERR_INVALID_ARG, "%s: token_stride of %s is 0", who, name), true;
  const int64_t strides[3] = {v.batch_stride, v.token_stride, v.head_stride}, extents[3] = {batch, tokens, heads};
  int64_t reach = 0;
  for (int i = 0; i < 3; ++i) {
    if (extents[i] == 1) continue;             // never stepped along: whatever it says
    if (strides[i] % unit) return set_error(TT_ERR_INVALID_ARG, "%s: strides of %s must be whole multiples of 16 bytes", who, name), true;
    if (strides[i] < 0 || strides[i] > MAX_STRIDE || strides[i] > (limit - reach) / (extents[i] - 1))
      return set_error(TT_ERR_INVALID_ARG, "%s: a stride of %s is negative or too large", who, name), true;
    reach += strides[i] * (extents[i] - 1);
  }
  return false;
}

// The axes of an output do not run into each other: sorted by stride, each steps over all of those before it.
bool folded(const char* who, const char* name, const tt_tokens& v, int64_t batch, int64_t tokens, int64_t heads, int64_t dim) {
  if (batch * tokens * heads == 0) return false;
  int64_t s[3] = {v.batch_stride, v.token_stride, v.head_stride}, n[3] = {batch, tokens, heads};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[j] < s[i]) { std::swap(s[i], s[j]); std::swap(n[i], n[j]); }
  int64_t span = dim;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (s[i] < span) return set_error(TT_ERR_INVALID_ARG, "%s: rows of %s overlap each other", who, name), true;
    span = s[i] * (n[i] - 1) + span;
  }
  return false;
}

// Strides of axes of extent 1 are taken as 0.
View view(const tt_tokens& v, int64_t batch, int64_t tokens, int64_t heads) {
  return {v.data, batch > 1 ? v.batch_stride : 0, tokens > 1 ? v.token_stride : 0, heads > 1 ? v.head_stride : 0};
}

bool bad_head_dim(const char* who, int32_t d) {
  if (d == 32 || d == 64 || d == 128) return false;
  return set_error(TT_ERR_UNSUPPORTED, "%s: head_dim must be 32, 64 or 128", who), true;
}
bool extent(int64_t n, int64_t least, int64_t most) { return n >= least && n <= most; }

}  // namespace

extern "C" {

tt_status tt_qk_norm_rope(const tt_qk_norm_rope_args* a, void* cuda_stream) {
  const char* who = "tt_qk_norm_rope";
  if (!a || a->struct_size != sizeof(*a)) return set_error(TT_ERR_INVALID_ARG, "%s: struct_size", who);
  if ((a->precision != TT_FP32 && a->precision != TT_BF16) || !extent(a->batch, 1, 65535) || !extent(a->tokens, 0, MAX_EXTENT) ||
      !extent(a->q_heads, 0, 4096) || !extent(a->k_heads, 0, 4096) || a->q_heads + a->k_heads < 1 || !std::isfinite(a->rot_scale) ||
      (a->norm && !(a->eps >= 0.f && std::isfinite(a->eps))) || a->position_stride < 0 || a->position_stride > MAX_REACH / 65536)
    return set_error(TT_ERR_INVALID_ARG, "%s: bad argument", who);
  if (bad_head_dim(who, a->head_dim)) return TT_ERR_UNSUPPORTED;
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 8)
    return set_error(TT_ERR_INVALID_ARG, "%s: rot_dim must be a multiple of 8 up to head_dim", who);
  const int size = a->precision == TT_BF16 ? 2 : 4;
  if (bad_view(who, "q", a->q, a->batch, a->tokens, a->q_heads, size) || bad_view(who, "q_out", a->q_out, a->batch, a->tokens, a->q_heads, size) ||
      bad_view(who, "k", a->k, a->batch, a->tokens, a->k_heads, size) || bad_view(who, "k_out", a->k_out, a->batch, a->tokens, a->k_heads, size) ||
      folded(who, "q_out", a->q_out, a->batch, a->tokens, a->q_heads, a->head_dim) || folded(who, "k_out", a->k_out, a->batch, a->tokens, a->k_heads, a->head_dim))
    return TT_ERR_INVALID_ARG;
  if (a->rot_dim && a->tokens && (!a->positions || !a->inv_freq)) return set_error(TT_ERR_INVALID_ARG, "%s: positions and inv_freq are needed for a rotation", who);
  if (misaligned(a->q_weight, 4) || misaligned(a->k_weight, 4) || misaligned(a->lengths, 4) || misaligned(a->positions, 8) || misaligned(a->inv_freq, 8))
    return set_error(TT_ERR_INVALID_ARG, "%s: misaligned pointer", who);
  if (a->tokens == 0) return TT_OK;
  RopeParams p{};
  p.x[0] = view(a->q, a->batch, a->tokens, a->q_heads); p.x[1] = view(a->k, a->batch, a->tokens, a->k_heads);
  p.y[0] = view(a->q_out, a->batch, a->tokens, a->q_heads); p.y[1] = view(a->k_out, a->batch, a->tokens, a->k_heads);
  p.weight[0] = a->norm ? a->q_weight : nullptr; p.weight[1] = a->norm ? a->k_weight : nullptr;
  p.positions = a->positions; p.inv_freq = a->inv_freq; p.lengths = a->lengths; p.pos_stride = a->position_stride;
  p.tokens = a->tokens; p.heads[0] = a->q_heads; p.heads[1] = a->k_heads; p.rot = a->rot_dim; p.norm = a->norm != 0;
  p.eps = a->eps; p.rot_scale = a->rot_scale; p.batch = a->batch;
  const cudaError_t e = launch_qk_norm_rope(p, size == 2, a->head_dim, a->interleaved != 0, reinterpret_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? TT_OK : set_error(TT_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

tt_status tt_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double trained, double slow_turns,
                              double fast_turns, double* inv_freq, float* rot_scale) {
  const char* who = "tt_rope_frequencies";
  if (rot_dim < 0 || rot_dim > 128 || rot_dim % 2 || !(base > 1.0) || !std::isfinite(base) || scaling < TT_ROPE_PLAIN || scaling > TT_ROPE_BY_PARTS ||
      (rot_dim && !inv_freq) || !rot_scale || (scaling != TT_ROPE_PLAIN && !(factor >= 1.0 && std::isfinite(factor))) ||
      (scaling == TT_ROPE_BASE && rot_dim == 2) ||
      (scaling == TT_ROPE_BY_PARTS && !(trained > 0.0 && std::isfinite(trained) && slow_turns >= 0.0 && fast_turns > slow_turns && std::isfinite(fast_turns))))
    return set_error(TT_ERR_INVALID_ARG, "%s: bad argument", who);
  if (scaling == TT_ROPE_BASE && rot_dim) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    if (scaling == TT_ROPE_LINEAR) f /= factor;
    if (scaling == TT_ROPE_BY_PARTS) {
      double keep = (trained * f / 6.283185307179586477 - slow_turns) / (fast_turns - slow_turns);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f *= keep + (1.0 - keep) / factor;
    }
    inv_freq[i] = f;
  }
  *rot_scale = scaling == TT_ROPE_BY_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return TT_OK;
}

static tt_status check_linear(const char* who, const tt_linear_attention_args* a) {
  if (!a || a->struct_size != sizeof(*a)) return set_error(TT_ERR_INVALID_ARG, "%s: struct_size", who);
  if ((a->precision != TT_FP32 && a->precision != TT_BF16) || !extent(a->batch, 1, 65535) || !extent(a->tokens, 0, MAX_EXTENT) ||
      !extent(a->heads, 1, 4096) || !extent(a->kv_heads, 1, a->heads) || a->heads % a->kv_heads || !extent(a->num_slots, 1, MAX_EXTENT) ||
      !std::isfinite(a->scale))
    return set_error(TT_ERR_INVALID_ARG, "%s: bad argument", who);
  if (bad_head_dim(who, a->head_dim)) return TT_ERR_UNSUPPORTED;
  if (!a->slots && a->batch > a->num_slots) return set_error(TT_ERR_INVALID_ARG, "%s: more entries than slots", who);
  return TT_OK;
}

uint64_t tt_linear_attention_scratch_bytes(const tt_linear_attention_args* a) {
  if (check_linear("tt_linear_attention_scratch_bytes", a) != TT_OK) return 0;
  int segments, seg_tokens;
  linear_plan(a->batch, a->tokens, a->heads, a->precision == TT_BF16, &segments, &seg_tokens);
  return segments > 1 ? (uint64_t)a->batch * (uint64_t)a->heads * (uint64_t)segments * (uint64_t)(a->head_dim * a->head_dim) * 4u : 0u;
}

tt_status tt_linear_attention(const tt_linear_attention_args* a, void* cuda_stream) {
  const char* who = "tt_linear_attention";
  const tt_status st = check_linear(who, a);
  if (st != TT_OK) return st;
  const bool bf16 = a->precision == TT_BF16;
  const int size = bf16 ? 2 : 4;
  if (bad_view(who, "q", a->q, a->batch, a->tokens, a->heads, size) || bad_view(who, "k", a->k, a->batch, a->tokens, a->kv_heads, size) ||
      bad_view(who, "v", a->v, a->batch, a->tokens, a->kv_heads, size) || bad_view(who, "out", a->out, a->batch, a->tokens, a->heads, size) ||
      folded(who, "out", a->out, a->batch, a->tokens, a->heads, a->head_dim))
    return TT_ERR_INVALID_ARG;
  if (!a->log_decay || !a->state || !a->state_out || misaligned(a->log_decay, 4) || misaligned(a->state, 16) || misaligned(a->state_out, 16) ||
      misaligned(a->slots, 4) || misaligned(a->lengths, 4) || misaligned(a->status_dev, 4))
    return set_error(TT_ERR_INVALID_ARG, "%s: log_decay, state or state_out is null, or a pointer is misaligned (states: 16 bytes)", who);
  const uint64_t need = tt_linear_attention_scratch_bytes(a);
  if (need && (!a->scratch || misaligned(a->scratch, 16) || a->scratch_bytes < need))
    return set_error(TT_ERR_INVALID_ARG, "%s: scratch is null, misaligned or smaller than %llu bytes", who, (unsigned long long)need);
  LinearParams p{};
  p.q = view(a->q, a->batch, a->tokens, a->heads); p.k = view(a->k, a->batch, a->tokens, a->kv_heads);
  p.v = view(a->v, a->batch, a->tokens, a->kv_heads); p.o = view(a->out, a->batch, a->tokens, a->heads);
  p.log_decay = a->log_decay; p.state = a->state; p.state_out = a->state_out; p.slots = a->slots; p.lengths = a->lengths;
  p.seg_state = static_cast<float*>(a->scratch); p.status = a->status_dev;
  p.batch = a->batch; p.tokens = a->tokens; p.heads = a->heads; p.group = a->heads / a->kv_heads; p.num_slots = a->num_slots;
  p.scale = a->scale;
  linear_plan(a->batch, a->tokens, a->heads, bf16, &p.segments, &p.seg_tokens);
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = a->tokens == 1             ? launch_linear_step(p, bf16, a->head_dim, s)
                        : bf16 && a->tokens > 0 ? launch_linear_tc(p, a->head_dim, s)
                                                : launch_linear_chunk(p, a->head_dim, s);
  return e == cudaSuccess ? TT_OK : set_error(TT_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

static tt_status check_delta(const char* who, const tt_delta_rule_args* a) {
  if (!a || a->struct_size != sizeof(*a)) return set_error(TT_ERR_INVALID_ARG, "%s: struct_size", who);
  if ((a->precision != TT_FP32 && a->precision != TT_BF16) || !extent(a->batch, 1, 65535) || !extent(a->tokens, 0, MAX_EXTENT) ||
      !extent(a->heads, 1, 4096) || !extent(a->qk_heads, 1, a->heads) || a->heads % a->qk_heads || !extent(a->num_slots, 1, MAX_EXTENT) ||
      !std::isfinite(a->scale))
    return set_error(TT_ERR_INVALID_ARG, "%s: bad argument", who);
  if (bad_head_dim(who, a->head_dim)) return TT_ERR_UNSUPPORTED;
  if (!a->slots && a->batch > a->num_slots) return set_error(TT_ERR_INVALID_ARG, "%s: more entries than slots", who);
  return TT_OK;
}

uint64_t tt_delta_rule_scratch_bytes(const tt_delta_rule_args* a) {
  if (check_delta("tt_delta_rule_scratch_bytes", a) != TT_OK || !delta_by_window(a->batch, a->tokens, a->heads, a->head_dim, a->precision == TT_BF16)) return 0;
  return delta_scratch(a->batch, a->tokens, a->heads, a->head_dim, a->precision == TT_BF16);
}

tt_status tt_delta_rule(const tt_delta_rule_args* a, void* cuda_stream) {
  const char* who = "tt_delta_rule";
  const tt_status st = check_delta(who, a);
  if (st != TT_OK) return st;
  const bool bf16 = a->precision == TT_BF16;
  const int size = bf16 ? 2 : 4;
  if (bad_view(who, "q", a->q, a->batch, a->tokens, a->qk_heads, size) || bad_view(who, "k", a->k, a->batch, a->tokens, a->qk_heads, size) ||
      bad_view(who, "v", a->v, a->batch, a->tokens, a->heads, size) || bad_view(who, "out", a->out, a->batch, a->tokens, a->heads, size) ||
      folded(who, "out", a->out, a->batch, a->tokens, a->heads, a->head_dim))
    return TT_ERR_INVALID_ARG;
  if ((a->tokens && !a->beta) || !a->state || !a->state_out || misaligned(a->log_decay, 4) || misaligned(a->beta, 4) || misaligned(a->state, 16) ||
      misaligned(a->state_out, 16) || misaligned(a->slots, 4) || misaligned(a->lengths, 4))
    return set_error(TT_ERR_INVALID_ARG, "%s: beta, state or state_out is null, or a pointer is misaligned (states: 16 bytes)", who);
  const uint64_t need = tt_delta_rule_scratch_bytes(a);
  if (need && (!a->scratch || misaligned(a->scratch, 16) || a->scratch_bytes < need))
    return set_error(TT_ERR_INVALID_ARG, "%s: scratch is null, misaligned or smaller than %llu bytes", who, (unsigned long long)need);
  DeltaParams p{};
  p.q = view(a->q, a->batch, a->tokens, a->qk_heads); p.k = view(a->k, a->batch, a->tokens, a->qk_heads);
  p.v = view(a->v, a->batch, a->tokens, a->heads); p.o = view(a->out, a->batch, a->tokens, a->heads);
  p.log_decay = a->log_decay; p.beta = a->beta; p.state = a->state; p.state_out = a->state_out; p.slots = a->slots; p.lengths = a->lengths;
  p.batch = a->batch; p.tokens = a->tokens; p.heads = a->heads; p.group = a->heads / a->qk_heads; p.num_slots = a->num_slots;
  p.scale = a->scale; p.records = a->scratch;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = delta_by_window(a->batch, a->tokens, a->heads, a->head_dim, bf16) ? launch_delta_chunk(p, bf16, a->head_dim, s) : launch_delta_step(p, bf16, a->head_dim, s);
  return e == cudaSuccess ? TT_OK : set_error(TT_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // extern "C"

// What tt_cross_attention and tt_differential_attention have in common: their arguments but for the end's have the same names.
template <typename Args>
static tt_status check_cross(const char* who, const Args* a) {
  if (!a || a->struct_size != sizeof(*a)) return set_error(TT_ERR_INVALID_ARG, "%s: struct_size", who);
  if ((a->precision != TT_FP32 && a->precision != TT_BF16) || !extent(a->batch, 1, 65535) || !extent(a->q_tokens, 0, MAX_EXTENT) ||
      !extent(a->kv_tokens, 0, MAX_EXTENT) || !extent(a->heads, 1, 4096) || !extent(a->kv_heads, 1, a->heads) || a->heads % a->kv_heads ||
      !((int64_t)a->q_tokens * (a->heads / a->kv_heads) <= MAX_EXTENT) || !(a->scale > 0.f && a->scale < 1e38f))
    return set_error(TT_ERR_INVALID_ARG, "%s: bad argument", who);
  if (bad_head_dim(who, a->head_dim)) return TT_ERR_UNSUPPORTED;
  return TT_OK;
}
template <typename Args>
static CrossPlan plan_of(const Args* a, int maps) {
  return cross_plan(a->batch, a->q_tokens, a->kv_tokens, a->heads, a->heads / a->kv_heads, a->head_dim, a->precision == TT_BF16, a->mask != nullptr, maps);
}
template <typename Args>
static tt_status check_cross_operands(const char* who, const Args* a, const CrossPlan& plan) {
  const int size = a->precision == TT_BF16 ? 2 : 4;
  if (bad_view(who, "q", a->q, a->batch, a->q_tokens, a->heads, size) || bad_view(who, "k", a->k, a->batch, a->kv_tokens, a->kv_heads, size) ||
      bad_view(who, "v", a->v, a->batch, a->kv_tokens, a->kv_heads, size) || bad_view(who, "out", a->out, a->batch, a->q_tokens, a->heads, size) ||
      folded(who, "out", a->out, a->batch, a->q_tokens, a->heads, a->head_dim))
    return TT_ERR_INVALID_ARG;
  if (misaligned(a->q_lengths, 4) || misaligned(a->kv_lengths, 4) || misaligned(a->status_dev, 4))
    return set_error(TT_ERR_INVALID_ARG, "%s: a length array or status_dev is misaligned", who);
  if (a->mask && (!extent(a->mask_batch_stride, 0, MAX_REACH / a->batch) || !extent(a->mask_query_stride, 0, MAX_REACH / (a->q_tokens + 1ll))))
    return set_error(TT_ERR_INVALID_ARG, "%s: a mask stride is negative or too large", who);
  if (plan.scratch && (!a->scratch || misaligned(a->scratch, 16) || a->scratch_bytes < plan.scratch))
    return set_error(TT_ERR_INVALID_ARG, "%s: scratch is null, misaligned or smaller than %llu bytes", who, (unsigned long long)plan.scratch);
  return TT_OK;
}
template <typename Args>
static void fill_cross(CrossParams& p, const Args* a, const CrossPlan& plan) {
  p.q = view(a->q, a->batch, a->q_tokens, a->heads); p.k = view(a->k, a->batch, a->kv_tokens, a->kv_heads);
  p.v = view(a->v, a->batch, a->kv_tokens, a->kv_heads); p.o = view(a->out, a->batch, a->q_tokens, a->heads);
  p.q_lengths = a->q_lengths; p.kv_lengths = a->kv_lengths; p.mask = a->mask; p.mask_b = a->mask_batch_stride; p.mask_q = a->mask_query_stride;
  p.part = static_cast<float*>(a->scratch); p.status = a->status_dev;
  p.batch = a->batch; p.q_tokens = a->q_tokens; p.kv_tokens = a->kv_tokens; p.heads = a->heads; p.group = a->heads / a->kv_heads;
  p.splits = plan.splits; p.split_keys = plan.split_keys; p.cluster = plan.cluster;
  p.scale_log2 = (float)((double)a->scale * 1.4426950408889634074);
}

extern "C" {

uint64_t tt_cross_attention_scratch_bytes(const tt_cross_attention_args* a) {
  return check_cross("tt_cross_attention_scratch_bytes", a) == TT_OK ? plan_of(a, 1).scratch : 0;
}

tt_status tt_cross_attention(const tt_cross_attention_args* a, void* cuda_stream) {
  const char* who = "tt_cross_attention";
  tt_status st = check_cross(who, a);
  if (st != TT_OK) return st;
  const CrossPlan plan = plan_of(a, 1);
  if ((st = check_cross_operands(who, a, plan)) != TT_OK) return st;
  if (a->q_tokens == 0) return TT_OK;
  CrossParams p{};
  fill_cross(p, a, plan);
  const cudaError_t e = launch_cross<1>(p, plan, a->precision == TT_BF16, a->head_dim, reinterpret_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? TT_OK : set_error(TT_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

uint64_t tt_differential_attention_scratch_bytes(const tt_differential_attention_args* a) {
  return check_cross("tt_differential_attention_scratch_bytes", a) == TT_OK ? plan_of(a, 2).scratch : 0;
}

tt_status tt_differential_attention(const tt_differential_attention_args* a, void* cuda_stream) {
  const char* who = "tt_differential_attention";
  tt_status st = check_cross(who, a);
  if (st != TT_OK) return st;
  if (!std::isfinite(a->lambda_init) || !std::isfinite(a->out_scale) || (a->norm && !(a->eps >= 0.f && std::isfinite(a->eps))) ||
      !extent(a->lambda_head_stride, 0, MAX_STRIDE))
    return set_error(TT_ERR_INVALID_ARG, "%s: lambda_init, out_scale, eps or lambda_head_stride", who);
  if (!a->lambda_vectors || misaligned(a->lambda_vectors, 4) || misaligned(a->norm_weight, 4))
    return set_error(TT_ERR_INVALID_ARG, "%s: lambda_vectors is null, or it or norm_weight misaligned", who);
  const CrossPlan plan = plan_of(a, 2);
  if ((st = check_cross_operands(who, a, plan)) != TT_OK) return st;
  if (a->q_tokens == 0) return TT_OK;
  DiffParams p{};
  fill_cross(p, a, plan);
  p.end.lambda = a->lambda_vectors; p.end.lambda_h = a->lambda_head_stride; p.end.weight = a->norm_weight;
  p.end.lambda_init = a->lambda_init; p.end.eps = a->eps; p.end.out_scale = a->out_scale; p.end.norm = a->norm != 0;
  const cudaError_t e = launch_cross<2>(p, plan, a->precision == TT_BF16, a->head_dim, reinterpret_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? TT_OK : set_error(TT_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // extern "C"

// What the kernels of tt_delta_rule over several tokens share: windows, operands cut into bf16 terms, and what is worked out of a window for the chain of states.
#pragma once

#include "linear_common.cuh"

#include "token_ptx.cuh"

namespace tt {
namespace tok {

constexpr int DELTA_C = 32;                  // tokens of a window
constexpr int DELTA_TT = DELTA_C / 8, DELTA_TK = DELTA_C / 16;      // tiles of them, products along them
constexpr int DELTA_GROUP = 128;             // threads that work together

// What is worked out of a window's keys, queries and gates, for every head: the inverse of its triangular system and the weights of its corrections in out, as the
// second operand's registers of products, for tile of 8 tokens `tile` the products along 16 tokens x = 0 .. tile / 2, and the gates.
template <int SEEN>
struct DeltaRecord {
  static constexpr int PLACES = 6;           // (tile, x)
  uint32_t inverse[PLACES][3][32][2];        // [][term][lane][]
  uint32_t weights[PLACES][SEEN][32][2];
  float beta[DELTA_C], up[DELTA_C], down[DELTA_C];      // G: the sum of log_decay up to and including a token; e^G, e^(G_C - G).  beta: NaN among them where a weight is not finite
  float whole;                               // e^G_C
  float pad[31];
};
__host__ __device__ constexpr int delta_place(int tile, int x) { return tile < 2 ? tile : 2 * tile - 2 + x; }

// a pair as three bf16 terms, a in the lower halves: the upper eight bits of what is left, cut off, which for the last term is all of it
__device__ __forceinline__ void cut(float a, float b, uint32_t (&t)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    t[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
    if (i < 2) {
      a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
      b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
    }
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
template <int THREADS>
__device__ __forceinline__ void barrier_of(int id) { asm volatile("barrier.sync %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
__device__ __forceinline__ void copy16(void* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
// A group's rows of a window, 16 bytes to a thread and pass
template <typename T, int ROWLEN>
struct Rows {
  static constexpr int EACH = 16 / (int)sizeof(T), ROW = ROWLEN / EACH, STEP = DELTA_GROUP / ROW, PASSES = (DELTA_C + STEP - 1) / STEP;
  const T* src;
  int64_t stride;
  int row, col;
  __device__ __forceinline__ Rows(const T* base, int64_t token_stride, int tid) : src(base), stride(token_stride), row(tid / ROW), col(tid % ROW * EACH) {}
  __device__ __forceinline__ void fetch(T* dst, int pitch, int first, int n) const {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = row + i * STEP;
      if (STEP * PASSES > DELTA_C && r >= DELTA_C) break;
      const bool there = first + r < n;
      copy16(dst + r * pitch + col, src + (there ? (int64_t)(first + r) * stride : 0) + col, there);
    }
  }
};

}  // namespace tok
}  // namespace tt

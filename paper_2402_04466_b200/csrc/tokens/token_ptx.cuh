// What the tensor-core kernels over tokens add to tc_ptx.cuh: operands in tensor memory, packed fp32 pairs, bounded waits that report
// to an optional status word.
#pragma once

#include "tokens.h"

#include "../tc_ptx.cuh"

namespace tt {
namespace tok {

using namespace tt::tc;

// Codes of waits that ran out: own hundreds beside those of tc_ptx.cuh.
constexpr int WAIT_CROSS_TC = 0xB00, WAIT_LINEAR_TC = 0xC00, WAIT_CROSS_FEW = 0xD00;

// D[tmem] += A[tmem] * B[shared]: A's row i is lane i, two bf16 to a column.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// instruction descriptor bits of operands whose rows are not along K but along M or N
constexpr uint32_t A_BY_ROWS = 1u << 15, B_BY_ROWS = 1u << 16;

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
// as tmem_ld32_async (tc_ptx.cuh), 16 columns
__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
// few registers: for the rare rescaling of an accumulator while a row of scores is held
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

typedef unsigned long long Two;        // two floats

// a * b + c and a + b on both halves of a pair
__device__ __forceinline__ unsigned long long fma2_of(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ unsigned long long add2_of(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul2_of(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long sub2_of(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Whether a barrier's phase is complete, without waiting: a fraction of what a try_wait takes.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r) : "r"(bar), "r"(parity) : "memory");
  return r != 0u;
}
// 2^x by the special-function unit: relative error about 2^-22, results below the normal range are 0
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// The columns of a row that belong to thread tx of 16, as pairs: four neighbours at 4 tx (and 64 + 4 tx), two at 2 tx where D is 32.
template <int D>
__device__ __forceinline__ void load_pairs(const float* row, int tx, Two (&f)[D / 32]) {
  if constexpr (D == 32) {
    f[0] = *reinterpret_cast<const Two*>(row + 2 * tx);
  } else {
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(row + 4 * tx + 64 * j);
      f[2 * j] = v.x; f[2 * j + 1] = v.y;
    }
  }
}

// Operand tile in shared memory whose rows (one token each) run along M or N: `group_bytes` from one group of 8 tokens to the next,
// `slab_bytes` from one run of 64 elements (128-byte rows) to the next.
__device__ __forceinline__ uint64_t make_rows_desc(uint32_t addr, uint32_t slab_bytes, uint32_t group_bytes, uint32_t layout_type) {
  return make_smem_desc_lbo(addr, slab_bytes, group_bytes, layout_type);
}

// SM cycles after which a wait gives up: the same as a context's default.
constexpr long long WAIT_LIMIT = DEFAULT_WAIT_LIMIT_CYCLES;

}  // namespace tok
}  // namespace tt

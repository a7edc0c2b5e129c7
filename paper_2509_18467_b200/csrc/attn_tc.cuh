// What the tensor-core attention kernels share: bounded waits, the A operand in tensor memory, tile loads, host-side planning.
#pragma once
#include "attn_exact.cuh"
#include "tc_common.cuh"

namespace lawcat {
namespace attn {

using namespace tc;

// D[tmem] (+)= A[tmem] * B[smem]: A has 16-bit elements, two to a 32-bit column, row r in lane r; a K step of 16 is 8 columns.
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Bounded wait: false when the block has been told to give up or the limit (clock cycles) ran out, which tells the others.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) {
      *abort_flag = 1;
      return false;
    }
  }
}

// rows x D channels of one head at token t into slabs of 64 channels (rows x 128 bytes, swizzled)
template <int D, int ROWS>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int t, int b) {
#pragma unroll
  for (int s = 0; s < D / 64; ++s) tma_load_4d(dst + s * (ROWS * 128), map, bar, s * 64, head, t, b);
}

// descriptor of a K-major operand tile (ROWS rows x D channels) at channel step kk (16 channels)
template <int ROWS>
__device__ __forceinline__ uint64_t kdesc(uint32_t tile, int kk) {
  return smem_desc(tile + (uint32_t)(kk >> 2) * (ROWS * 128) + (uint32_t)(kk & 3) * 32, 16, 1024, LAYOUT_SW128);
}
// descriptor of the same tile as an MN-major operand (its rows are the K index) at row step kk (16 rows)
template <int ROWS>
__device__ __forceinline__ uint64_t mdesc(uint32_t tile, int kk) {
  return smem_desc(tile + (uint32_t)kk * 2048, ROWS * 128, 1024, LAYOUT_SW128);
}

__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

}  // namespace attn
}  // namespace lawcat

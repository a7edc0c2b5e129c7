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

// Bounded wait: false when the block has been told to give up or the limit (clock cycles) ran out, which tells the others. (A
// try_wait may take microseconds to come back: under a limit of less, which only a test sets, the barrier is looked at instead.)
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
  const bool look = limit < 1000000LL;
  if (look ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
    if (look) {
      if (mbar_test_wait(bar, parity)) return true;
    } else {
#pragma unroll 1
      for (int i = 0; i < 64; ++i)
        if (mbar_try_wait(bar, parity)) return true;
    }
    if (*abort_flag) return false;
    if (clock64() - t0 > limit) {
      *abort_flag = 1;
      return false;
    }
  }
}

// The bound for a role that waits for the end of an item of n tiles: the others' bounds are on one step each, and tell this one when
// something is lost; by itself an item may take as long as its tiles do (2 s for each 64 of them, which take 0.1 ms).
__device__ __forceinline__ long long item_limit(long long limit, int n) { return limit * (1 + n / 64); }

// n / d for 0 <= n < 2^31: items are numbered, and their digits are run-time sizes (a division proper costs as much as an exponential
// of a whole row).
struct FastDiv {
  uint32_t d, mul, shift;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((1u << s) < d && s < 31) ++s;
  return FastDiv{d, (uint32_t)(((1ull << (31 + s)) / d) + 1), 31 + s};
}
__device__ __forceinline__ int quot(int n, const FastDiv& f) { return (int)(((uint64_t)(uint32_t)n * f.mul) >> f.shift); }
__device__ __forceinline__ int rest(int n, int q, const FastDiv& f) { return n - q * (int)f.d; }

__device__ __forceinline__ void tma_store_wait_read_1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }

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

// The launch has one block per item, and as many run as there are SMs: a running block takes over blocks that have not started
// (cluster launch control), whoever is free first. Their numbers fall with the items' lengths where a mask makes them differ.
__device__ __forceinline__ void ask_item(uint32_t answer, uint32_t bar) {
  fence_proxy_async();   // (the last answer has been read)
  mbar_arrive_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
// the number of the block that was taken over, or -1: all have started
__device__ __forceinline__ int read_item(uint32_t answer) {
  uint32_t got, idx;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
      : "=r"(got), "=r"(idx)
      : "r"(answer)
      : "memory");
  return got ? (int)idx : -1;
}

// Items of a block that came out not finite (noted by any of eight warps), for a second computation behind everything else. A block
// takes over no further items once it has one, so that the list holds those that are on their way then.
constexpr int BAD_MAX = 64;
__device__ __forceinline__ void note_bad(int* list, int* count, int idx) {
  const int at = atomicAdd(count, 1);
  if (at < BAD_MAX) list[at] = idx;
}
__device__ __forceinline__ bool noted_before(const int* list, int at) {
  for (int i = 0; i < at; ++i)
    if (list[i] == list[at]) return true;
  return false;
}

// s <- c2 tanh(s k) for N scores of a thread (all 32 lanes of a warp together). While no |s k| of the warp passes 0.4 (0.8), tanh is
// y P(y^2) with P of degree 3 (5) on the FMA pipe, k and c2 multiplied into its coefficients: least-maximum fits of tanh(y) / y over
// the range, relative error 1e-7 (5e-8), 2e-7 with their fp32 arithmetic. The two special functions of the other form would be three
// times the whole softmax's load on their pipe. Scores under a cap of 30 seldom pass 12.
template <int N, int DEG>
__device__ __forceinline__ void cap_poly(float (&s)[N], float k, float c2, const float (&coef)[DEG + 1]) {
  uint64_t c[DEG + 1];
  float f = k * c2;
#pragma unroll
  for (int i = 0; i <= DEG; ++i) {
    c[i] = f2_pack(coef[i] * f, coef[i] * f);
    f *= k * k;
  }
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const uint64_t x = f2_pack(s[i], s[i + 1]), z = f2_mul(x, x);
    uint64_t r = f2_fma(c[DEG], z, c[DEG - 1]);
#pragma unroll
    for (int d = DEG - 2; d >= 0; --d) r = f2_fma(r, z, c[d]);
    f2_unpack(f2_mul(x, r), s[i], s[i + 1]);
  }
}
// what scores `top` and below are in caps, for the choice of the cap's form
__device__ __forceinline__ float cap_reach(float top, float k) { return fabsf(k) < 1e4f ? top * fabsf(k) : 1.f; }
// y: cap_reach of this thread's scores
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], float k, float c2, float y) {
  if (__all_sync(0xffffffffu, y <= 0.4f)) {
    const float coef[4] = {0.9999998807907104f, -0.333313912153244f, 0.1327143758535385f, -0.04757280275225639f};
    cap_poly<N, 3>(s, k, c2, coef);
  } else if (__all_sync(0xffffffffu, y <= 0.8f)) {
    const float coef[6] = {0.9999999403953552f, -0.33332714438438416f, 0.13321532309055328f, -0.05313541740179062f, 0.019130872562527657f, -0.004378729499876499f};
    cap_poly<N, 5>(s, k, c2, coef);
  } else {
    const float k1 = 2.f * LOG2E * k;
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = c2 - 2.f * c2 * rcpf(1.f + ex2f(s[c] * k1));
  }
}
template <int N>
__device__ __forceinline__ float top_score(const float (&s)[N]) {
  float b0 = 0.f, b1 = 0.f;
#pragma unroll
  for (int c = 0; c < N; c += 4) {
    b0 = fmaxf(b0, fmaxf(fabsf(s[c]), fabsf(s[c + 1])));
    b1 = fmaxf(b1, fmaxf(fabsf(s[c + 2]), fabsf(s[c + 3])));
  }
  return fmaxf(b0, b1);
}
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], float k, float c2) { cap_scores(s, k, c2, cap_reach(top_score(s), k)); }

}  // namespace attn
}  // namespace lawcat

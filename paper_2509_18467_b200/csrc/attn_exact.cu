// Launches of the exact attention kernels (attn_exact.cuh).
// A block has 256 threads and 64 rows (RM = 4), or 16 rows (RM = 1) where blocks of 64 would leave most SMs idle: a tile's loads
// then serve a quarter of the products, but a call of 4 heads x 512 queries runs on 128 blocks instead of 32.
#include "attn_exact.cuh"

namespace lawcat {
namespace attn {

constexpr int THREADS = 256;

template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_fwd_exact_kernel(const Args a, int tiles) {
  extern __shared__ __align__(16) float sm[];
  const int bh = blockIdx.x % (a.B * a.H);
  const int t0 = (tiles - 1 - (int)(blockIdx.x / (a.B * a.H))) * 16 * RM;  // (under a causal mask the longest rows first)
  fwd_rows<T, D, RM, THREADS>(a, sm, bh / a.H, bh % a.H, t0, 0, a.mask.T_k, nullptr, nullptr);
}

// dq, and (lse log2e, dO.o) of every query for the other kernel
template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_dq_exact_kernel(const Args a, int tiles) {
  extern __shared__ __align__(16) float sm[];
  const int bh = blockIdx.x % (a.B * a.H);
  const int t0 = (tiles - 1 - (int)(blockIdx.x / (a.B * a.H))) * 16 * RM;
  dq_rows<T, D, RM, THREADS>(a, sm, bh / a.H, bh % a.H, t0);
}

template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_dkdv_exact_kernel(const Args a, int tiles) {
  extern __shared__ __align__(16) float sm[];
  const int bg = blockIdx.x % (a.B * a.H_kv);
  dkdv_rows<T, D, RM, THREADS>(a, sm, bg / a.H_kv, bg % a.H_kv, (int)(blockIdx.x / (a.B * a.H_kv)) * 16 * RM);
}

template <typename K>
static int set_smem(K kernel, size_t bytes) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) return LAWCAT_OK;
  cudaGetLastError();
  note_cuda_error(e, __FILE__, __LINE__);
  return LAWCAT_ERR_CUDA;
}

// blocks for `rows` rows of n heads in blocks of bm; 0 where the grid would not hold them
static unsigned blocks(long long rows, long long n, int bm) {
  const long long x = (rows + bm - 1) / bm * n;
  return x <= 0x7fffffffLL ? (unsigned)x : 0;
}
// 64 rows per block, or 16 where that leaves more than half of the SMs without a block
static int rows_per_thread(long long rows, long long n) { return (rows + 63) / 64 * n * 2 < sm_count() ? 1 : 4; }

template <typename T, int D, int RM>
static int fwd(const AttnCall& c) {
  const int tiles = (c.a.mask.T + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T, (long long)c.a.B * c.a.H, 16 * RM);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = fwd_smem<D, RM, THREADS>();
  if (int r = set_smem(attn_fwd_exact_kernel<T, D, RM>, sm)) return r;
  LAWCAT_LAUNCH("attn_fwd_exact", c.stream, attn_fwd_exact_kernel<T, D, RM><<<n, THREADS, sm, c.stream>>>(c.a, tiles));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <typename T, int D, int RM>
static int dq(const AttnCall& c) {
  const int tiles = (c.a.mask.T + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T, (long long)c.a.B * c.a.H, 16 * RM);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = dq_smem<D, RM, THREADS>();
  if (int r = set_smem(attn_dq_exact_kernel<T, D, RM>, sm)) return r;
  LAWCAT_LAUNCH("attn_dq_exact", c.stream, attn_dq_exact_kernel<T, D, RM><<<n, THREADS, sm, c.stream>>>(c.a, tiles));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <typename T, int D, int RM>
static int dkdv(const AttnCall& c) {
  const int tiles = (c.a.mask.T_k + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T_k, (long long)c.a.B * c.a.H_kv, 16 * RM);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = dkdv_smem<D, RM, THREADS>();
  if (int r = set_smem(attn_dkdv_exact_kernel<T, D, RM>, sm)) return r;
  LAWCAT_LAUNCH("attn_dkdv_exact", c.stream, attn_dkdv_exact_kernel<T, D, RM><<<n, THREADS, sm, c.stream>>>(c.a, tiles));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <typename F>
static int dispatch(const AttnCall& c, F f) {
  auto width = [&](auto t) {
    switch (c.d) {
      case 16: return f(t, std::integral_constant<int, 16>{});
      case 32: return f(t, std::integral_constant<int, 32>{});
      case 64: return f(t, std::integral_constant<int, 64>{});
      default: return f(t, std::integral_constant<int, 128>{});
    }
  };
  return c.dtype == LAWCAT_F32 ? width(float{}) : width(bf16{});
}

}  // namespace attn

int launch_attn_fwd_exact(const AttnCall& c) {
  return attn::dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return attn::rows_per_thread(c.a.mask.T, (long long)c.a.B * c.a.H) == 1 ? attn::fwd<T, D, 1>(c) : attn::fwd<T, D, 4>(c);
  });
}

int launch_attn_bwd_exact(const AttnCall& c) {
  return attn::dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    int r = LAWCAT_OK;
    if (c.a.mask.T > 0)
      r = attn::rows_per_thread(c.a.mask.T, (long long)c.a.B * c.a.H) == 1 ? attn::dq<T, D, 1>(c) : attn::dq<T, D, 4>(c);
    if (r || c.a.mask.T_k == 0) return r;
    return attn::rows_per_thread(c.a.mask.T_k, (long long)c.a.B * c.a.H_kv) == 1 ? attn::dkdv<T, D, 1>(c) : attn::dkdv<T, D, 4>(c);
  });
}

}  // namespace lawcat

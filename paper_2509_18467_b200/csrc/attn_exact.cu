// Launches of the exact attention kernels (attn_exact.cuh), and the sums of what is shared out over several blocks.
// A block has 256 threads and 64 rows (RM = 4: a tile's loads serve four products), or 16 (RM = 1) in calls of no more. Where the
// blocks would leave SMs idle, each row block's tiles are shared out over several, whose results in fp32 a small kernel joins in a
// fixed order (4 heads x 512 tokens of 64 in fp32, forward and gradients: 32 blocks of 64 rows, or 128 of 16 rows as it was before,
// 163 us).
#include <algorithm>

#include "attn_exact.cuh"

namespace lawcat {
namespace attn {

constexpr int THREADS = 256;

struct Parts {
  int n;
  float *x, *y;   // [n, heads, rows, D]: weighted values; dq; dk and dv
  float2* ml;     // [n, B, H, T] (maximum in log2 units, sum)
};

template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_fwd_exact_kernel(const Args a, int tiles, const Parts p) {
  behind_last_kernel();
  extern __shared__ __align__(16) float sm[];
  const int part = blockIdx.x % p.n, x = blockIdx.x / p.n, bh = x % (a.B * a.H), b = bh / a.H;
  const int t0 = (tiles - 1 - x / (a.B * a.H)) * 16 * RM;  // (under a causal mask the longest rows first)
  if (p.n == 1) {
    fwd_rows<T, D, RM, THREADS>(a, sm, b, bh % a.H, t0, 0, a.mask.T_k, nullptr, nullptr);
    return;
  }
  const int lo = interval(a.mask, b, t0).x, hi = interval(a.mask, b, min(t0 + 16 * RM, a.mask.T) - 1).y;
  const int per = ((hi - lo + BN - 1) / BN + p.n - 1) / p.n * BN;
  const size_t at = ((size_t)part * a.B * a.H + bh) * a.mask.T;
  fwd_rows<T, D, RM, THREADS>(a, sm, b, bh % a.H, t0, lo + part * per, lo + (part + 1) * per, p.x + at * D, p.ml + at);
}

// dq, and (-lse log2e, -dO.o) of every query for the other kernel
template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_dq_exact_kernel(const Args a, int tiles, const Parts p) {
  behind_last_kernel();
  extern __shared__ __align__(16) float sm[];
  const int part = blockIdx.x % p.n, x = blockIdx.x / p.n, bh = x % (a.B * a.H);
  const int t0 = (tiles - 1 - x / (a.B * a.H)) * 16 * RM;
  dq_rows<T, D, RM, THREADS>(a, sm, bh / a.H, bh % a.H, t0, part, p.n, p.x + ((size_t)part * a.B * a.H + bh) * a.mask.T * D);
}

template <typename T, int D, int RM>
__global__ void __launch_bounds__(THREADS) attn_dkdv_exact_kernel(const Args a, int tiles, const Parts p) {
  behind_last_kernel();
  extern __shared__ __align__(16) float sm[];
  const int part = blockIdx.x % p.n, x = blockIdx.x / p.n, bg = x % (a.B * a.H_kv);
  const size_t at = ((size_t)part * a.B * a.H_kv + bg) * a.mask.T_k * D;
  dkdv_rows<T, D, RM, THREADS>(a, sm, bg / a.H_kv, bg % a.H_kv, x / (a.B * a.H_kv) * 16 * RM, part, p.n, p.x + at, p.y + at);
}

// o and lse of every query from its parts; one warp per (batch, token, head)
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_fwd_join_kernel(const Args a, const Parts p) {
  behind_last_kernel();
  const size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) >> 5, rows = (size_t)a.B * a.mask.T * a.H;
  const int lane = threadIdx.x & 31;
  if (row >= rows) return;
  const int h = (int)(row % a.H);
  const size_t bt = row / a.H, b = bt / a.mask.T, t = bt % a.mask.T;
  const size_t at = (b * a.H + h) * a.mask.T + t, step = (size_t)a.B * a.H * a.mask.T;
  constexpr int NC = D / 32 > 0 ? D / 32 : 1;
  const bool mine = lane * NC < D;
  float m = -INFINITY, l = 0.f, acc[NC] = {};
  constexpr int U = 8;
  using V = std::conditional_t<NC == 4, float4, std::conditional_t<NC == 2, float2, float>>;
  for (int i0 = 0; i0 < p.n; i0 += U) {   // (eight parts' loads in flight)
    float2 ml[U];
    alignas(16) float x[U][NC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = i0 + u < p.n;
      ml[u] = there ? p.ml[(i0 + u) * step + at] : make_float2(-INFINITY, 0.f);
      V v{};
      if (there && mine) v = *reinterpret_cast<const V*>(p.x + ((i0 + u) * step + at) * D + lane * NC);
      *reinterpret_cast<V*>(x[u]) = v;
    }
    float n = m;
#pragma unroll
    for (int u = 0; u < U; ++u) n = fmaxf(n, ml[u].x);
    const float base = n == -INFINITY ? 0.f : n, f = exp2f(m - base);
    m = n;
    l *= f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {   // (a part without keys: maximum -infinity, sum and values zero)
      const float w = exp2f(ml[u].x - base);
      l = fmaf(w, ml[u].y, l);
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] = fmaf(w, x[u][c], acc[c]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.o + row * D + lane * NC;
  if (mine)
#pragma unroll
    for (int c = 0; c < NC; ++c) stf<T>(o + c, acc[c] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}

// out [B, rows, heads, D] = the sum of the parts [n, B, heads, rows, D], of x and (gridDim.y = 2) of y; four channels per thread
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_sum_kernel(const Parts p, T* out_x, T* out_y, int B, int heads, int rows) {
  behind_last_kernel();
  const float* const x = blockIdx.y ? p.y : p.x;
  T* const out = blockIdx.y ? out_y : out_x;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, all = (size_t)B * heads * rows * (D / 4);
  if (i >= all) return;
  const int c = (int)(i % (D / 4));
  const size_t r = i / (D / 4), t = r % rows, bh = r / rows;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < p.n; ++k) {
    const float4 v = reinterpret_cast<const float4*>(x)[k * all + i];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  T* o = out + (((bh / heads) * rows + t) * heads + bh % heads) * D + c * 4;
  stf<T>(o, s.x); stf<T>(o + 1, s.y); stf<T>(o + 2, s.z); stf<T>(o + 3, s.w);
}

// blocks for `rows` rows of n heads in blocks of bm; 0 where the grid would not hold them
static unsigned blocks(long long rows, long long n, int bm, int parts) {
  const long long x = (rows + bm - 1) / bm * n * parts;
  return x <= 0x7fffffffLL ? (unsigned)x : 0;
}
static int rows_per_thread(int rows) { return rows <= 16 ? 1 : 4; }
// Parts that a row block's `tiles` tiles are shared out into: as many as give every SM two blocks, four where the blocks differ in length
// and there are fewer than that (1500 tokens, 32/8 heads of 64 in fp32, 192 blocks of keys: the gradients of K and V take 636 + 9 us,
// 888 us with a block each; 4 x 300 tokens, 8 heads: the three kernels within 3 % either way).
// Where all blocks have the same tiles to walk or nearly so (`even`), of up to twice as many the number whose blocks fill the SMs' places
// best in whole rounds (forward and gradients in fp32, 187 queries behind 1313 keys, 32/4 heads of 64: 446 -> 369 us; 1500 tokens without
// a mask, 4 heads of 128: 732 -> 675; 1196 causal ones, whose blocks differ, would go from 266 to 275).
// `resident`: the blocks that an SM holds of the kernel that is launched, asked of the runtime where it matters (in fp32 one of the
// forward and of dQ at width 128 and of dK and dV from width 64 on, else two or more; 2 x 1057 tokens without a mask, 4/2 heads of 128 in
// fp32, forward: four parts for two blocks an SM 190 us, three for one 177).
template <typename F>
static int parts_of(int rows, long long n, long long tiles, F resident, bool even) {
  const long long x = (rows + 63) / 64 * n, sms = sm_count(), most = std::min(tiles, 16LL);
  if (x == 0 || x >= 4 * sms || most < 2) return 1;
  const long long least = std::min(((x < sms ? 2 : 4) * sms + x - 1) / x, most);
  if (!even || least == most) return (int)least;
  const long long places = sms * resident();
  long long best = least;
  auto rounds = [&](long long p) { return (x * p + places - 1) / places; };   // each a p-th of a block's work
  for (long long p = least + 1; p <= std::min(2 * least, most); ++p)
    if (rounds(p) * best * 100 < rounds(best) * p * 95) best = p;
  return (int)best;
}
static bool even(const Mask& m) { return !m.causal || m.off >= m.T; }
// Blocks of a kernel that an SM holds, from its registers and shared memory. Asked once per device, and the first answer stays (1 where
// there is none): the scratch that a call asked for and its launch agree.
template <auto KERNEL>
static int resident(size_t smem) {
  static std::atomic<int> known[64] = {};
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    cudaGetLastError();
    return 1;
  }
  if ((n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
  if (grant_smem<KERNEL>(smem) != LAWCAT_OK || cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, THREADS, smem) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = 1;
  }
  int none = 0;
  return known[dev].compare_exchange_strong(none, n) ? n : none;
}
// parts of a block of queries (its head's keys), and of a block of keys (the queries of its group's heads)
template <typename F>
static int parts_q(const AttnCall& c, F resident) {
  const Mask& m = c.a.mask;
  const long long keys = m.window && m.window < m.T_k ? std::min<long long>(m.T_k, (long long)m.window + 63) : m.T_k;
  return parts_of(m.T, (long long)c.a.B * c.a.H, (keys + 63) / 64, resident, even(m));
}
template <typename F>
static int parts_k(const AttnCall& c, F resident) {
  const Mask& m = c.a.mask;
  const long long queries = m.window && m.window < m.T ? std::min<long long>(m.T, (long long)m.window + 63) : m.T;
  return parts_of(m.T_k, (long long)c.a.B * c.a.H_kv, (queries + 63) / 64 * (c.a.H / c.a.H_kv), resident, even(m));
}
// one part's sums behind another's: forward, queries, keys
static size_t part_bytes(int parts, size_t rows, int d) { return parts == 1 ? 0 : align_up(sizeof(float) * parts * rows * d, 256); }

template <typename T, int D, int RM>
static int fwd(const AttnCall& c, const Parts& p) {
  const int tiles = (c.a.mask.T + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T, (long long)c.a.B * c.a.H, 16 * RM, p.n);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = fwd_smem<D, RM, THREADS>();
  if (int r = grant_smem<attn_fwd_exact_kernel<T, D, RM>>(sm)) return r;
  LAWCAT_LAUNCH("attn_fwd_exact", c.stream, launch_behind(attn_fwd_exact_kernel<T, D, RM>, dim3(n), dim3(THREADS), sm, c.stream, c.a, tiles, p));
  LAWCAT_CHECK_LAUNCH();
  return p.n > 1 ? launch_attn_fwd_join(c, p.n, p.x, p.ml) : (int)LAWCAT_OK;
}

template <typename T, int D>
static int sum(const AttnCall& c, const Parts& p, void* out_x, void* out_y, int heads, int rows) {
  const long long n = ((long long)c.a.B * heads * rows * (D / 4) + 255) / 256;
  LAWCAT_LAUNCH("attn_sum", c.stream,
                launch_behind(attn_sum_kernel<T, D>, dim3((unsigned)n, out_y ? 2 : 1), dim3(256), 0, c.stream, p, (T*)out_x, (T*)out_y, c.a.B, heads, rows));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

template <typename T, int D, int RM>
static int dq(const AttnCall& c, const Parts& p) {
  const int tiles = (c.a.mask.T + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T, (long long)c.a.B * c.a.H, 16 * RM, p.n);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = dq_smem<D, RM, THREADS>();
  if (int r = grant_smem<attn_dq_exact_kernel<T, D, RM>>(sm)) return r;
  LAWCAT_LAUNCH("attn_dq_exact", c.stream, launch_behind(attn_dq_exact_kernel<T, D, RM>, dim3(n), dim3(THREADS), sm, c.stream, c.a, tiles, p));
  LAWCAT_CHECK_LAUNCH();
  return p.n > 1 ? sum<T, D>(c, p, c.a.dq, nullptr, c.a.H, c.a.mask.T) : (int)LAWCAT_OK;
}

template <typename T, int D, int RM>
static int dkdv(const AttnCall& c, const Parts& p) {
  const int tiles = (c.a.mask.T_k + 16 * RM - 1) / (16 * RM);
  const unsigned n = blocks(c.a.mask.T_k, (long long)c.a.B * c.a.H_kv, 16 * RM, p.n);
  if (!n) return LAWCAT_ERR_UNSUPPORTED;
  constexpr size_t sm = dkdv_smem<D, RM, THREADS>();
  if (int r = grant_smem<attn_dkdv_exact_kernel<T, D, RM>>(sm)) return r;
  LAWCAT_LAUNCH("attn_dkdv_exact", c.stream, launch_behind(attn_dkdv_exact_kernel<T, D, RM>, dim3(n), dim3(THREADS), sm, c.stream, c.a, tiles, p));
  LAWCAT_CHECK_LAUNCH();
  return p.n > 1 ? sum<T, D>(c, p, c.a.dk, c.a.dv, c.a.H_kv, c.a.mask.T_k) : (int)LAWCAT_OK;
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

int launch_attn_fwd_join(const AttnCall& c, int parts, const float* part_o, const float2* part_ml) {
  return attn::dispatch(c, [&](auto t, auto d) -> int {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    const attn::Parts p{parts, const_cast<float*>(part_o), nullptr, const_cast<float2*>(part_ml)};
    const size_t n = (size_t)c.a.B * c.a.H * c.a.mask.T;
    LAWCAT_LAUNCH("attn_fwd_join", c.stream, launch_behind(attn::attn_fwd_join_kernel<T, D>, dim3((unsigned)((n + 7) / 8)), dim3(256), 0, c.stream, c.a, p));
    LAWCAT_CHECK_LAUNCH();
    return LAWCAT_OK;
  });
}

namespace attn {
static int parts_fwd(const AttnCall& c) {
  return dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return rows_per_thread(c.a.mask.T) == 1 ? parts_q(c, [] { return resident<attn_fwd_exact_kernel<T, D, 1>>(fwd_smem<D, 1, THREADS>()); })
                                            : parts_q(c, [] { return resident<attn_fwd_exact_kernel<T, D, 4>>(fwd_smem<D, 4, THREADS>()); });
  });
}
static int parts_dq(const AttnCall& c) {
  return dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return rows_per_thread(c.a.mask.T) == 1 ? parts_q(c, [] { return resident<attn_dq_exact_kernel<T, D, 1>>(dq_smem<D, 1, THREADS>()); })
                                            : parts_q(c, [] { return resident<attn_dq_exact_kernel<T, D, 4>>(dq_smem<D, 4, THREADS>()); });
  });
}
static int parts_dkdv(const AttnCall& c) {
  return dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return rows_per_thread(c.a.mask.T_k) == 1 ? parts_k(c, [] { return resident<attn_dkdv_exact_kernel<T, D, 1>>(dkdv_smem<D, 1, THREADS>()); })
                                              : parts_k(c, [] { return resident<attn_dkdv_exact_kernel<T, D, 4>>(dkdv_smem<D, 4, THREADS>()); });
  });
}
}  // namespace attn

size_t attn_fwd_exact_workspace_bytes(const AttnCall& c) {
  const int parts = attn::parts_fwd(c);
  const size_t rows = (size_t)c.a.B * c.a.H * c.a.mask.T;
  return parts == 1 ? 0 : attn::part_bytes(parts, rows, c.d) + align_up(sizeof(float2) * parts * rows, 256);
}

int launch_attn_fwd_exact(const AttnCall& c, void* ws) {
  attn::Parts p{ws ? attn::parts_fwd(c) : 1, (float*)ws, nullptr, nullptr};
  if (p.n > 1) p.ml = (float2*)((char*)ws + attn::part_bytes(p.n, (size_t)c.a.B * c.a.H * c.a.mask.T, c.d));
  return attn::dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return attn::rows_per_thread(c.a.mask.T) == 1 ? attn::fwd<T, D, 1>(c, p) : attn::fwd<T, D, 4>(c, p);
  });
}

size_t attn_bwd_exact_workspace_bytes(const AttnCall& c) {
  const size_t q = attn::part_bytes(attn::parts_dq(c), (size_t)c.a.B * c.a.H * c.a.mask.T, c.d);
  const size_t k = attn::part_bytes(attn::parts_dkdv(c), (size_t)c.a.B * c.a.H_kv * c.a.mask.T_k, c.d);
  return std::max(q, 2 * k);
}

int launch_attn_bwd_exact(const AttnCall& c, void* ws) {
  const attn::Parts pq{ws ? attn::parts_dq(c) : 1, (float*)ws, nullptr, nullptr};
  attn::Parts pk{ws ? attn::parts_dkdv(c) : 1, (float*)ws, nullptr, nullptr};
  if (pk.n > 1) pk.y = (float*)((char*)ws + attn::part_bytes(pk.n, (size_t)c.a.B * c.a.H_kv * c.a.mask.T_k, c.d));
  return attn::dispatch(c, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    int r = LAWCAT_OK;
    if (c.a.mask.T > 0) r = attn::rows_per_thread(c.a.mask.T) == 1 ? attn::dq<T, D, 1>(c, pq) : attn::dq<T, D, 4>(c, pq);
    if (r || c.a.mask.T_k == 0) return r;
    return attn::rows_per_thread(c.a.mask.T_k) == 1 ? attn::dkdv<T, D, 1>(c, pk) : attn::dkdv<T, D, 4>(c, pk);
  });
}

}  // namespace lawcat

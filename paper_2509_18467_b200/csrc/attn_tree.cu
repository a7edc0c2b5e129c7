// Attention of drafted tokens over a cache, and accepted tokens into it: entry points, the CUDA-core kernels, the join of parts.
//
// The general kernel: a block takes 32 rows of one (sequence, key-value head) and a part of the keys, walks them in tiles of 64 that it
// widens to fp32 in shared memory, and keeps the running maximum and sum of each row (four rows to a warp: a key or value that is read from
// shared memory serves four). The keys are cut into as many parts as fill the SMs, by the capacity alone, so that a captured step may be
// replayed at every length; a second kernel joins them. For small calls latency is all of it (2 sequences of 500 tokens, 13 nodes, 4 heads of 64 in
// fp32: 10.7 us, both launches); over long caches fp32 products from shared memory (16 sequences of 8190 tokens, 20 rows, 8/2 heads of 128, exact: 262 us,
// over 4 bits 217; the tensor cores take 40 and 32).
//
// Rows of one tile see different keys of it, and a weight of zero times a value that is not finite is a NaN: a row that comes out not finite
// is computed again by itself, from the keys that it sees and nothing else.
#include <algorithm>
#include <cmath>

#include "attn_tree.cuh"

namespace lawcat {
namespace attn {

constexpr int TREE_ROWS = 32, TREE_KEYS = 64, TREE_THREADS = 256, TREE_RW = 4;   // rows and keys of a tile; rows of a warp

template <int D>
struct TreeLay {
  static constexpr int LD = D + 4;
  static constexpr size_t OFF_V = (size_t)TREE_KEYS * LD, OFF_Q = OFF_V + (size_t)TREE_KEYS * LD, OFF_P = OFF_Q + (size_t)TREE_ROWS * LD;
  static constexpr size_t OFF_PATHS = OFF_P + (size_t)TREE_KEYS * TREE_ROWS, FLOATS = OFF_PATHS + sizeof(Paths) / 4;
};

// T: storage type of the step's own tensors; QUANT: the cache holds 4-bit codes
template <typename T, int D, bool QUANT>
__global__ void __launch_bounds__(TREE_THREADS) attn_tree_kernel(const __grid_constant__ TreeArgs a) {
  using L = TreeLay<D>;
  constexpr int LD = L::LD, V8 = D / 8, NC = D / 32 > 0 ? D / 32 : 1, RW = TREE_RW, TK = TREE_KEYS;
  extern __shared__ __align__(16) float sm[];
  float *const K = sm, *const V = sm + L::OFF_V, *const Q = sm + L::OFF_Q, *const P = sm + L::OFF_P;   // P: [warp][key][RW]
  Paths& paths = *reinterpret_cast<Paths*>(sm + L::OFF_PATHS);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.H / a.H_kv, R = a.N * G, row_blocks = (R + TREE_ROWS - 1) / TREE_ROWS;
  const int part = blockIdx.x % a.parts, rb = blockIdx.x / a.parts % row_blocks, bg = blockIdx.x / a.parts / row_blocks;
  const int b = bg / a.H_kv, g = bg % a.H_kv, r0 = rb * TREE_ROWS;
  behind_last_kernel();
  const int pos = a.pos[b];
  find_paths<TREE_THREADS>(a, b, paths, tid, 1);
  auto row_at = [&](int r) { return ((size_t)b * a.N + r / G) * a.H + g * G + r % G; };   // of [B, N, H]
  // keys: the nodes' own up to the last one of these rows, then the cached ones from the newest on; tiles of 64, each of one kind
  const int nodes = pos < 0 ? 0 : min(a.N, (r0 + TREE_ROWS - 1) / G + 1), cached = cached_keys(pos, a.W);
  const int node_tiles = (nodes + TK - 1) / TK, tiles = node_tiles + (cached + TK - 1) / TK;
  const int per = (tiles + a.parts - 1) / a.parts, i0 = min(tiles, part * per), i1 = min(tiles, i0 + per);
#pragma unroll 2
  for (int i = tid; i < TREE_ROWS * V8; i += TREE_THREADS) {
    const int r = i / V8, c0 = i % V8 * 8;
    float x[8] = {};
    if (r0 + r < R) load8((const T*)a.q + row_at(r0 + r) * D + c0, x);
#pragma unroll
    for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4*>(Q + r * LD + c0 + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
  }
  int depth[RW];
  float slope[RW], m[RW], l[RW], acc[RW][NC];
#pragma unroll
  for (int j = 0; j < RW; ++j) {
    const int r = min(r0 + warp * RW + j, R - 1);
    depth[j] = node_depth(paths, r / G, a.N);
    if (pos < 0) depth[j] = -1;
    slope[j] = a.slopes ? a.slopes[g * G + r % G] : 0.f;
    m[j] = -INFINITY;
    l[j] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[j][c] = 0.f;
  }
  const int ps = pos < 0 ? 0 : pos % a.C;
  const bool none = r0 + warp * RW >= R;   // (a warp without rows leaves shared memory to the others)

  for (int t = i0; t < i1; ++t) {
    const bool fresh = t < node_tiles;
    const int k0 = (fresh ? t : t - node_tiles) * TK, keys = min(TK, (fresh ? nodes : cached) - k0);
    __syncthreads();
    for (int i = tid; i < TK * V8; i += TREE_THREADS) {
      const int r = i / V8, c0 = i % V8 * 8, k = k0 + r;
      float x[8] = {}, y[8] = {};
      if (fresh) {
        const size_t src = (((size_t)b * a.N + min(k, a.N - 1)) * a.H_kv + g) * D + c0;
        const bool there = r < keys && paths.on[min(k, a.N - 1)][min(k, a.N - 1) / 32] != 0u;   // (whatever the others hold stays out)
        if (there) {
          load8((const T*)a.k_t + src, x);
          load8((const T*)a.v_t + src, y);
        }
        if constexpr (QUANT) {   // (all lanes together: a row's groups may lie in one warp with another row's)
          quantize8<D, sizeof(T) == 2>(x, c0, nullptr, nullptr, false, 0xffffffffu);
          quantize8<D, sizeof(T) == 2>(y, c0, nullptr, nullptr, false, 0xffffffffu);
        }
      } else if (r < keys) {
        const int back = k + 1;
        size_t slot = ps >= back ? ps - back : ps - back + a.C;
        if constexpr (QUANT) {
          constexpr int NG = D / quant_group(D);
          const size_t row = ((size_t)b * a.H_kv + g) * a.C + slot;
          widen8(codes8<D>(a.kq + row * (D / 2), a.kp + row * (2 * NG), c0), x);
          widen8(codes8<D>(a.vq + row * (D / 2), a.vp + row * (2 * NG), c0), y);
        } else {
          const size_t row = (((size_t)b * a.C + slot) * a.H_kv + g) * D + c0;
          load8((const T*)a.K + row, x);
          load8((const T*)a.V + row, y);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        *reinterpret_cast<float4*>(K + r * LD + c0 + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
        *reinterpret_cast<float4*>(V + r * LD + c0 + j) = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
      }
    }
    __syncthreads();
    if (none) continue;
    float s[RW][2] = {};
    const float* const Qw = Q + warp * RW * LD;
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      const float4 ka = *reinterpret_cast<const float4*>(K + lane * LD + c), kb = *reinterpret_cast<const float4*>(K + (lane + 32) * LD + c);
#pragma unroll
      for (int j = 0; j < RW; ++j) {
        const float4 x = *reinterpret_cast<const float4*>(Qw + j * LD + c);
        s[j][0] = fmaf(x.w, ka.w, fmaf(x.z, ka.z, fmaf(x.y, ka.y, fmaf(x.x, ka.x, s[j][0]))));
        s[j][1] = fmaf(x.w, kb.w, fmaf(x.z, kb.z, fmaf(x.y, kb.y, fmaf(x.x, kb.x, s[j][1]))));
      }
    }
#pragma unroll
    for (int j = 0; j < RW; ++j) {
      const int node = min(r0 + warp * RW + j, R - 1) / G;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = lane + 32 * u, k = k0 + r;
        bool see = r < keys && depth[j] >= 0;
        int dist = k + 1 + depth[j];
        if (fresh) {
          const int kk = min(k, a.N - 1);
          see = see && (paths.on[node][kk >> 5] >> (kk & 31) & 1u);
          dist = see ? depth[j] - node_depth(paths, kk, a.N) : 0;
        }
        s[j][u] = see && dist < a.W ? tree_score(a, s[j][u], slope[j], dist) : -INFINITY;
      }
      const float mx = fmaxf(m[j], warp_max(fmaxf(s[j][0], s[j][1]))), base = mx == -INFINITY ? 0.f : mx, f = exp2f(m[j] - base);
      m[j] = mx;
      s[j][0] = exp2f(s[j][0] - base);
      s[j][1] = exp2f(s[j][1] - base);
      l[j] = l[j] * f + warp_sum(s[j][0] + s[j][1]);
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[j][c] *= f;
    }
    float4* const Pw = reinterpret_cast<float4*>(P) + warp * TK;
#pragma unroll
    for (int u = 0; u < 2; ++u) Pw[lane + 32 * u] = make_float4(s[0][u], s[1][u], s[2][u], s[3][u]);
    __syncwarp();
#pragma unroll 4
    for (int r = 0; r < keys; ++r) {
      const float4 w = Pw[r];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float y = V[r * LD + (D >= 32 ? lane + 32 * c : lane % D)];
        acc[0][c] = fmaf(w.x, y, acc[0][c]);
        acc[1][c] = fmaf(w.y, y, acc[1][c]);
        acc[2][c] = fmaf(w.z, y, acc[2][c]);
        acc[3][c] = fmaf(w.w, y, acc[3][c]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < RW; ++j) {
    const int r = r0 + warp * RW + j;
    if (r >= R) continue;
    const size_t row = row_at(r);
    if (a.parts == 1) {
      const float inv = l[j] == 0.f ? 0.f : 1.f / l[j];
      bool fine = true;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const float o = l[j] == 0.f ? 0.f * acc[j][c] : acc[j][c] * inv;   // (a row that sees nothing: 0, or NaN from another row's)
        fine = fine && isfinite(o);
        if (lane + 32 * c < D) stf<T>((T*)a.o + row * D + lane + 32 * c, o);
      }
      if (!__all_sync(0xffffffffu, fine)) tree_row_again<T, D, QUANT>(a, b, r / G, g * G + r % G);
    } else {
      float* const w = a.part + (row * a.parts + part) * (D + 2);
      if (lane == 0) {
        w[0] = m[j];
        w[1] = l[j];
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (lane + 32 * c < D) w[2 + lane + 32 * c] = acc[j][c];
    }
  }
}

// The parts of a row: W warps share them out, each at the maximum of its own, four parts' loads in flight; then the warps' sums at the
// common maximum.
template <typename T, int D, bool QUANT, int W>
__global__ void __launch_bounds__(32 * W) attn_tree_join_kernel(const __grid_constant__ TreeArgs a) {
  constexpr int NC = D / 32 > 0 ? D / 32 : 1, U = 4;
  __shared__ float s_acc[W][D], s_ml[W][2];
  const size_t row = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  behind_last_kernel();
  const float* w = a.part + row * a.parts * (D + 2);
  float m = -INFINITY, l = 0.f, acc[NC] = {};
  for (int i0 = warp; i0 < a.parts; i0 += U * W) {
    float pm[U], pl[U], x[U][NC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * W;
      const float* p = w + (size_t)i * (D + 2);
      pm[u] = i < a.parts ? p[0] : -INFINITY;
      pl[u] = i < a.parts ? p[1] : 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) x[u][c] = i < a.parts && lane + 32 * c < D ? p[2 + lane + 32 * c] : 0.f;
    }
    float n = m;
#pragma unroll
    for (int u = 0; u < U; ++u) n = fmaxf(n, pm[u]);
    const float base = n == -INFINITY ? 0.f : n, f = exp2f(m - base);
    m = n;
    l *= f;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool some = pl[u] != 0.f;               // (a part without keys has no weights)
      const float g = exp2f(pm[u] - base);
      l += some ? g * pl[u] : 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[c] += some ? g * x[u][c] : 0.f;
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (lane + 32 * c < D) s_acc[warp][lane + 32 * c] = acc[c];
  if (lane == 0) {
    s_ml[warp][0] = m;
    s_ml[warp][1] = l;
  }
  __syncthreads();
  const float top = warp_max(lane < W ? s_ml[lane][0] : -INFINITY), base = top == -INFINITY ? 0.f : top;
  const float f = lane < W ? exp2f(s_ml[lane][0] - base) : 0.f, sum = warp_sum(lane < W ? f * s_ml[lane][1] : 0.f);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  bool fine = true;
  for (int c = threadIdx.x; c < (D < 32 ? 32 : D); c += 32 * W) {
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) o = fmaf(__shfl_sync(0xffffffffu, f, i), s_acc[i][c < D ? c : 0], o);
    o *= inv;
    fine = fine && isfinite(o);
    if (c < D) stf<T>((T*)a.o + row * D + c, o);
  }
  if (__syncthreads_or(!fine) && warp == 0) tree_row_again<T, D, QUANT>(a, (int)(row / ((size_t)a.N * a.H)), (int)(row / a.H % a.N), (int)(row % a.H));
}

// Parts of the keys: as many as give each SM two blocks, and no more than there are tiles (one sequence, 1468 tokens, 1 node,
// 4 heads of 128 in fp32: 20.4 us with one part less, whose blocks have two tiles, and no warp idle; 11.4).
static int tree_parts(const AttnTree& c) {
  const attn::TreeArgs& a = c.a;
  const long long rows = (long long)a.N * (a.H / a.H_kv), n = (long long)a.B * a.H_kv * ((rows + TREE_ROWS - 1) / TREE_ROWS);
  const int most = (a.N + TREE_KEYS - 1) / TREE_KEYS + (std::min(a.W, a.C) - 1 + TREE_KEYS - 1) / TREE_KEYS;
  const long long want = (2LL * sm_count() + n - 1) / (n > 0 ? n : 1);
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

// --------------------------------------------------------------------------------------------------------------- accepted tokens
struct AcceptArgs {
  const void *k, *v;          // [B, T, H_kv, D]
  const int *pos, *path;      // [B], [B, M] or null
  int* pos_out;
  void *K, *V;                // [B, C, H_kv, D]
  uint8_t *kq, *vq;
  bf16 *kp, *vp;
  int T, M, H_kv, C, chunks;  // M: entries of a path, or T
  int row;                    // pieces of a row: 16 bytes, or eight channels in the 4-bit form
};
constexpr int ACCEPT_THREADS = 256, ACCEPT_PIECES = 4;   // pieces of a thread

// A block has 1024 pieces of one sequence's accepted rows of k (blockIdx.y = 0) or v: copies, bound by the launch where paths are short (64
// sequences, paths of up to 8 rows of 8 heads of 128: 6.8 us with the host's call).
template <typename T, int D, bool QUANT>
__global__ void __launch_bounds__(ACCEPT_THREADS) cache_accept_kernel(const AcceptArgs a) {
  const int b = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks, tid = threadIdx.x;
  const bool is_v = blockIdx.y;
  behind_last_kernel();
  const int pos = a.pos[b];
  int rows = a.M;
  __shared__ int s_first;
  if (a.path) {   // the entries in front of the first that is no row
    if (tid == 0) s_first = a.M;
    __syncthreads();
    for (int i = tid; i < a.M; i += ACCEPT_THREADS)
      if ((unsigned)a.path[(size_t)b * a.M + i] >= (unsigned)a.T) atomicMin(&s_first, i);
    __syncthreads();
    rows = s_first;
  }
  if (pos < 0) rows = 0;
  if (a.pos_out && chunk == 0 && !is_v && tid == 0) a.pos_out[b] = (int)min((long long)pos + rows, 0x7fffffffLL);
  const int ps = pos < 0 ? 0 : pos % a.C;
  // (of more rows than slots the last stay)
  const long long first = (long long)max(0, rows - a.C) * a.row, last = (long long)rows * a.row;
  for (int u = 0; u < ACCEPT_PIECES; ++u) {
    const long long i = first + ((long long)chunk * ACCEPT_PIECES + u) * ACCEPT_THREADS + tid;
    if (i - tid >= last) break;                    // (the same for the block)
    const bool some = i < last;
    const int t = some ? (int)(i / a.row) : rows - 1, e = some ? (int)(i % a.row) : tid % a.row;
    const size_t from = (size_t)b * a.T + (a.path ? a.path[(size_t)b * a.M + t] : t);
    const size_t slot = ((long long)ps + t) % a.C;
    if constexpr (QUANT) {
      constexpr int V8 = D / 8, NG = D / quant_group(D);
      const int g = e / V8, c0 = e % V8 * 8;
      const size_t row = ((size_t)b * a.H_kv + g) * a.C + slot;
      float x[8];
      load8((const T*)(is_v ? a.v : a.k) + (from * a.H_kv + g) * D + c0, x);
      quantize8<D, sizeof(T) == 2>(x, c0, (is_v ? a.vq : a.kq) + row * (D / 2), (is_v ? a.vp : a.kp) + row * (2 * NG), some, 0xffffffffu);
    } else if (some) {
      reinterpret_cast<uint4*>(is_v ? a.V : a.K)[((size_t)b * a.C + slot) * a.row + e] = reinterpret_cast<const uint4*>(is_v ? a.v : a.k)[from * a.row + e];
    }
  }
}

}  // namespace attn

namespace {

template <typename F>
int by_width(int d, F f) {
  switch (d) {
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    default: return f(std::integral_constant<int, 128>{});
  }
}
template <typename F>
int by_form(int d, int dtype, bool quant, F f) {   // f(width, value of the storage type, whether the cache is in 4 bits)
  return by_width(d, [&](auto dd) {
    if (dtype == LAWCAT_F32) return quant ? f(dd, float{}, std::true_type{}) : f(dd, float{}, std::false_type{});
    return quant ? f(dd, bf16{}, std::true_type{}) : f(dd, bf16{}, std::false_type{});
  });
}

size_t part_bytes(const AttnTree& c, int parts) { return parts == 1 ? 0 : align_up(sizeof(float) * (size_t)c.a.B * c.a.N * c.a.H * parts * (c.d + 2), 256); }

int launch_tree_exact(const AttnTree& c) {
  attn::TreeArgs a = c.a;
  a.parts = attn::tree_parts(c);
  a.part = (float*)c.ws;
  const long long rows = (long long)a.N * (a.H / a.H_kv);
  const long long blocks = (long long)a.B * a.H_kv * ((rows + attn::TREE_ROWS - 1) / attn::TREE_ROWS) * a.parts;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  return by_form(c.d, c.dtype, a.kq != nullptr, [&](auto dd, auto t, auto quant) -> int {
    constexpr int D = decltype(dd)::value;
    using T = decltype(t);
    constexpr auto kernel = attn::attn_tree_kernel<T, D, decltype(quant)::value>;
    constexpr size_t sm = sizeof(float) * attn::TreeLay<D>::FLOATS;
    if (int r = grant_smem<kernel>(sm)) return r;
    LAWCAT_LAUNCH("attn_tree", c.stream, launch_behind(kernel, dim3((unsigned)blocks), dim3(attn::TREE_THREADS), sm, c.stream, a));
    LAWCAT_CHECK_LAUNCH();
    if (a.parts == 1) return (int)LAWCAT_OK;
    AttnTree j = c;
    j.a = a;
    return launch_attn_tree_join(j);
  });
}

// (a node's rows are one box of a tile: 128 query heads to a key-value head at most)
bool tree_tc_supported(const AttnTree& c) { return attn_tc_supported(c.dtype, c.d, c.exact) && c.a.H / c.a.H_kv <= 128; }

int tree_check(const lawcat_attn_params* p) {
  int r = attn_check(p);
  if (r || (r = attn_check_cache(p))) return r;
  if (p->T > attn::TREE_MAX) return LAWCAT_ERR_UNSUPPORTED;
  if ((long long)p->B * p->T * p->H > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  return LAWCAT_OK;
}

AttnTree make_tree(const lawcat_attn_params* p) {
  AttnTree c{};
  c.a.B = p->B; c.a.N = p->T; c.a.H = p->H; c.a.H_kv = p->H_kv; c.a.C = p->T_k;
  c.a.W = p->window ? p->window : p->T_k;
  c.a.scale = p->scale; c.a.cap = p->cap;
  c.d = p->d; c.dtype = p->dtype; c.exact = p->exact;
  return c;
}

bool aligned(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; }

int tree(const lawcat_attn_params* p, AttnTree& c, const void* const (&req)[8], const void* opt, size_t ws_bytes) {
  for (const void* x : req)
    if (!x || !aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  for (const void* x : {opt, (const void*)c.a.parent, (const void*)c.a.slopes, (const void*)c.ws})
    if (!aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  const size_t need = lawcat_attn_workspace_bytes(p, LAWCAT_OP_ATTN_TREE);
  if (need && (!c.ws || ws_bytes < need)) return LAWCAT_ERR_WORKSPACE_TOO_SMALL;
  if (!tree_tc_supported(c)) return launch_tree_exact(c);
  return c.a.kq ? launch_attn_tree_quant_tc(c) : launch_attn_tree_tc(c);
}

template <bool QUANT>
int accept(const lawcat_attn_params* p, int M, attn::AcceptArgs a, void* stream) {
  int r = attn_check(p);
  if (r || (r = attn_check_cache(p))) return r;
  if (M < 0) return LAWCAT_ERR_INVALID_ARG;
  if (!a.path) M = p->T;
  if (p->B == 0) return LAWCAT_OK;
  if (!a.pos || a.pos == a.pos_out) return LAWCAT_ERR_INVALID_ARG;
  const bool none = p->T == 0 || M == 0;   // (nothing to take: pos goes out as it came)
  for (const void* x : {a.k, a.v, (const void*)(QUANT ? a.kq : a.K), (const void*)(QUANT ? a.vq : a.V), QUANT ? (const void*)a.kp : a.K, QUANT ? (const void*)a.vp : a.V})
    if ((!x && !none) || !aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  for (const void* x : {(const void*)a.pos, (const void*)a.path, (const void*)a.pos_out})
    if (!aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  if (none && !a.pos_out) return LAWCAT_OK;
  const int es = p->dtype == LAWCAT_F32 ? 4 : 2;
  a.T = p->T; a.M = M; a.H_kv = p->H_kv; a.C = p->T_k;
  a.row = QUANT ? p->H_kv * p->d / 8 : (int)((long long)p->H_kv * p->d * es / 16);
  const long long pieces = (long long)std::min(M, p->T_k) * a.row, per = (long long)attn::ACCEPT_THREADS * attn::ACCEPT_PIECES;
  const long long chunks = std::max(1LL, (pieces + per - 1) / per), blocks = chunks * p->B;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  a.chunks = (int)chunks;
  cudaStream_t s = (cudaStream_t)stream;
  const dim3 grid((unsigned)blocks, 2);
  auto go = [&](auto dd, auto t, auto) -> int {
    LAWCAT_LAUNCH("cache_accept", s, launch_behind(attn::cache_accept_kernel<decltype(t), decltype(dd)::value, QUANT>, grid, dim3(attn::ACCEPT_THREADS), 0, s, a));
    LAWCAT_CHECK_LAUNCH();
    return LAWCAT_OK;
  };
  if constexpr (QUANT) return by_form(p->d, p->dtype, true, go);
  else return go(std::integral_constant<int, 16>{}, bf16{}, 0);   // (pieces of 16 bytes, whatever they hold)
}

}  // namespace

int launch_attn_tree_join(const AttnTree& c) {
  return by_form(c.d, c.dtype, c.a.kq != nullptr, [&](auto dd, auto t, auto quant) -> int {
    constexpr int D = decltype(dd)::value;
    using T = decltype(t);
    constexpr bool Q = decltype(quant)::value;
    const dim3 grid((unsigned)((size_t)c.a.B * c.a.N * c.a.H));
    if (c.a.parts > 16) LAWCAT_LAUNCH("attn_tree_join", c.stream, launch_behind(attn::attn_tree_join_kernel<T, D, Q, 16>, grid, dim3(512), 0, c.stream, c.a));
    else LAWCAT_LAUNCH("attn_tree_join", c.stream, launch_behind(attn::attn_tree_join_kernel<T, D, Q, 4>, grid, dim3(128), 0, c.stream, c.a));
    LAWCAT_CHECK_LAUNCH();
    return LAWCAT_OK;
  });
}

size_t attn_tree_workspace_bytes(const lawcat_attn_params* p) {
  if (tree_check(p) != LAWCAT_OK) return 0;
  const AttnTree c = make_tree(p);
  if (c.a.B == 0 || c.a.N == 0) return 0;
  if (tree_tc_supported(c)) return std::max(attn_tree_tc_workspace_bytes(c), attn_tree_quant_tc_workspace_bytes(c));
  return part_bytes(c, attn::tree_parts(c));
}

}  // namespace lawcat

using namespace lawcat;

extern "C" {

int lawcat_attn_tree(const lawcat_attn_params* p, const void* q_t, const void* k_t, const void* v_t, const void* K, const void* V,
                     const int32_t* pos, const int32_t* parent, const float* slopes, void* o_t, void* ws, size_t ws_bytes, void* stream,
                     int* dev_status) {
  if (int r = tree_check(p)) return r;
  if (p->B == 0 || p->T == 0) return LAWCAT_OK;
  AttnTree c = make_tree(p);
  c.a.q = q_t; c.a.k_t = k_t; c.a.v_t = v_t; c.a.K = K; c.a.V = V;
  c.a.pos = pos; c.a.parent = parent; c.a.slopes = slopes; c.a.o = o_t;
  c.ws = ws; c.dev_status = dev_status; c.stream = (cudaStream_t)stream;
  return tree(p, c, {q_t, k_t, v_t, K, V, pos, o_t, o_t}, nullptr, ws_bytes);
}

int lawcat_attn_tree_quant(const lawcat_attn_params* p, const void* q_t, const void* k_t, const void* v_t, const void* kq, const void* kp,
                           const void* vq, const void* vp, const int32_t* pos, const int32_t* parent, const float* slopes, void* o_t, void* ws,
                           size_t ws_bytes, void* stream, int* dev_status) {
  if (int r = tree_check(p)) return r;
  if (p->B == 0 || p->T == 0) return LAWCAT_OK;
  AttnTree c = make_tree(p);
  c.a.q = q_t; c.a.k_t = k_t; c.a.v_t = v_t;
  c.a.kq = (const uint8_t*)kq; c.a.kp = (const bf16*)kp; c.a.vq = (const uint8_t*)vq; c.a.vp = (const bf16*)vp;
  c.a.pos = pos; c.a.parent = parent; c.a.slopes = slopes; c.a.o = o_t;
  c.ws = ws; c.dev_status = dev_status; c.stream = (cudaStream_t)stream;
  if (!o_t) return LAWCAT_ERR_INVALID_ARG;
  return tree(p, c, {q_t, k_t, v_t, kq, kp, vq, vp, pos}, o_t, ws_bytes);
}

int lawcat_cache_accept(const lawcat_attn_params* p, int32_t M, const void* k_t, const void* v_t, const int32_t* pos, const int32_t* path, void* K,
                        void* V, int32_t* pos_out, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  attn::AcceptArgs a{};
  a.k = k_t; a.v = v_t; a.pos = pos; a.path = path; a.pos_out = pos_out;
  a.K = K; a.V = V;
  return accept<false>(p, M, a, stream);
}

int lawcat_cache_accept_quant(const lawcat_attn_params* p, int32_t M, const void* k_t, const void* v_t, const int32_t* pos, const int32_t* path,
                              void* kq, void* kp, void* vq, void* vp, int32_t* pos_out, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  attn::AcceptArgs a{};
  a.k = k_t; a.v = v_t; a.pos = pos; a.path = path; a.pos_out = pos_out;
  a.kq = (uint8_t*)kq; a.kp = (bf16*)kp; a.vq = (uint8_t*)vq; a.vp = (bf16*)vp;
  return accept<true>(p, M, a, stream);
}

}  // extern "C"

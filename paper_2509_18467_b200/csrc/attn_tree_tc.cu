// Attention of drafted tokens over a cache on the tensor cores: bf16 storage, d = 64 or 128; the cache in the storage type or in 4 bits.
//
// A block takes up to 256 rows (node, query head) of one (sequence, key-value head) and a part of the keys, in tiles of 64:
//   two warpgroups    softmax, one thread per row: S from tensor memory, masks, running maximum and sum in registers, P = exp2(x - m) over S
//   copy warp         K and V tiles through a ring of stages by TMA; over 4 bits a warpgroup in its place, which unpacks codes into the stages
//   product warp      S = Q K^T (shared memory), O += P V (P from tensor memory); fp32 accumulation
// Of more than 128 rows each warpgroup has a tile of 128, and both meet every key; of fewer, both have the same rows and take the key tiles in
// turn, each with sums of its own that meet at the end. S has two places per warpgroup; O is rescaled only when a maximum grew by more than
// 2^8.
//
// The keys are walked from the newest to the oldest: the nodes' own rows first (loaded by all threads; rows of nodes that are not there are
// zeros), then the cached ones, whose tiles end where the newest slot, or slot C - 1, does. What a tile holds below its oldest key are slots
// in front of slot 0, which read as zeros, or older tokens: never a slot without a token. So a row sees a tile's columns from one limit on.
//
// Over 4 bits all operands are fp16: a code becomes 1024 + code by an OR into the mantissa, less 1024, times scale, plus minimum (all times 16),
// one rounding of 2^-11; queries are scaled by a power of two per row. Values beyond 4094 leave fp16's range, and outputs below 2^-18 feel the
// smallest numbers that it holds: such rows, like all that come out not finite, are computed again on the CUDA cores. Channels of eight
// are held in the order 0 4 1 5 2 6 3 7, in which a word of codes unpacks two at a time.
//
// Rounding: weights to bf16 (fp16) as an operand, o once; all else fp32.
#include <algorithm>

#include "attn_tree.cuh"

namespace lawcat {
namespace attn {

constexpr float TREE_RESCALE = 8.f;
constexpr int PREFETCH = 3;        // tiles of codes on their way

struct TreePlan {
  int row_blocks, two;   // blocks of up to 256 rows; whether a block has two tiles of rows
  int parts;
};

struct TreeTcArgs {
  TreeArgs a;
  int row_blocks, two, rows_pad;   // rows_pad: the group's rows as the parts' scratch has them
  float2* part_ml;                 // [B H_kv, parts, rows_pad] (maximum in log2 units, sum) where parts > 1
  float* part_o;                   // [B H_kv, parts, D, rows_pad]
  long long limit;
  int* dev_status;
};

template <int D, bool QUANT>
struct TreeTc {
  static constexpr uint32_t TILE = 128 * D * 2, KT = 64 * D * 2;   // rows' queries; keys or values of a tile
  static constexpr int ST = D == 64 ? 16 : 8;                      // stages, K and V tiles in turn
  static constexpr uint32_t OFF_RING = 2 * TILE, OFF_PATHS = OFF_RING + ST * KT, OFF_DEPTH = OFF_PATHS + sizeof(Paths), OFF_SCALE = OFF_DEPTH + TREE_MAX * 4;
  static constexpr uint32_t OFF_ML = OFF_SCALE + 256 * 4, OFF_BAR = OFF_ML + 128 * 8, BYTES = OFF_BAR + 512;
  static constexpr int LOADERS = QUANT ? 128 : 32, THREADS = 256 + LOADERS + 32;
  static constexpr int B_FULL = 0, B_EMPTY = ST, B_S = 2 * ST, B_P = B_S + 4, B_O = B_P + 4, B_DONE = B_O + 4, NBAR = B_DONE + 1;
  static constexpr int FMT = QUANT ? FMT_F16 : FMT_BF16;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 512 && 256 + 2 * D <= 512 && 128 * D * 4 <= ST * KT, "shared memory, tensor memory");
};

// Cached tile j of a sequence: its slots are s0 ... s0 + 63, slot s0 + c lies `back0 - c` in front of pos, and slots below `lo` are none.
struct CachedTile {
  int s0, back0, lo;
};
struct Ring {
  int cached, near, near_tiles, tiles, ps;   // keys; those up to slot ps - 1, in tiles; all tiles
};
__device__ __forceinline__ Ring ring_of(int pos, int C, int W) {
  Ring r;
  r.cached = cached_keys(pos, W);
  r.ps = pos < 0 ? 0 : pos % C;
  r.near = min(r.cached, r.ps);
  r.near_tiles = (r.near + 63) / 64;
  r.tiles = r.near_tiles + (r.cached - r.near + 63) / 64;
  return r;
}
__device__ __forceinline__ CachedTile cached_tile(const Ring& r, int j, int C) {
  CachedTile t;
  if (j < r.near_tiles) {
    t.s0 = r.ps - 64 * (j + 1);
    t.back0 = 64 * (j + 1);
    t.lo = t.s0 < 0 ? -t.s0 : 0;
  } else {
    j -= r.near_tiles;
    t.s0 = C - 64 * (j + 1);
    t.back0 = r.near + 64 * (j + 1);
    t.lo = 0;   // (slots below 0 lie C or more behind, which no row sees)
  }
  return t;
}

// eight channels as halves in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ uint4 halves_in_order(const float (&x)[8]) {
  return make_uint4(pack_f16(x[0], x[4]), pack_f16(x[1], x[5]), pack_f16(x[2], x[6]), pack_f16(x[3], x[7]));
}
constexpr float V_FACTOR = 16.f;                    // (of keys and values over 4 bits)
constexpr float SMALL = 1.f / (1 << 18);            // (the least difference of fp16 numbers, 2^-24 / 16, is 2^-10 of it)

__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
struct GroupScale {
  __half2 s1, s16, low;   // scale, scale / 16, minimum
};
__device__ __forceinline__ GroupScale group_scale(uint32_t pair) {   // (scale, minimum) in bf16
  const float s = bf16_lo(pair) * V_FACTOR, l = bf16_hi(pair) * V_FACTOR;
  return GroupScale{__floats2half2_rn(s, s), __floats2half2_rn(s * 0.0625f, s * 0.0625f), __floats2half2_rn(l, l)};
}
// a word of eight codes -> eight values in the order above
__device__ __forceinline__ uint4 unpack8(uint32_t w, const GroupScale& g) {
  const __half2 k = as_half2(0x64006400u);   // 1024
  const uint32_t hi = w >> 8;
  auto val = [&](uint32_t bits, __half2 s) { return as_word(__hfma2(__hsub2(as_half2(bits | 0x64006400u), k), s, g.low)); };
  return make_uint4(val(w & 0x000F000Fu, g.s1), val(w & 0x00F000F0u, g.s16), val(hi & 0x000F000Fu, g.s1), val(hi & 0x00F000F0u, g.s16));
}

// BIAS also serves a scale that is not positive: the scores are scaled before anything else looks at them
template <int D, bool QUANT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(TreeTc<D, QUANT>::THREADS, 1)
attn_tree_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TreeTcArgs f) {
  using L = TreeTc<D, QUANT>;
  constexpr int ST = L::ST;
  extern __shared__ __align__(1024) uint8_t smem[];
  const TreeArgs& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);   // tmem base, abort
  volatile int* const s_abort = s_flags + 1;
  Paths& paths = *reinterpret_cast<Paths*>(smem + L::OFF_PATHS);
  int* const s_depth = reinterpret_cast<int*>(smem + L::OFF_DEPTH);
  float* const s_scale = reinterpret_cast<float*>(smem + L::OFF_SCALE);
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };

  const int G = a.H / a.H_kv, R = a.N * G;
  const int part = blockIdx.x % a.parts, rb = blockIdx.x / a.parts % f.row_blocks, bg = blockIdx.x / a.parts / f.row_blocks;
  const int b = bg / a.H_kv, g = bg % a.H_kv, r0 = rb * (f.two ? 256 : 128);
  const bool two = f.two;
  const int warp_products = (256 + L::LOADERS) / 32;

  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar(L::B_FULL + i), QUANT ? 128 : 1);
      mbar_init(bar(L::B_EMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
      mbar_init(bar(L::B_O + i), 1);
    }
    mbar_init(bar(L::B_DONE), 1);
    s_flags[1] = 0;
    mbar_fence_init();
    if constexpr (!QUANT) {
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
    }
  }
  behind_last_kernel();
  if (warp == warp_products) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 512);
    tmem_relinquish();
  }
  const int pos = a.pos[b];
  const Ring ring = ring_of(pos, a.C, a.W);
  // tiles: the nodes' own up to the last one of these rows, then the cached ones
  const int nodes = pos < 0 ? 0 : min(a.N, (min(R, r0 + (two ? 256 : 128)) - 1) / G + 1), node_tiles_all = (nodes + 63) / 64;
  const int tiles = node_tiles_all + ring.tiles, per = (tiles + a.parts - 1) / a.parts, t0 = min(tiles, part * per), n = min(tiles - t0, per);
  const int node_tiles = max(0, min(node_tiles_all - t0, n));   // of this part
  find_paths(a, b, paths);
  if (tid < a.N) s_depth[tid] = pos < 0 ? -1 : node_depth(paths, tid, a.N);
  __syncthreads();

  // queries; rows that are not there are zeros
  const int q_rows = two ? 256 : 128;
  for (int i = tid; i < q_rows * (D / 8); i += L::THREADS) {
    const int r = i / (D / 8), j = i % (D / 8), row = r0 + r;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (row < R && s_depth[row / G] >= 0) w = *reinterpret_cast<const uint4*>((const bf16*)a.q + (((size_t)b * a.N + row / G) * a.H + g * G + row % G) * D + j * 8);
    if constexpr (QUANT) {
      float x[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
      for (int o = 1; o < D / 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));   // (a row's threads lie side by side; whole warps run)
      const uint32_t e2 = min(max(top >> 23, 1u), 253u);
      const float down = __uint_as_float((254u - e2) << 23);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= down;
      w = halves_in_order(x);
      if (j == 0) s_scale[r] = __uint_as_float(e2 << 23) / V_FACTOR;
    }
    sts128(sb + (uint32_t)(r >> 7) * L::TILE + (uint32_t)(j >> 3) * 16384 + sw128(r & 127, j & 7), w);
  }
  // the nodes' keys and values, into the first stages
  for (int i = tid; i < node_tiles * 64 * (D / 8); i += L::THREADS) {
    const int r = i / (D / 8), j = i % (D / 8), k = t0 * 64 + r;
    uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
    if (k < nodes && s_depth[k] >= 0) {
      const size_t src = (((size_t)b * a.N + k) * a.H_kv + g) * D + j * 8;
      x = *reinterpret_cast<const uint4*>((const bf16*)a.k_t + src);
      y = *reinterpret_cast<const uint4*>((const bf16*)a.v_t + src);
    }
    if constexpr (QUANT) {
      auto held = [&](uint4& w) {
        float u[8] = {bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y), bf16_lo(w.z), bf16_hi(w.z), bf16_lo(w.w), bf16_hi(w.w)};
        quantize8<D, true>(u, j * 8, nullptr, nullptr, false, 0xffffffffu);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] *= V_FACTOR;
        w = halves_in_order(u);
      };
      held(x);
      held(y);
    }
    const uint32_t st = sb + L::OFF_RING + (uint32_t)(r >> 6) * 2 * L::KT, at = (uint32_t)(j >> 3) * 8192 + sw128(r & 63, j & 7);
    sts128(st + at, x);
    sts128(st + L::KT + at, y);
  }
  fence_proxy_async();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0];
  auto s_col = [&](int u, int step) { return tmem + (uint32_t)(u * 128 + (step & 1) * 64); };
  auto o_col = [&](int u) { return tmem + (uint32_t)(256 + u * D); };
  // a warpgroup's steps: every tile, or every other one
  auto steps_of = [&](int u) { return two ? n : (n + 1 - u) / 2; };

  if (warp < 8) {
    // ------------------------------------------------------------------------------------------------ softmax
    const int u = warp >> 2, r128 = tid & 127, r = r0 + (two ? 128 * u : 0) + r128, steps = steps_of(u);
    const int node = min(r, R - 1) / G, h = g * G + min(r, R - 1) % G;
    const int depth = s_depth[node];
    const bool there = r < R && depth >= 0;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, O = o_col(u) + lanes;
    const float unit = QUANT ? s_scale[(two ? 128 * u : 0) + r128] : 1.f;   // of a product in tensor memory
    const float scale2 = a.scale * LOG2E * unit, slope2 = BIAS && a.slopes ? a.slopes[h] * LOG2E : 0.f;
    // the farthest key that the row sees, and the least of the warp's (rows that are not there weigh zeros, and are stored as zeros)
    const int far = there ? min(a.W - 1 - depth, pos) : 0x3fffffff;
    const int far_all = __reduce_min_sync(0xffffffffu, far);
    const bool idle = !__any_sync(0xffffffffu, there);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int step = 0; step < steps; ++step) {
      ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, f.limit));
      if (!ok) break;
      tc_fence_after_sync();
      const int it = two ? step : 2 * step + u;
      const uint32_t S = s_col(u, step) + lanes;
      float s[64];
      if (idle) {   // (no row of the warp is there, and none is stored: whatever stands for its weights)
        mbar_arrive(bar(L::B_P + 2 * u + (step & 1)));
        continue;
      }
#pragma unroll
      for (int c = 0; c < 64; c += 32) tmem_ld32(S + c, s + c);
      tmem_wait_ld();
      if constexpr (CAP) cap_scores(s, a.scale * unit / a.cap, a.cap * LOG2E);
      float by = CAP ? 1.f : scale2;
      if (it < node_tiles) {
        // the nodes' own: those of the path, by their distance
        const int j0 = (t0 + it) * 64;
        const uint32_t w0 = paths.on[node][j0 / 32], w1 = paths.on[node][j0 / 32 + 1];
#pragma unroll
        for (int c = 0; c < 64; c += 4) {
          const int4 e = *reinterpret_cast<const int4*>(s_depth + j0 + c);
          const int dist[4] = {depth - e.x, depth - e.y, depth - e.z, depth - e.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool see = ((c < 32 ? w0 : w1) >> (c + i & 31) & 1u) && dist[i] < a.W;
            float x = s[c + i];
            if constexpr (BIAS) x = fmaf(x, by, -slope2 * (float)dist[i]);
            s[c + i] = see ? x : -INFINITY;
          }
        }
        if constexpr (BIAS) by = 1.f;
      } else {
        const CachedTile t = cached_tile(ring, t0 + it - node_tiles_all, a.C);
        if constexpr (BIAS) {
          const uint64_t by2 = f2_pack(by, by), two2 = f2_pack(2.f * slope2, 2.f * slope2);
          const float first = -slope2 * (float)(t.back0 + depth);
          uint64_t add = f2_pack(first, first + slope2);
#pragma unroll
          for (int c = 0; c < 64; c += 2) {
            f2_unpack(f2_fma(f2_pack(s[c], s[c + 1]), by2, add), s[c], s[c + 1]);
            add = f2_add(add, two2);
          }
          by = 1.f;
        }
        if (t.back0 > far_all || t.lo > 0) {
          const int cl = max(t.back0 - far, t.lo);
#pragma unroll
          for (int c = 0; c < 64; ++c) s[c] = c < cl ? -INFINITY : s[c];
        }
      }
      float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
      for (int c = 0; c < 16; c += 2) {
        mx0 = fmaxf(fmaxf(mx0, s[c]), s[c + 1]);
        mx1 = fmaxf(fmaxf(mx1, s[c + 16]), s[c + 17]);
        mx2 = fmaxf(fmaxf(mx2, s[c + 32]), s[c + 33]);
        mx3 = fmaxf(fmaxf(mx3, s[c + 48]), s[c + 49]);
      }
      const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * by;
      const bool grow = mx > m + TREE_RESCALE || (m == -INFINITY && mx > m);
      if (__any_sync(0xffffffffu, grow)) {
        const float base = grow ? mx : m, factor = m == -INFINITY ? 0.f : ex2f(m - base);
        if (step > 0) {
          ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_O + 2 * u + (step - 1 & 1)), (step - 1) >> 1 & 1, s_abort, f.limit));   // (the product in front)
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            tmem_ld32(O + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= factor;
            tmem_st32(O + c, o);
          }
          tmem_wait_st();
        }
        l *= factor;
        m = base;
      }
      const float base = m == -INFINITY ? 0.f : m;
      const uint64_t sc = f2_pack(by, by), nb = f2_pack(-base, -base);
      uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
      for (int q = 0; q < 32; q += 8) {
        uint64_t z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = f2_fma(f2_pack(s[2 * (q + e)], s[2 * (q + e) + 1]), sc, nb);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x, y;
          f2_unpack(z[e], x, y);
          z[e] = f2_pack(ex2f(x), ex2f(y));
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          sum0 = f2_add(sum0, z[e]);
          sum1 = f2_add(sum1, z[e + 1]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x, y;
          f2_unpack(z[e], x, y);
          s[q + e] = __uint_as_float(QUANT ? pack_f16(x, y) : pack_bf16(x, y));
        }
      }
      tmem_st32(S, s);
      float x, y;
      f2_unpack(f2_add(sum0, sum1), x, y);
      l += x + y;
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive(bar(L::B_P + 2 * u + (step & 1)));
    }
    // ------------------------------------------------------------------------------------------------ outputs
    if (n > 0) ok = ok && __all_sync(0xffffffffu, wait_bar(bar(L::B_DONE), 0, s_abort, item_limit(f.limit, n)));
    tc_fence_after_sync();
    float* const s_o = reinterpret_cast<float*>(smem + L::OFF_RING);        // [D / 4][128] four channels of a row: every product is done
    float2* const s_ml = reinterpret_cast<float2*>(smem + L::OFF_ML);
    if (!two) {
      if (u == 1) {
        s_ml[r128] = make_float2(m, l);
        if (steps > 0) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            tmem_ld32(O + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(s_o + ((c + e) / 4 * 128 + r128) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
      }
      named_bar_sync(2, 256);
    }
    if (u == 0 || two) {
      float fa = 1.f, fb = 0.f;
      if (!two) {
        const float2 ml = s_ml[r128];
        const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.f : top;
        fa = ex2f(m - base);
        fb = ex2f(ml.x - base);
        if (m == -INFINITY) fa = 0.f;
        if (ml.x == -INFINITY) fb = 0.f;
        l = l * fa + ml.y * fb;
        m = top;
      }
      const bool both = !two && steps_of(1) > 0, some = steps > 0;
      if (!there) l = 0.f;
      const float inv = (a.parts > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l) * (QUANT ? 1.f / V_FACTOR : 1.f);
      float test = l * 0.f, largest = 0.f;
      const size_t row = ((size_t)b * a.N + node) * a.H + h;
      const size_t prow = (size_t)bg * a.parts + part;
      bf16* const dst = (bf16*)a.o + row * D;
      float* const pdst = f.part_o + prow * D * f.rows_pad + r;
#pragma unroll 1
      for (int c = 0; c < D; c += 32) {
        float o[32];
        if (some) {
          tmem_ld32(O + c, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (!two) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (both) x = *reinterpret_cast<const float4*>(s_o + ((c + e) / 4 * 128 + r128) * 4);
            const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) o[e + i] = (fa == 0.f ? 0.f : o[e + i] * fa) + (fb == 0.f ? 0.f : y[i] * fb);
          }
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          o[e] *= inv;
          test = fmaf(o[e], 0.f, test);
          if constexpr (QUANT) largest = fmaxf(largest, fabsf(o[e]));
        }
        if constexpr (QUANT) {   // channels of eight back into their order
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            const float x[8] = {o[e], o[e + 1], o[e + 2], o[e + 3], o[e + 4], o[e + 5], o[e + 6], o[e + 7]};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[e + i] = x[2 * i];
              o[e + 4 + i] = x[2 * i + 1];
            }
          }
        }
        if (r < R) {
          if (a.parts > 1) {
#pragma unroll
            for (int e = 0; e < 32; ++e) pdst[(size_t)(c + e) * f.rows_pad] = o[e];
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(dst + c + e) = l == 0.f ? make_uint4(0u, 0u, 0u, 0u)
                                                                : make_uint4(pack_bf16(o[e], o[e + 1]), pack_bf16(o[e + 2], o[e + 3]), pack_bf16(o[e + 4], o[e + 5]), pack_bf16(o[e + 6], o[e + 7]));
          }
        }
      }
      if (r < R && a.parts > 1) f.part_ml[prow * f.rows_pad + r] = make_float2(m, l);
      // rows to be computed again (with several parts the join looks)
      const bool bad = ok && there && a.parts == 1 && (!(test == 0.f) || (QUANT && largest < SMALL));
      uint32_t left = __ballot_sync(0xffffffffu, bad);
      __syncwarp();   // (behind the stores of the row's own thread)
      for (; left; left &= left - 1) {
        const int from = __ffs(left) - 1;
        tree_row_again<bf16, D, QUANT>(a, b, __shfl_sync(0xffffffffu, node, from), __shfl_sync(0xffffffffu, h, from));
      }
    }
  } else if (warp < warp_products) {
    if constexpr (!QUANT) {
      // ---------------------------------------------------------------------------------------------- copies
      if (elect_one()) {
        for (int it = 0; it < node_tiles; ++it) {
          mbar_arrive(bar(L::B_FULL + 2 * it));
          mbar_arrive(bar(L::B_FULL + 2 * it + 1));
        }
        bool ok = true;
        for (int it = node_tiles; it < n && ok; ++it) {
          const CachedTile t = cached_tile(ring, t0 + it - node_tiles_all, a.C);
#pragma unroll
          for (int v = 0; v < 2 && ok; ++v) {
            const int at = 2 * it + v, s = at % ST;
            if (at >= ST) ok = wait_bar(bar(L::B_EMPTY + s), (at / ST - 1) & 1, s_abort, f.limit);
            if (!ok) break;
            mbar_arrive_expect_tx(bar(L::B_FULL + s), L::KT);
            load_tile<D, 64>(sb + L::OFF_RING + s * L::KT, v ? &tm_v : &tm_k, bar(L::B_FULL + s), g, t.s0, b);
          }
        }
      }
    } else {
      // ---------------------------------------------------------------------------------------------- codes
      // a thread has half of a slot's channels of K and of V: D / 64 groups each
      constexpr int NG = D / 64;
      const int ltid = tid - 256, slot = ltid >> 1, half = ltid & 1;
      const size_t head = ((size_t)b * a.H_kv + g) * a.C;
      struct Codes {
        uint4 k[NG], v[NG];
        uint32_t kp[NG], vp[NG];
      } buf[PREFETCH];
      auto fetch = [&](int it, Codes& x) {
        const CachedTile t = cached_tile(ring, t0 + it - node_tiles_all, a.C);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          x.k[i] = x.v[i] = make_uint4(0u, 0u, 0u, 0u);
          x.kp[i] = x.vp[i] = 0u;
        }
        if (slot < t.lo || t.s0 + slot < 0 || t.back0 - slot > ring.cached) return;   // (zeros)
        const size_t row = head + (t.s0 + slot);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          x.k[i] = __ldcs(reinterpret_cast<const uint4*>(a.kq + row * (D / 2)) + half * NG + i);
          x.v[i] = __ldcs(reinterpret_cast<const uint4*>(a.vq + row * (D / 2)) + half * NG + i);
          x.kp[i] = __ldcs(reinterpret_cast<const uint32_t*>(a.kp + row * (D / 16)) + half * NG + i);
          x.vp[i] = __ldcs(reinterpret_cast<const uint32_t*>(a.vp + row * (D / 16)) + half * NG + i);
        }
      };
      for (int it = 0; it < node_tiles; ++it) {
        mbar_arrive(bar(L::B_FULL + 2 * it));
        mbar_arrive(bar(L::B_FULL + 2 * it + 1));
      }
#pragma unroll
      for (int p = 0; p < PREFETCH; ++p)
        if (node_tiles + p < n) fetch(node_tiles + p, buf[p]);
      bool ok = true;
      auto put = [&](int at, const uint4 (&codes)[NG], const uint32_t (&pairs)[NG]) {
        const int s = at % ST;
        if (at >= ST) ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_EMPTY + s), (at / ST - 1) & 1, s_abort, f.limit));
        if (!ok) return;
        const uint32_t st = sb + L::OFF_RING + s * L::KT;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const GroupScale gs = group_scale(pairs[i]);
          const uint32_t w[4] = {codes[i].x, codes[i].y, codes[i].z, codes[i].w};
          const int j0 = (half * NG + i) * 4;   // chunks of eight channels
#pragma unroll
          for (int e = 0; e < 4; ++e) sts128(st + (uint32_t)(j0 >> 3) * 8192 + sw128(slot, (j0 & 7) + e), unpack8(w[e], gs));
        }
        fence_proxy_async();
        mbar_arrive(bar(L::B_FULL + s));
      };
      for (int it0 = node_tiles; it0 < n && ok; it0 += PREFETCH) {
#pragma unroll
        for (int p = 0; p < PREFETCH; ++p) {
          const int it = it0 + p;
          if (it >= n || !ok) break;
          put(2 * it, buf[p].k, buf[p].kp);
          if (ok) put(2 * it + 1, buf[p].v, buf[p].vp);
          if (it + PREFETCH < n) fetch(it + PREFETCH, buf[p]);
        }
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ products
    if (n > 0 && elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, L::FMT, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_o = instr_desc(128, D, L::FMT, MAJOR_K, MAJOR_MN);
      auto stage = [&](int at) { return sb + L::OFF_RING + (uint32_t)(at % ST) * L::KT; };
      auto full = [&](int at) { return wait_bar(bar(L::B_FULL + at % ST), (at / ST) & 1, s_abort, f.limit); };
      auto scores = [&](int u, int it, int step, bool first, bool last) {   // first, last: of the warpgroups that meet the tile
        if (first && !full(2 * it)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(u, step), kdesc<128>(sb + (two ? u : 0) * L::TILE, kk), kdesc<64>(stage(2 * it), kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + 2 * it % ST));
        return true;
      };
      auto values = [&](int u, int it, int step, bool first, bool last) {
        if (first && !full(2 * it + 1)) return false;
        if (!wait_bar(bar(L::B_P + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, f.limit)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(o_col(u), s_col(u, step) + kk * 8, mdesc<64>(stage(2 * it + 1), kk), id_o, (step | kk) != 0);
        mma_commit(bar(L::B_O + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + (2 * it + 1) % ST));
        return true;
      };
      bool ok = true;
      if (two) {
        ok = scores(0, 0, 0, true, false) && scores(1, 0, 0, false, true);
        for (int it = 0; it < n && ok; ++it) {
#pragma unroll
          for (int u = 0; u < 2 && ok; ++u) {
            if (it + 1 < n) ok = scores(u, it + 1, it + 1, u == 0, u == 1);
            if (ok) ok = values(u, it, it, u == 0, u == 1);
          }
        }
      } else {
        ok = scores(0, 0, 0, true, true) && (n < 2 || scores(1, 1, 0, true, true));
        for (int it = 0; it < n && ok; ++it) {
          if (it + 2 < n) ok = scores(it & 1, it + 2, (it >> 1) + 1, true, true);
          if (ok) ok = values(it & 1, it, it >> 1, true, true);
        }
      }
      if (ok) mma_commit(bar(L::B_DONE));
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && f.dev_status) atomicMax(f.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == warp_products) tmem_dealloc(tmem, 512);
}

// The parts of a group's rows: a thread has eight channels of a row (a warp 32 rows side by side), in one pass over the parts.
template <int D, bool QUANT>
__global__ void __launch_bounds__(D * 4) attn_tree_join_tc_kernel(const __grid_constant__ TreeTcArgs f) {
  const TreeArgs& a = f.a;
  const int G = a.H / a.H_kv, R = a.N * G, chunks = (R + 31) / 32;
  const int bg = blockIdx.x / chunks, r = blockIdx.x % chunks * 32 + (threadIdx.x & 31), c0 = threadIdx.x / 32 * 8, lane = threadIdx.x & 31;
  const int b = bg / a.H_kv, g = bg % a.H_kv;
  __shared__ uint32_t s_bad;
  __shared__ uint32_t s_large;
  if (threadIdx.x == 0) s_bad = s_large = 0u;
  __syncthreads();
  behind_last_kernel();
  const size_t p0 = (size_t)bg * a.parts;
  float m = -INFINITY, l = 0.f, acc[8] = {};
  if (r < R) {
    constexpr int U = 2;
    for (int i0 = 0; i0 < a.parts; i0 += U) {
      float2 ml[U];
      float x[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool some = i0 + u < a.parts;
        const size_t p = p0 + (some ? i0 + u : 0);
        ml[u] = some ? f.part_ml[p * f.rows_pad + r] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = f.part_o[(p * D + c0 + e) * f.rows_pad + r];
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, ml[u].x);
      const float base = top == -INFINITY ? 0.f : top, k = ex2f(m - base);
      m = top;
      l *= k;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= k;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = ex2f(ml[u].x - base);
        if (ml[u].y != 0.f) {               // (a part without keys has no weights)
          l += w * ml[u].y;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, x[u][e], acc[e]);
        }
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float test = l * 0.f, largest = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    acc[e] *= inv;
    test = fmaf(acc[e], 0.f, test);
    largest = fmaxf(largest, fabsf(acc[e]));
  }
  const int node = min(r, R - 1) / G, h = g * G + min(r, R - 1) % G;
  if (r < R)
    *reinterpret_cast<uint4*>((bf16*)a.o + (((size_t)b * a.N + node) * a.H + h) * D + c0) =
        make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
  const uint32_t bad = __ballot_sync(0xffffffffu, r < R && !(test == 0.f)), large = __ballot_sync(0xffffffffu, !(r < R) || l == 0.f || !(largest < SMALL));
  if (lane == 0) {
    if (bad) atomicOr(&s_bad, bad);
    if (large) atomicOr(&s_large, large);
  }
  __syncthreads();
  const uint32_t again = s_bad | (QUANT ? ~s_large : 0u);
  for (int i = threadIdx.x / 32; i < 32; i += blockDim.x / 32)   // (behind the barrier: nobody writes these rows any more)
    if (again >> i & 1u) {
      const int row = blockIdx.x % chunks * 32 + i;
      tree_row_again<bf16, D, QUANT>(a, b, row / G, g * G + row % G);
    }
}

static TreePlan tree_plan(int B, int N, int H, int H_kv, int C, int W) {
  TreePlan p;
  const int R = N * (H / H_kv);
  p.two = R > 128;
  p.row_blocks = (R + 255) / 256;
  // Parts of the keys: as many as give every SM a few rounds, and no more than there are pieces of 256 keys.
  const long long blocks = (long long)B * H_kv * p.row_blocks, want = (2LL * sm_count() + blocks - 1) / std::max(1LL, blocks);
  const int most = std::min(W, C) / 256 + 1;
  p.parts = (int)std::max(1LL, std::min<long long>(want, most));
  return p;
}

template <int D, bool QUANT, bool CAP, bool BIAS>
static int tree_tc(const AttnTree& c) {
  using L = TreeTc<D, QUANT>;
  const TreeArgs& a = c.a;
  const TreePlan p = tree_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W);
  const long long blocks = (long long)a.B * a.H_kv * p.row_blocks * p.parts;
  if (blocks > 0x7fffffffLL) return LAWCAT_ERR_UNSUPPORTED;
  CUtensorMap tk{}, tv{};
  if (!QUANT && (!tensor_map(&tk, a.K, false, a.H_kv, a.C, a.B, D, 64, 64, true) || !tensor_map(&tv, a.V, false, a.H_kv, a.C, a.B, D, 64, 64, true)))
    return LAWCAT_ERR_CUDA;
  TreeTcArgs f{a, p.row_blocks, p.two, (a.N * (a.H / a.H_kv) + 31) / 32 * 32, nullptr, nullptr, wait_limit(), c.dev_status};
  f.a.parts = p.parts;
  if (p.parts > 1) {
    f.part_ml = (float2*)c.ws;
    f.part_o = (float*)((char*)c.ws + align_up(sizeof(float2) * (size_t)a.B * a.H_kv * p.parts * f.rows_pad, 256));
  }
  constexpr auto kernel = attn_tree_tc_kernel<D, QUANT, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_tree_tc", c.stream, launch_behind(kernel, dim3((unsigned)blocks), dim3(L::THREADS), L::BYTES, c.stream, tk, tv, f));
  LAWCAT_CHECK_LAUNCH();
  if (p.parts == 1) return LAWCAT_OK;
  const unsigned join = (unsigned)((long long)a.B * a.H_kv * (f.rows_pad / 32));
  LAWCAT_LAUNCH("attn_tree_join_tc", c.stream, launch_behind(attn_tree_join_tc_kernel<D, QUANT>, dim3(join), dim3(D * 4), 0, c.stream, f));
  LAWCAT_CHECK_LAUNCH();
  return LAWCAT_OK;
}

}  // namespace attn

size_t attn_tree_tc_workspace_bytes(int B, int N, int H, int H_kv, int C, int W, int d) {
  const attn::TreePlan p = attn::tree_plan(B, N, H, H_kv, C, W);
  if (p.parts == 1) return 0;
  const size_t rows = (size_t)B * H_kv * p.parts * ((N * (H / H_kv) + 31) / 32 * 32);
  return align_up(sizeof(float2) * rows, 256) + align_up(sizeof(float) * rows * d, 256);
}

int launch_attn_tree_tc(const AttnTree& c) {
  auto by = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    if (c.a.kq) return c.d == 128 ? attn::tree_tc<128, true, CAP, BIAS>(c) : attn::tree_tc<64, true, CAP, BIAS>(c);
    return c.d == 128 ? attn::tree_tc<128, false, CAP, BIAS>(c) : attn::tree_tc<64, false, CAP, BIAS>(c);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (c.a.cap > 0.f) return c.a.slopes ? by(yes, yes) : by(yes, no);
  return c.a.slopes || !(c.a.scale > 0.f) ? by(no, yes) : by(no, no);
}

}  // namespace lawcat

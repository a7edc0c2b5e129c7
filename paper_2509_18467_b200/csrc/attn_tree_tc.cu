// Attention of drafted tokens over a cache on the tensor cores: bf16, d = 64 or 128; the cache in the storage type, or in 4 bits where there are
// more rows than attn_tree_quant_tc.cu has columns.
//
// A block walks segments of up to 256 rows (node, query head) of one (sequence, key-value head) and their keys, in tiles of 64:
//   two warpgroups    softmax, one thread per row: S from tensor memory, masks, running maximum and sum in registers, P = exp2(x - m) over S;
//                     then the segment's outputs
//   copy warp         queries, K and V tiles (through a ring of stages) by TMA, on into the next segment while this one ends;
//                     over 4 bits seven warps in its place, which unpack codes into the stages (a warp at a time 32 groups of 32 channels), and
//                     the queries come by the softmax warps
//   product warp      S = Q K^T (shared memory), O += P V (P from tensor memory); fp32 accumulation
// A tile of rows is as many whole nodes as 128 rows hold. Of two tiles each warpgroup has one, and both meet every key; of one, both have its
// rows and take the key tiles in turn, each with sums of its own (in the same lanes of tensor memory) that meet at the segment's end. S has two
// places per warpgroup; O is rescaled only when a maximum grew by more than 2^8.
//
// Cycles of an SM a tile of keys: 1300 up to 128 rows at d = 128, with 256 rows 1990 (1590 at d = 64), where the softmax's chain of product, maximum,
// weights, product bounds it. 16 sequences of 4095 to 8190 tokens, 32/8 heads of 128, 32 nodes: 85 us, of which HBM alone would take 63 and the tiles take
// 56; what is over is set-up and the join of cut segments. The same over 4 bits 125 us, with 64 nodes 171 (the warps that unpack).
//
// The keys are walked from the newest to the oldest: the nodes' own rows first (the values of nodes that are not there are set to zero), then
// the cached ones, whose tiles end where the newest slot, or slot C - 1, does. What a tile holds below its oldest key are slots in front of
// slot 0, which read as zeros, or older tokens: never a slot without a token. So a row sees a tile's columns from one limit on.
//
// Rounding: weights to bf16 as an operand (over 4 bits they, keys, values and queries to fp16, attn_tree_tc.cuh), o once; all else fp32.
#include <algorithm>

#include "attn_tree_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float TREE_RESCALE = 8.f;

template <int D, bool QUANT>
struct TreeTc {
  static constexpr uint32_t TILE = 128 * D * 2, KT = 64 * D * 2;   // rows' queries; keys or values of a tile
  static constexpr int ST = D == 64 ? 16 : 8;                      // stages, K and V tiles in turn
  static constexpr uint32_t OFF_RING = 2 * TILE, OFF_PATHS = OFF_RING + ST * KT, OFF_DEPTH = OFF_PATHS + sizeof(Paths), OFF_ML = OFF_DEPTH + TREE_MAX * 4;
  static constexpr uint32_t OFF_BAD = OFF_ML + 256 * 8, OFF_SCALE = OFF_BAD + 64, OFF_BAR = OFF_SCALE + 256 * 4, BYTES = OFF_BAR + 512;
  static constexpr int LOADERS = QUANT ? 7 : 1, THREADS = 288 + 32 * LOADERS, FMT = QUANT ? FMT_F16 : FMT_BF16;
  static constexpr int ITEMS = D / 32;   // a tile's parts over 4 bits: 2 x 32 groups of 32 channels of keys and of values
  static constexpr int B_FULL = 0, B_EMPTY = ST, B_S = 2 * ST, B_P = B_S + 4, B_O = B_P + 4, B_DONE = B_O + 4, B_Q = B_DONE + 1, B_QE = B_Q + 2, B_OE = B_QE + 2, B_FIX = B_OE + 1, NBAR = B_FIX + 1;
  static_assert(BYTES <= 232448 && NBAR * 8 + 16 <= 512 && 256 + 2 * D <= 512 && TREE_MAX / 64 * 2 <= ST, "shared memory, tensor memory");
};

// BIAS also serves a scale that is not positive: the scores are scaled before anything else looks at them
template <int D, bool QUANT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(TreeTc<D, QUANT>::THREADS, 1)
attn_tree_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_kt,
                    const __grid_constant__ CUtensorMap tm_vt, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ TreeTcArgs f) {
  using L = TreeTc<D, QUANT>;
  constexpr int ST = L::ST;
  extern __shared__ __align__(1024) uint8_t smem[];
  const TreeArgs& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 8 * L::NBAR);   // tmem base, abort
  volatile int* const s_abort = s_flags + 1;
  auto bar = [&](int i) { return sb + L::OFF_BAR + 8 * (uint32_t)i; };
  uint32_t* const s_bad = reinterpret_cast<uint32_t*>(smem + L::OFF_BAD);   // [8] rows to be computed again
  uint32_t* const s_large = s_bad + 8;                                       // [8] over 4 bits: rows that are not small everywhere
  const int G = a.H / a.H_kv, R = a.N * G;
  const bool two = f.rows > f.tile_rows;
  const int q_tiles = two ? 2 : 1, q_places = two || QUANT ? 1 : 2;   // of a segment, and segments whose queries fit

  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(bar(L::B_FULL + i), L::LOADERS);
      mbar_init(bar(L::B_EMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(L::B_S + i), 1);
      mbar_init(bar(L::B_P + i), 128);
      mbar_init(bar(L::B_O + i), 1);
    }
    mbar_init(bar(L::B_DONE), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(L::B_Q + i), QUANT ? 256 : 1);
      mbar_init(bar(L::B_QE + i), 1);
    }
    mbar_init(bar(L::B_OE), 256);
    mbar_init(bar(L::B_FIX), 256);
    s_flags[1] = 0;
    for (int i = 0; i < 16; ++i) s_bad[i] = 0u;
    mbar_fence_init();
    if constexpr (!QUANT) {
      tma_prefetch_desc(&tm_q);
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
      tma_prefetch_desc(&tm_kt);
      tma_prefetch_desc(&tm_vt);
    }
  }
  behind_last_kernel();
  const int pos_lane = lane_position(f);
  if (warp == 9) {
    tmem_alloc(sb + L::OFF_BAR + 8 * L::NBAR, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0];
  auto s_col = [&](int u, int step) { return tmem + (uint32_t)(u * 128 + (step & 1) * 64); };
  auto o_col = [&](int u) { return tmem + (uint32_t)(256 + u * D); };
  // a warpgroup's steps of a piece: every tile, or every other one
  auto steps_of = [&](int u, int n) { return two ? n : (n + 1 - u) / 2; };
  // What the copy and product warps wait for may come behind rows of the last piece that are computed again: as many keys as its segment has. So
  // they wait as long as the longest segment so far allows.
  long long patience = f.limit;
  Walk<64> walk;
  const int share = share_of_block(f);
  if (tid == 0 && !f.whole && !f.apart) f.told[share] = 0ull;   // (what a call that gave up may have left)
  walk.start(f, share, pos_lane);
  Piece w;

  if (warp < 8) {
    // ------------------------------------------------------------------------------------------------ softmax
    Paths& paths = *reinterpret_cast<Paths*>(smem + L::OFF_PATHS);
    int* const s_depth = reinterpret_cast<int*>(smem + L::OFF_DEPTH);
    float2* const s_ml = reinterpret_cast<float2*>(smem + L::OFF_ML);   // [2][128]
    const int u = warp >> 2, r128 = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, O = o_col(u) + lanes;
    float* const s_scale = reinterpret_cast<float*>(smem + L::OFF_SCALE);   // over 4 bits: what a row's queries were divided by
    int step = 0, seq = 0, at = 0, b_last = -1;   // steps, pieces and tiles so far
    bool ok = true;
    while (walk.next(f, w)) {
      const int b = w.b, pos = w.pos, n = w.n, steps = steps_of(u, n), node_tiles = max(0, min(f.node_tiles - w.t0, n));
      if (b != b_last) {
        find_paths<256>(a, b, paths, tid, 1);
        if (tid < a.N) s_depth[tid] = pos < 0 ? -1 : node_depth(paths, tid, a.N);
        named_bar_sync(1, 256);
        b_last = b;
      }
      if constexpr (QUANT) {   // (all products with the last piece's are done; queries of rows that are not there may be anything)
#pragma unroll 4
        for (int i = tid; i < q_tiles * 128 * (D / 8); i += 256) {
          const int p = i / (D / 8), j = i % (D / 8), row = min(row_of_piece(f, w.rb, p), R - 1), nd = quot(row, f.group);
          const uint4 x = *reinterpret_cast<const uint4*>((const bf16*)a.q + (((size_t)b * a.N + nd) * a.H + w.g * G + rest(row, nd, f.group)) * D + j * 8);
          uint4 y;
          const float up = scale_query<D>(x, y, a.scale);
          sts128(sb + (uint32_t)(p >> 7) * L::TILE + (uint32_t)(j >> 3) * 16384 + sw128(p & 127, j & 7), y);
          if (j == 0) s_scale[p] = up / KV_FACTOR;
        }
        fence_proxy_async();
        mbar_arrive(bar(L::B_Q));
        named_bar_sync(2, 256);   // (s_scale)
      }
      // the values of nodes that are not there: zeros (their weights are, and whatever they hold must not meet those); with a cap their keys too,
      // whose scores would help to choose its form
      for (int it = 0; it < node_tiles; ++it) {
        const int st = 2 * (at + it) + 1, k = (w.t0 + it) * 64 + (tid >> 2);
        if (k < a.N && s_depth[k] < 0) {
          ok = ok && wait_bar(bar(L::B_FULL + st % ST), (st / ST) & 1, s_abort, f.limit) &&
               (!CAP || wait_bar(bar(L::B_FULL + st % ST - 1), (st / ST) & 1, s_abort, f.limit));
          if (ok)
#pragma unroll
            for (int j = tid & 3; j < D / 8; j += 4) {
              const uint32_t at = sb + L::OFF_RING + (uint32_t)(st % ST) * L::KT + (uint32_t)(j >> 3) * 8192 + sw128(tid >> 2, j & 7);
              sts128(at, make_uint4(0u, 0u, 0u, 0u));
              if (CAP) sts128(at - L::KT, make_uint4(0u, 0u, 0u, 0u));
            }
          fence_proxy_async();
        }
      }
      if (node_tiles) mbar_arrive(bar(L::B_FIX));   // (once for all of them: the ring holds them together)
      __syncwarp();
      ok = __all_sync(0xffffffffu, ok);

      const int rp = (two ? 128 * u : 0) + r128, r = row_of_piece(f, w.rb, rp);
      const int node = quot(min(r, R - 1), f.group), h = w.g * G + rest(min(r, R - 1), node, f.group);
      const int depth = s_depth[node];
      const bool there = r < R && depth >= 0;
      const float unit = QUANT ? s_scale[rp] : 1.f;   // of a product in tensor memory
      const float cap_scale = CAP ? a.scale * unit / a.cap : 0.f;
      const float scale2 = a.scale * LOG2E * unit, slope2 = BIAS && a.slopes ? a.slopes[h] * LOG2E : 0.f;
      const Ring<64> ring = ring_of<64>(pos, a.C, a.W);
      // the farthest key that the row sees, and the least of the warp's (of rows that are not there nothing is stored but zeros)
      const int far = there ? min(a.W - 1 - depth, pos) : 0x3fffffff;
      const int far_all = __reduce_min_sync(0xffffffffu, far);
      const bool idle = !__any_sync(0xffffffffu, there);
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < steps && ok; ++i, ++step) {
        ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_S + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, f.limit));
        if (!ok) break;
        tc_fence_after_sync();
        if (idle) {   // (no row of the warp is there, and none is stored: whatever stands for its weights)
          tc_fence_before_sync();
          mbar_arrive(bar(L::B_P + 2 * u + (step & 1)));
          continue;
        }
        const int it = w.t0 + (two ? i : 2 * i + u);
        const uint32_t S = s_col(u, step) + lanes;
        float s[64];
#pragma unroll
        for (int c = 0; c < 64; c += 32) tmem_ld32(S + c, s + c);
        tmem_wait_ld();
        // (the cap's form is chosen by the warp's scores: none of rows that are not there, whatever they hold)
        if constexpr (CAP) cap_scores(s, cap_scale, a.cap * LOG2E, there ? cap_reach(top_score(s), cap_scale) : 0.f);
        float by = CAP ? 1.f : scale2;
        if (it < f.node_tiles) {
          // the nodes' own: those of the path, by their distance
          const int j0 = it * 64;
          const uint32_t w0 = paths.on[node][j0 / 32], w1 = paths.on[node][j0 / 32 + 1];
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const int4 e = *reinterpret_cast<const int4*>(s_depth + j0 + c);
            const int dist[4] = {depth - e.x, depth - e.y, depth - e.z, depth - e.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const bool see = ((c < 32 ? w0 : w1) >> (c + k & 31) & 1u) && dist[k] < a.W;
              float x = s[c + k];
              if constexpr (BIAS) x = fmaf(x, by, -slope2 * (float)dist[k]);
              s[c + k] = see ? x : -INFINITY;
            }
          }
          if constexpr (BIAS) by = 1.f;
        } else {
          const CachedTile t = cached_tile(ring, it - f.node_tiles, a.C);
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
          if (i > 0) {
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
        const float less = QUANT ? WEIGHT_SHIFT - base : -base;
        const uint64_t sc = f2_pack(by, by), nb = f2_pack(less, less);
        uint64_t sum0 = 0, sum1 = 0;
#pragma unroll
        for (int q = 0; q < 32; q += 8) {   // (step by step over eight pairs: what one warp has in flight is all that hides latencies)
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
      // ---------------------------------------------------------------------------------------------- outputs
      ok = ok && __all_sync(0xffffffffu, wait_bar(bar(L::B_DONE), seq & 1, s_abort, item_limit(f.limit, n)));
      tc_fence_after_sync();
      // with one tile of rows a warpgroup has half of the channels of both sums
      const bool join = is_joined_here(f, w), direct = is_whole(w) || join;
      float f0 = 1.f, f1 = 0.f;
      bool none0 = false, none1 = false;   // (sums without keys: whatever stands there; a weight that underflows takes a NaN along)
      if (!two) {
        s_ml[u * 128 + r128] = make_float2(m, l);
        named_bar_sync(2, 256);
        const float2 x = s_ml[r128], y = s_ml[128 + r128];
        const float top = fmaxf(x.x, y.x), base = top == -INFINITY ? 0.f : top;
        none0 = x.x == -INFINITY;
        none1 = y.x == -INFINITY;
        f0 = none0 ? 0.f : ex2f(x.x - base);
        f1 = none1 ? 0.f : ex2f(y.x - base);
        l = x.y * f0 + y.y * f1;
        m = top;
      }
      if (!there) l = 0.f;
      // the other pieces of the segment, where this block joins them
      const int others = join ? w.last - share : 0;
      auto other_ml = [&](int i) { return __ldcg(f.part_ml + (size_t)(share + 1 + i) * f.rows_pad + rp); };
      if (join) {
        bool told = true;
        if (tid == 0)
          for (int i = 0; i < others && told; ++i) told = wait_told(f.told + share + 1 + i, f.number, s_abort, item_limit(f.limit, w.tiles));
        ok = !named_bar_or(2, 256, !told || !ok);
        float top = l == 0.f ? -INFINITY : m, sum = 0.f;
        if (r < R)
          for (int i = 0; i < others; ++i) {
            const float2 x = other_ml(i);
            const float was = top;
            if (x.y == 0.f) continue;   // (a piece without keys has no weights)
            top = fmaxf(top, x.x);
            sum = sum * (was == -INFINITY ? 0.f : ex2f(was - top)) + x.y * ex2f(x.x - top);
          }
        const float own = m == -INFINITY || top == -INFINITY ? 0.f : ex2f(m - top);
        f0 *= own;
        f1 *= own;
        l = there ? l * own + sum : 0.f;
        m = top;
      }
      if (QUANT) {
        f0 *= 1.f / KV_FACTOR;
        f1 *= 1.f / KV_FACTOR;
      }
      const float inv = !direct ? 1.f : l == 0.f ? 0.f : 1.f / l;
      float test = l * 0.f, largest = 0.f;
      bf16* const dst = (bf16*)a.o + (((size_t)b * a.N + node) * a.H + h) * D;
      float* const pdst = f.part_o + (size_t)share * D * f.rows_pad + rp;
      const int c0 = two ? 0 : u * (D / 2), c1 = two ? D : c0 + D / 2;
      const uint32_t O0 = o_col(two ? u : 0) + lanes, O1 = o_col(1) + lanes;
      const bool both = !two && n > 1;
#pragma unroll 1
      for (int c = c0; c < c1; c += 16) {   // (code that runs once per piece is short: it comes from the instruction caches' far end)
        float o[16];
        tmem_ld16(O0 + c, o);
        if (both) {
          float y[16];
          tmem_ld16(O1 + c, y);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = (none0 ? 0.f : o[e] * f0) + (none1 ? 0.f : y[e] * f1);
        } else {
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] *= f0;
        }
        if constexpr (QUANT) {   // channels of eight back into their order
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            const float x[8] = {o[e], o[e + 1], o[e + 2], o[e + 3], o[e + 4], o[e + 5], o[e + 6], o[e + 7]};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              o[e + k] = x[2 * k];
              o[e + 4 + k] = x[2 * k + 1];
            }
          }
        }
        if (r < R)
#pragma unroll 1
          for (int i = 0; i < others; ++i) {
            const float2 y = other_ml(i);
            const float* const from = f.part_o + ((size_t)(share + 1 + i) * D + c) * f.rows_pad + rp;
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = __ldcg(from + e * f.rows_pad);
            const float k = ex2f(y.x - m);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] += y.y == 0.f ? 0.f : k * x[e];
          }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          o[e] *= inv;
          test = fmaf(o[e], 0.f, test);
          if constexpr (QUANT) largest = fmaxf(largest, fabsf(o[e]));
        }
        if (r < R) {
          if (!direct) {
            float* const to = pdst + (size_t)c * f.rows_pad;
#pragma unroll
            for (int e = 0; e < 16; ++e) to[e * f.rows_pad] = o[e];
          } else {
#pragma unroll
            for (int e = 0; e < 16; e += 8)
              *reinterpret_cast<uint4*>(dst + c + e) = l == 0.f ? make_uint4(0u, 0u, 0u, 0u)
                                                                : make_uint4(pack_bf16(o[e], o[e + 1]), pack_bf16(o[e + 2], o[e + 3]), pack_bf16(o[e + 4], o[e + 5]), pack_bf16(o[e + 6], o[e + 7]));
          }
        }
      }
      tc_fence_before_sync();
      mbar_arrive(bar(L::B_OE));
      if (r < R && !direct && (two || u == 0)) f.part_ml[(size_t)share * f.rows_pad + rp] = make_float2(m, l);
      // rows to be computed again (of a segment in pieces whoever joins them looks)
      const uint32_t bad = __ballot_sync(0xffffffffu, ok && there && direct && !(test == 0.f));
      const uint32_t large = QUANT ? __ballot_sync(0xffffffffu, !(ok && there && direct) || l == 0.f || !(largest < SMALL)) : 0xffffffffu;
      if (lane == 0) {
        if (bad) atomicOr(s_bad + (rp >> 5), bad);
        if (QUANT && large) atomicOr(s_large + (rp >> 5), large);
      }
      if (named_bar_or(2, 256, bad != 0u || large != 0xffffffffu)) {
        bool small = false;
        if constexpr (QUANT)
          if (named_bar_or(2, 256, ~s_large[rp >> 5] != 0u)) small = named_bar_or(2, 256, small_values<D, 256>(a, b, w.g, tid));
        for (int i = warp; i < q_tiles * 128; i += 8)
          if ((s_bad[i >> 5] | (small ? ~s_large[i >> 5] : 0u)) >> (i & 31) & 1u) {
            const int row = row_of_piece(f, w.rb, i), again = quot(row, f.group);
            tree_row_again<bf16, D, QUANT>(a, b, again, w.g * G + rest(row, again, f.group));
          }
      }
      ++seq;
      at += n;
      if (named_bar_or(2, 256, !ok)) break;   // (s_ml, the paths and the flags have been read)
      if (tid < 16) s_bad[tid] = 0u;          // (written again behind other barriers)
      if (!direct && !f.apart && tid == 0) tell(f.told + share, f.number);
    }
  } else if (warp != 9) {
    // ------------------------------------------------------------------------------------------------ copies
    if constexpr (QUANT) {
      // Parts of tiles, taken up by the warps in turn: the keys and the values of 2 x 32 / (D / 32) slots, so that one fence (some 700 cycles of a
      // warp's time) does for four stores of 32 groups. Zeros where no row may see a slot.
      constexpr int NG = D / 32, SLOTS = 32 / NG, AHEAD = 6;   // AHEAD: tiles towards L2
      const int me = warp == 8 ? 0 : warp - 9, slot = lane / NG, grp = lane % NG;
      int tile = 0;   // tiles of the pieces so far
      bool ok = true;
      while (ok && walk.next(f, w)) {
        patience = max(patience, item_limit(f.limit, w.tiles));
        const Ring<64> ring = ring_of<64>(w.pos, a.C, a.W);
        const size_t head = ((size_t)w.b * a.H_kv + w.g) * a.C;
        const int fresh = max(0, min(f.node_tiles - w.t0, w.n)), all = w.n * L::ITEMS;
        uint4 q[4];       // keys of the first and second slots, then values
        uint32_t pr[4];
        auto fetch = [&](int x) {   // part x of the piece
          const int it = (uint32_t)x / L::ITEMS;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            q[e] = make_uint4(0u, 0u, 0u, 0u);
            pr[e] = 0u;
          }
          if (x >= all || it < fresh) return;
          const CachedTile t = cached_tile(ring, w.t0 + it - f.node_tiles, a.C);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int c = ((uint32_t)x % L::ITEMS * 2 + e) * SLOTS + slot;
            if (c < t.lo || t.s0 + c < 0 || t.back0 - c > ring.cached) continue;
            const size_t row = head + (uint32_t)(t.s0 + c);
            q[e] = __ldcs(reinterpret_cast<const uint4*>(a.kq + row * (D / 2)) + grp);
            q[2 + e] = __ldcs(reinterpret_cast<const uint4*>(a.vq + row * (D / 2)) + grp);
            pr[e] = __ldcs(reinterpret_cast<const uint32_t*>(a.kp + row * (D / 16)) + grp);
            pr[2 + e] = __ldcs(reinterpret_cast<const uint32_t*>(a.vp + row * (D / 16)) + grp);
          }
        };
        auto to_l2 = [&](int it) {   // codes of keys and values, their pairs: a warp each
          if (me >= 4 || lane != 0 || it < fresh || it >= w.n) return;
          tile_to_l2<64>(cached_tile(ring, w.t0 + it - f.node_tiles, a.C),
                         me < 2 ? (me ? a.vq : a.kq) + head * (D / 2) : (const uint8_t*)((me == 2 ? a.kp : a.vp) + head * (D / 16)), me < 2 ? D / 2 : D / 8);
        };
        for (int it = 0; it < AHEAD; ++it) to_l2(it);
        fetch(me);
        int x = me;   // this warp's next part
        // Tile by tile, and each warp's arrival belongs to every tile, whether or not it has a part of it: a barrier's phase bit tells a stage that
        // is free from one that is still to be used twice only while no stage is used again before all warps have seen it free. (With arrivals
        // for parts alone a warp without one could find its bit a use too late, and both it and the products wait for good.)
#pragma unroll 1
        for (int it = 0; it < w.n; ++it) {
          const int at = 2 * (tile + it), s = (uint32_t)at % ST;
          if (at >= ST)
            ok = __all_sync(0xffffffffu, wait_bar(bar(L::B_EMPTY + s), ((uint32_t)at / ST - 1) & 1, s_abort, patience) &&
                                             wait_bar(bar(L::B_EMPTY + s + 1), ((uint32_t)at / ST - 1) & 1, s_abort, patience));
          if (!ok) break;
          to_l2(it + AHEAD);
          const uint32_t st = sb + L::OFF_RING + (uint32_t)s * L::KT;
          if (x < (it + 1) * L::ITEMS) {
            const int p = (uint32_t)x % L::ITEMS;
            if (it < fresh) {   // nodes, as the cache would hold them
#pragma unroll 1
              for (int y = lane; y < 2 * 2 * SLOTS * (D / 8); y += 32) {
                const bool v = y >= 2 * SLOTS * (D / 8);
                const int z = y % (2 * SLOTS * (D / 8)), r = p * 2 * SLOTS + z / (D / 8), j = z % (D / 8), k = (w.t0 + it) * 64 + r;
                float h[8];
                load8((const bf16*)(v ? a.v_t : a.k_t) + (((size_t)w.b * a.N + min(k, a.N - 1)) * a.H_kv + w.g) * D + j * 8, h);
                quantize8<D, true>(h, j * 8, nullptr, nullptr, false, 0xffffffffu);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[i] = k < a.N ? held(h[i] * KV_FACTOR) : 0.f;
                sts128(st + (v ? L::KT : 0u) + (uint32_t)(j >> 3) * 8192 + sw128(r, j & 7), halves_in_order(h));
              }
            } else {
              const bool turn = grp >= 2;   // (the second 64 channels: in another order, so that eight threads' stores take different banks)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const GroupScale gs = group_scale(pr[e]);
                const uint32_t word[4] = {turn ? q[e].z : q[e].x, turn ? q[e].w : q[e].y, turn ? q[e].x : q[e].z, turn ? q[e].y : q[e].w};
                const int r = (p * 2 + (e & 1)) * SLOTS + slot;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  sts128(st + (e >> 1) * L::KT + (uint32_t)(grp >> 1) * 8192 + sw128(r, (grp & 1) * 4 + (turn ? i ^ 2 : i)), unpack8(word[i], gs));
              }
            }
            x += L::LOADERS;
            fetch(x);
            fence_proxy_async();
            __syncwarp();
          }
          if (lane == 0) {
            mbar_arrive(bar(L::B_FULL + s));
            mbar_arrive(bar(L::B_FULL + s + 1));
          }
        }
        tile += w.n;
      }
    } else if (elect_one()) {
      int at = 0, seq = 0;
      bool ok = true;
      while (ok && walk.next(f, w)) {
        patience = max(patience, item_limit(f.limit, w.tiles));
        const Ring<64> ring = ring_of<64>(w.pos, a.C, a.W);
        const int qb = seq % q_places;
        if (seq >= q_places) ok = wait_bar(bar(L::B_QE + qb), (seq / q_places - 1) & 1, s_abort, patience);
        if (!ok) break;
        mbar_arrive_expect_tx(bar(L::B_Q + qb), (uint32_t)(q_tiles * (D / 64) * f.tile_rows * 128));
        for (int i = 0; i < q_tiles; ++i)
#pragma unroll
          for (int s = 0; s < D / 64; ++s)
            tma_load_4d(sb + (uint32_t)(qb + i) * L::TILE + s * 16384, &tm_q, bar(L::B_Q + qb), s * 64, w.g * G, quot(w.rb * f.rows + i * f.tile_rows, f.group), w.b);
        ++seq;
        for (int it = w.t0; it < w.t0 + w.n && ok; ++it) {
          const bool fresh = it < f.node_tiles;
          const int s0 = fresh ? it * 64 : cached_tile(ring, it - f.node_tiles, a.C).s0;
#pragma unroll
          for (int v = 0; v < 2; ++v, ++at) {
            const int s = at % ST;
            if (at >= ST) ok = ok && wait_bar(bar(L::B_EMPTY + s), (at / ST - 1) & 1, s_abort, patience);
            if (!ok) break;
            mbar_arrive_expect_tx(bar(L::B_FULL + s), L::KT);
            load_tile<D, 64>(sb + L::OFF_RING + s * L::KT, fresh ? v ? &tm_vt : &tm_kt : v ? &tm_v : &tm_k, bar(L::B_FULL + s), w.g, s0, w.b);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------------------------------------ products
    if (elect_one()) {
      constexpr uint32_t id_s = instr_desc(128, 64, L::FMT, MAJOR_K, MAJOR_K);
      constexpr uint32_t id_o = instr_desc(128, D, L::FMT, MAJOR_K, MAJOR_MN);
      auto stage = [&](int at) { return sb + L::OFF_RING + (uint32_t)(at % ST) * L::KT; };
      auto full = [&](int at) { return wait_bar(bar(L::B_FULL + at % ST), (at / ST) & 1, s_abort, f.limit); };
      int tile = 0, seq = 0, fixed = 0, steps[2] = {0, 0};   // tiles, pieces, those with node tiles, and the warpgroups' products so far
      int qb = 0;
      auto scores = [&](int u, int it, int step, bool first, bool last) {   // first, last: of the warpgroups that meet the tile
        if (first && !full(2 * it)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_f16(s_col(u, step), kdesc<128>(sb + (qb + (two ? u : 0)) * L::TILE, kk), kdesc<64>(stage(2 * it), kk), id_s, kk != 0);
        mma_commit(bar(L::B_S + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + 2 * it % ST));
        return true;
      };
      auto values = [&](int u, int it, int step, bool first, bool last, bool begin) {
        if (first && !full(2 * it + 1)) return false;
        if (!wait_bar(bar(L::B_P + 2 * u + (step & 1)), (step >> 1) & 1, s_abort, patience)) return false;
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) mma_ts(o_col(u), s_col(u, step) + kk * 8, mdesc<64>(stage(2 * it + 1), kk), id_o, !begin || kk != 0);
        mma_commit(bar(L::B_O + 2 * u + (step & 1)));
        if (last) mma_commit(bar(L::B_EMPTY + (2 * it + 1) % ST));
        return true;
      };
      bool ok = true;
      while (ok && walk.next(f, w)) {
        patience = max(patience, item_limit(f.limit, w.tiles));
        const int n = w.n;
        bool fix = w.t0 < f.node_tiles;
        qb = seq % q_places;
        ok = wait_bar(bar(L::B_Q + qb), (seq / q_places) & 1, s_abort, patience);
        if (CAP && ok && fix) {
          ok = wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, patience);
          fix = false;
        }
        if (!ok) break;
        auto outputs_read = [&] { return seq == 0 || wait_bar(bar(L::B_OE), (seq - 1) & 1, s_abort, patience); };
        if (two) {
          ok = scores(0, tile, steps[0], true, false) && scores(1, tile, steps[0], false, true);
          for (int it = 0; it < n && ok; ++it, ++tile, ++steps[0]) {
#pragma unroll
            for (int u = 0; u < 2 && ok; ++u) {
              if (it + 1 < n) ok = scores(u, tile + 1, steps[0] + 1, u == 0, u == 1);
              if (ok && it == 0 && u == 0) ok = outputs_read();
              if (it + 1 == n && u == 1) mma_commit(bar(L::B_QE));   // (the queries' last product)
              if (ok && fix) ok = wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, patience);
              fix = false;
              if (ok) ok = values(u, tile, steps[0], u == 0, u == 1, it == 0);
            }
          }
        } else {
          ok = scores(0, tile, steps[0], true, true) && (n < 2 || scores(1, tile + 1, steps[1], true, true));
          for (int it = 0; it < n && ok; ++it, ++tile) {
            const int u = it & 1;
            if (it + 2 < n) ok = scores(u, tile + 2, steps[u] + 1, true, true);
            if (it + 1 == n) mma_commit(bar(L::B_QE + qb));   // (the queries' last product)
            if (ok && it == 0) ok = outputs_read();
            if (ok && fix) ok = wait_bar(bar(L::B_FIX), fixed++ & 1, s_abort, patience);
            fix = false;
            if (ok) ok = values(u, tile, steps[u], true, true, it < 2);
            ++steps[u];
          }
        }
        if (ok) mma_commit(bar(L::B_DONE));
        ++seq;
      }
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);   // (copies in flight land before the block gives up its shared memory)
    if (tid == 0 && f.dev_status) atomicMax(f.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// a tile of rows: as many whole nodes as 128 rows hold; two of them where there are more
static TreePlan rows_plan(const TreeArgs& a) {
  const int G = a.H / a.H_kv, tile = 128 / G * G;
  return tree_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W, a.N * G > tile ? 2 * tile : tile, tile, 128, 64, 1);
}

template <int D, bool QUANT, bool CAP, bool BIAS>
static int tree_tc(const AttnTree& c) {
  using L = TreeTc<D, QUANT>;
  const TreeArgs& a = c.a;
  const TreePlan p = rows_plan(a);
  if (!p.fits) return LAWCAT_ERR_UNSUPPORTED;
  const TreeTcArgs f = tree_tc_args(c, p);
  const int G = a.H / a.H_kv;
  CUtensorMap tk{}, tv{}, tkt{}, tvt{}, tq{};
  if (!QUANT &&
      (!tensor_map_of(&tk, a.K, a.H_kv, a.C, a.B, D, 1, 64) || !tensor_map_of(&tv, a.V, a.H_kv, a.C, a.B, D, 1, 64) || !tensor_map_of(&tkt, a.k_t, a.H_kv, a.N, a.B, D, 1, 64) ||
      !tensor_map_of(&tvt, a.v_t, a.H_kv, a.N, a.B, D, 1, 64) || !tensor_map_of(&tq, a.q, a.H, a.N, a.B, D, G, 128 / G)))
    return LAWCAT_ERR_CUDA;
  constexpr auto kernel = attn_tree_tc_kernel<D, QUANT, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_tree_tc", c.stream, launch_behind(kernel, dim3((unsigned)f.shares), dim3(L::THREADS), L::BYTES, c.stream, tk, tv, tkt, tvt, tq, f));
  LAWCAT_CHECK_LAUNCH();
  return f.whole ? (int)LAWCAT_OK : launch_tree_join<D, QUANT, 64, true>(c, f);
}

}  // namespace attn

size_t attn_tree_tc_workspace_bytes(const AttnTree& c) {
  return attn::tree_plan_bytes(attn::rows_plan(c.a), c.d);
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

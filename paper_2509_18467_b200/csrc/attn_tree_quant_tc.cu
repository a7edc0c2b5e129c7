// Attention of drafted tokens over a cache in 4 bits on the tensor cores: bf16, d = 64 or 128.
//
// A block of 128 threads walks segments of up to NCOL rows (node, query head) of one (sequence, key-value head) and their keys, in tiles of 128
// slots, one thread per slot, and several blocks share an SM:
//   S^T [128 slots x NCOL] = K Q^T, each thread turns its slot's row into weights, O^T [D channels x NCOL] += V^T P
// A thread unpacks its slot's codes, keys into tensor memory (the first product's A operand), values into shared memory. The weights are
// relative to a reference per row that moves only when a score exceeds it by more than 2^8: one vote of the block per tile, and a maximum
// is looked for only then. Sums stay with the slots' threads until the segment's end.
//
// All operands are fp16: a code becomes 1024 + code by an OR into the mantissa, less 1024, times scale, plus minimum (both times 16), one
// rounding of 2^-11; queries are scaled by a power of two per row. Values beyond 4094 leave fp16's range, and outputs below 2^-18 feel the
// smallest numbers that it holds: such rows, like all that come out not finite, are computed again on the CUDA cores. Channels of eight are
// held in the order 0 4 1 5 2 6 3 7, in which a word of codes unpacks two at a time.
//
// The keys are walked from the newest to the oldest: the nodes' own first, quantized as the cache would hold them, then the cached ones.
// Slots that no row sees, and nodes that are not there, are zeros, whatever they hold.
//
// Rounding: keys, values and weights to fp16 as operands, o once; all else fp32.
#include <algorithm>

#include "attn_tree_tc.cuh"

namespace lawcat {
namespace attn {

constexpr float COL_RESCALE = 8.f, NO_REFERENCE = -1e30f;   // (below every score: the first one that is seen moves it)

__device__ __forceinline__ __half2 as_half2(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
__device__ __forceinline__ uint32_t as_word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
struct GroupScale {
  __half2 s1, s16, low;   // scale, scale / 16, minimum
};
__device__ __forceinline__ GroupScale group_scale(uint32_t pair) {   // (scale, minimum) in bf16
  const float s = bf16_lo(pair) * KV_FACTOR, l = bf16_hi(pair) * KV_FACTOR;
  return GroupScale{__floats2half2_rn(s, s), __floats2half2_rn(s * 0.0625f, s * 0.0625f), __floats2half2_rn(l, l)};
}
// a word of eight codes -> eight values in the order above
__device__ __forceinline__ uint4 unpack8(uint32_t w, const GroupScale& g) {
  const __half2 k = as_half2(0x64006400u);   // 1024
  const uint32_t hi = w >> 8;
  auto val = [&](uint32_t bits, __half2 s) { return as_word(__hfma2(__hsub2(as_half2(bits | 0x64006400u), k), s, g.low)); };
  return make_uint4(val(w & 0x000F000Fu, g.s1), val(w & 0x00F000F0u, g.s16), val(hi & 0x000F000Fu, g.s1), val(hi & 0x00F000F0u, g.s16));
}

template <int D, int NCOL>
struct ColLay {
  static constexpr int NG = D / 32, WPR = D / 8;
  static constexpr uint32_t V = 128 * D * 2, OFF_Q = V, OFF_P = OFF_Q + (D / 64) * NCOL * 128, OFF_COL = OFF_P + (NCOL / 8) * 2048;
  static constexpr uint32_t OFF_ON = OFF_COL + 6 * NCOL * 4, OFF_RED = OFF_ON + NCOL * (TREE_MAX / 32) * 4, OFF_BAR = OFF_RED + 6 * NCOL * 4;
  static constexpr uint32_t BYTES0 = OFF_BAR + 64, BYTES = BYTES0 > 32768u ? BYTES0 : 32768u;   // (D = 64: the product reads 32 KB from V on)
  static constexpr uint32_t K_COLS = D / 2, COLS = K_COLS + 2 * NCOL <= 128 ? 128 : 256;
  static constexpr int RESIDENT = COLS == 128 ? 4 : 2;
  static_assert(K_COLS + 2 * NCOL <= COLS && OFF_P % 1024 == 0 && OFF_BAR % 16 == 0 && sizeof(Paths) <= V && RESIDENT * BYTES <= 232448, "layout");
};

// BIAS: distance biases
template <int D, int NCOL, bool CAP, bool BIAS>
__global__ void __launch_bounds__(128, ColLay<D, NCOL>::RESIDENT) attn_tree_quant_tc_kernel(const __grid_constant__ TreeTcArgs f) {
  using L = ColLay<D, NCOL>;
  constexpr int NG = L::NG, WPR = L::WPR;
  extern __shared__ __align__(1024) uint8_t smem[];
  const TreeArgs& a = f.a;
  const uint32_t sb = smem_u32(smem);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  float* const s_sc = reinterpret_cast<float*>(smem + L::OFF_COL);   // [NCOL / 2] (scale, scale, -reference, -reference) of two columns; CAP: scale without the softmax's
  float* const s_bias = s_sc + 2 * NCOL;                             // [NCOL / 2] (-slope, -slope, -slope depth, -slope depth)
  int* const s_far = reinterpret_cast<int*>(s_bias + 2 * NCOL);      // [NCOL] the farthest key that is seen
  int* const s_depth = s_far + NCOL;
  uint32_t(*const s_on)[TREE_MAX / 32] = reinterpret_cast<uint32_t(*)[TREE_MAX / 32]>(smem + L::OFF_ON);
  float* const s_red = reinterpret_cast<float*>(smem + L::OFF_RED);  // [4][NCOL], then [NCOL] factors, then [NCOL] sums
  float* const s_factor = s_red + 4 * NCOL;
  float* const s_sum = s_factor + NCOL;
  Paths& paths = *reinterpret_cast<Paths*>(smem);                    // (over V, ahead of a segment's tiles)
  volatile int* const s_flags = reinterpret_cast<volatile int*>(smem + L::OFF_BAR + 16);   // tensor memory, abort, rows to be computed again
  volatile int* const s_abort = s_flags + 1;
  uint32_t* const s_bad = const_cast<uint32_t*>(reinterpret_cast<volatile uint32_t*>(s_flags + 2));     // [2]
  uint32_t* const s_large = s_bad + 2;
  const uint32_t bar_s = sb + L::OFF_BAR, bar_o = bar_s + 8;
  const int G = a.H / a.H_kv, R = a.N * G;

  if (tid == 0) {
    mbar_init(bar_s, 1);
    mbar_init(bar_o, 1);
    s_flags[1] = 0;
    mbar_fence_init();
  }
  behind_last_kernel();
  if (warp == 0) {
    tmem_alloc(sb + L::OFF_BAR + 16, L::COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)s_flags[0], k_col = tmem, s_col = tmem + L::K_COLS, o_col = s_col + NCOL, lanes = (uint32_t)(warp * 32) << 16;

  Walk<128> walk;
  walk.start(f, (int)blockIdx.x);
  Piece w;
  int count = 0;   // tiles so far
  bool fail = false;
  while (walk.next(f, w)) {
    const int b = w.b, pos = w.pos, r0 = w.rb * NCOL, n = w.n;
    const Ring<128> ring = ring_of<128>(pos, a.C, a.W);
    const size_t head = ((size_t)b * a.H_kv + w.g) * a.C;
    // this thread's slot of a tile
    uint32_t kc[WPR], vc[WPR], kp[NG], vp[NG];
    auto slot_of = [&](int it, size_t& row) {   // whether any row may see it
      const CachedTile t = cached_tile(ring, it - f.node_tiles, a.C);
      row = head + (t.s0 + tid);
      return tid >= t.lo && t.s0 + tid >= 0 && t.back0 - tid <= ring.cached;
    };
    auto fetch = [&](int it, const uint8_t* q, const bf16* p, uint32_t (&codes)[WPR], uint32_t (&pairs)[NG]) {
      size_t row;
      if (slot_of(it, row)) {
#pragma unroll
        for (int i = 0; i < WPR / 4; ++i) {
          const uint4 x = __ldcs(reinterpret_cast<const uint4*>(q + row * (D / 2)) + i);
          codes[4 * i] = x.x; codes[4 * i + 1] = x.y; codes[4 * i + 2] = x.z; codes[4 * i + 3] = x.w;
        }
        if constexpr (NG == 4) {
          const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p + row * (2 * NG)));
          pairs[0] = x.x; pairs[1] = x.y; pairs[2] = x.z; pairs[3] = x.w;
        } else {
          const uint2 x = __ldcs(reinterpret_cast<const uint2*>(p + row * (2 * NG)));
          pairs[0] = x.x; pairs[1] = x.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < WPR; ++i) codes[i] = 0u;
#pragma unroll
        for (int i = 0; i < NG; ++i) pairs[i] = 0u;
      }
    };
    // a node's row as the cache would hold it
    auto hold = [&](const void* src, bool some, int node, uint32_t (&codes)[WPR], uint32_t (&pairs)[NG]) {
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        pairs[i] = codes[4 * i] = codes[4 * i + 1] = codes[4 * i + 2] = codes[4 * i + 3] = 0u;
        if (!some) continue;
        const bf16* const p = (const bf16*)src + (((size_t)b * a.N + node) * a.H_kv + w.g) * D + i * 32;
        float x[32];
#pragma unroll
        for (int j = 0; j < 32; j += 8) {
          float y[8];
          load8(p + j, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[j + e] = y[e];
        }
        float lo = x[0], hi = x[0], scale, low;
#pragma unroll
        for (int j = 1; j < 32; ++j) {
          lo = min_nan(lo, x[j]);
          hi = max_nan(hi, x[j]);
        }
        quant_params(lo, hi, isfinite(lo) && isfinite(hi), scale, low);
        const float inv = __frcp_rn(scale);
#pragma unroll
        for (int j = 0; j < 32; ++j) codes[4 * i + j / 8] |= code_bits(quant_code(x[j], scale, low, inv)) << (4 * (j & 7));
        pairs[i] = pack_bf16(scale, low);
      }
    };
    if (w.t0 >= f.node_tiles) {
      fetch(w.t0, a.kq, a.kp, kc, kp);
      fetch(w.t0, a.vq, a.vp, vc, vp);
    }

    // ------------------------------------------------------------------------------------------------ rows
    find_paths<128>(a, b, paths, tid, 1);
    int my_depth[TREE_MAX / 128];   // of this thread's nodes
#pragma unroll
    for (int i = 0; i < TREE_MAX / 128; ++i) my_depth[i] = pos >= 0 && tid + 128 * i < a.N ? node_depth(paths, tid + 128 * i, a.N) : -1;
    if (tid < NCOL) {
      const int r = min(r0 + tid, R - 1), node = quot(r, f.group), h = w.g * G + rest(r, node, f.group);
      const int depth = pos >= 0 && r0 + tid < R ? node_depth(paths, node, a.N) : -1;
      const float slope = BIAS ? a.slopes[h] * LOG2E : 0.f;
      s_depth[tid] = depth;
      s_far[tid] = depth >= 0 ? min(a.W - 1 - depth, pos) : 0x3fffffff;   // (rows that are not there weigh zeros, and are stored as zeros)
      const int at = tid / 2 * 4 + (tid & 1);
      s_sc[at + 2] = depth >= 0 ? -NO_REFERENCE : 0.f;
      s_bias[at] = depth >= 0 ? -slope : 0.f;
      s_bias[at + 2] = depth >= 0 ? -slope * (float)depth : 0.f;
#pragma unroll
      for (int i = 0; i < TREE_MAX / 32; ++i) s_on[tid][i] = depth >= 0 ? paths.on[node][i] : 0u;
    }
    if (tid == 0) {
      s_bad[0] = s_bad[1] = s_large[0] = s_large[1] = 0u;
    }
    named_bar_sync(1, 128);
#pragma unroll 2
    for (int i = tid; i < NCOL * (D / 8); i += 128) {
      const int c = i / (D / 8), j = i % (D / 8), r = min(r0 + c, R - 1), node = quot(r, f.group);
      uint4 q = make_uint4(0u, 0u, 0u, 0u);
      if (s_depth[c] >= 0) q = *reinterpret_cast<const uint4*>((const bf16*)a.q + (((size_t)b * a.N + node) * a.H + w.g * G + rest(r, node, f.group)) * D + j * 8);
      float x[8] = {bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y), bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w)};
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
      for (int o = 1; o < D / 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));   // (a row's threads lie side by side)
      const uint32_t e2 = min(max(top >> 23, 1u), 253u);   // largest value in [1, 2)
      const float down = __uint_as_float((254u - e2) << 23);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= down;
      sts128(sb + L::OFF_Q + (uint32_t)(j >> 3) * (NCOL * 128) + sw128(c, j & 7), make_uint4(pack_f16(x[0], x[4]), pack_f16(x[1], x[5]), pack_f16(x[2], x[6]), pack_f16(x[3], x[7])));
      if (j == 0) s_sc[c / 2 * 4 + (c & 1)] = (CAP ? 1.f : a.scale * LOG2E) * (s_depth[c] >= 0 ? __uint_as_float(e2 << 23) / KV_FACTOR : 0.f);
    }
    fence_proxy_async();
    named_bar_sync(1, 128);
    int far_all = s_far[lane % NCOL];
    if (NCOL == 64) far_all = min(far_all, s_far[lane + 32]);
    far_all = __reduce_min_sync(0xffffffffu, far_all);
    float l[NCOL];
#pragma unroll
    for (int c = 0; c < NCOL; ++c) l[c] = 0.f;

    // ------------------------------------------------------------------------------------------------ tiles
    for (int i = 0; i < n; ++i, ++count) {
      const int it = w.t0 + i;
      const bool fresh = it < f.node_tiles;
      if (fresh) {
        const int node = it * 128 + tid;
        int depth = my_depth[0];
#pragma unroll
        for (int e = 1; e < TREE_MAX / 128; ++e) depth = it == e ? my_depth[e] : depth;
        hold(a.k_t, depth >= 0, node, kc, kp);
        hold(a.v_t, depth >= 0, node, vc, vp);
      }
#pragma unroll
      for (int s = 0; s < D / 64; ++s) {
        float x[32];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4 y = unpack8(kc[8 * s + e], group_scale(kp[2 * s + e / 4]));
          x[4 * e] = __uint_as_float(y.x); x[4 * e + 1] = __uint_as_float(y.y); x[4 * e + 2] = __uint_as_float(y.z); x[4 * e + 3] = __uint_as_float(y.w);
        }
        tmem_st32(k_col + lanes + 32 * s, x);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      named_bar_sync(2, 128);
      if (warp == 0 && elect_one()) {
        constexpr uint32_t id_s = instr_desc(128, NCOL, FMT_F16, MAJOR_K, MAJOR_K);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) mma_ts(s_col, k_col + kk * 8, kdesc<NCOL>(sb + L::OFF_Q, kk), id_s, kk != 0);
        mma_commit(bar_s);
      }
      __syncwarp();
      const bool more = i + 1 < n && it + 1 >= f.node_tiles;
      if (more) fetch(it + 1, a.kq, a.kp, kc, kp);
      // (values and weights of the tile in front have been read)
      if (i > 0 && !fail) fail = !wait_bar(bar_o, (count - 1) & 1, s_abort, f.limit);
      __syncwarp();
#pragma unroll
      for (int e = 0; e < WPR; ++e) sts128(sb + (uint32_t)(e >> 3) * 16384 + sw128(tid, e & 7), unpack8(vc[e], group_scale(vp[e / 4])));
      if (more) fetch(it + 1, a.vq, a.vp, vc, vp);
      if (!fail) fail = !wait_bar(bar_s, count & 1, s_abort, f.limit);
      __syncwarp();
      tc_fence_after_sync();

      CachedTile t{0, 0, 0};
      if (!fresh) t = cached_tile(ring, it - f.node_tiles, a.C);
      const int back = t.back0 - tid;
      const bool whole = !fresh && t.back0 <= far_all && t.lo == 0;   // every row sees every slot
      float z[NCOL];
      // scores in log2 units, less the references (or not)
      auto scores = [&](bool relative) {
#pragma unroll
        for (int c = 0; c < NCOL; c += 16) tmem_ld16(s_col + lanes + c, z + c);
        tmem_wait_ld();
        if constexpr (CAP) {
#pragma unroll
          for (int c = 0; c < NCOL; ++c) z[c] *= s_sc[c / 2 * 4 + (c & 1)];
          cap_scores(z, a.scale / a.cap, a.cap * LOG2E);
        }
        const float d = fresh ? 0.f : (float)back;
        const uint64_t back2 = f2_pack(d, d);
#pragma unroll
        for (int c = 0; c < NCOL; c += 2) {
          const float4 k = *reinterpret_cast<const float4*>(s_sc + 2 * c);
          uint64_t add = relative ? f2_pack(k.z, k.w) : 0ull;
          if constexpr (BIAS) {
            const float4 e = *reinterpret_cast<const float4*>(s_bias + 2 * c);
            add = f2_add(add, f2_fma(f2_pack(e.x, e.y), back2, f2_pack(e.z, e.w)));
          }
          const uint64_t x = f2_pack(z[c], z[c + 1]);
          f2_unpack(CAP ? f2_add(x, add) : f2_fma(x, f2_pack(k.x, k.y), add), z[c], z[c + 1]);
        }
        if (!whole) {
          if (fresh) {   // nodes of the row's path, by their distance
            const int j = it * 128 + tid;
            int mine = my_depth[0];
#pragma unroll
            for (int e = 1; e < TREE_MAX / 128; ++e) mine = it == e ? my_depth[e] : mine;
#pragma unroll
            for (int c = 0; c < NCOL; ++c) {
              const bool see = (s_on[c][j >> 5] >> (j & 31) & 1u) && s_depth[c] - mine < a.W;
              if constexpr (BIAS) z[c] -= s_bias[c / 2 * 4 + (c & 1)] * (float)mine;   // (back = -depth)
              z[c] = see ? z[c] : -INFINITY;
            }
          } else {
#pragma unroll
            for (int c = 0; c < NCOL; ++c) z[c] = back <= s_far[c] && tid >= t.lo ? z[c] : -INFINITY;
          }
        }
      };
      scores(true);
      float mx0 = z[0], mx1 = z[1];
#pragma unroll
      for (int c = 2; c < NCOL; c += 2) {
        mx0 = fmaxf(mx0, z[c]);
        mx1 = fmaxf(mx1, z[c + 1]);
      }
      if (named_bar_or(3, 128, fmaxf(mx0, mx1) > COL_RESCALE || fail)) {
        // new references: the block's maximum of each row
        if (named_bar_or(3, 128, fail)) break;
        scores(false);
#pragma unroll
        for (int c = 0; c < NCOL; ++c) {
          const float x = warp_max(z[c]);
          if (lane == 0) s_red[warp * NCOL + c] = x;
        }
        named_bar_sync(3, 128);
        if (tid < NCOL) {
          const float x = fmaxf(fmaxf(s_red[tid], s_red[NCOL + tid]), fmaxf(s_red[2 * NCOL + tid], s_red[3 * NCOL + tid]));
          float& neg = s_sc[tid / 2 * 4 + 2 + (tid & 1)];
          const bool grow = x > -neg + COL_RESCALE;
          s_factor[tid] = grow ? ex2f(-neg - x) : 1.f;
          if (grow) neg = -x;
        }
        named_bar_sync(3, 128);
#pragma unroll
        for (int c = 0; c < NCOL; ++c) l[c] *= s_factor[c];
        if (i > 0) {
#pragma unroll
          for (int c = 0; c < NCOL; c += 16) {
            float o[16];
            tmem_ld16(o_col + lanes + c, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= s_factor[c + e];
            tmem_st16(o_col + lanes + c, o);
          }
          tmem_wait_st();
        }
        scores(true);
      }
#pragma unroll
      for (int c = 0; c < NCOL; c += 8) {
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = ex2f(z[c + 2 * e]), y = ex2f(z[c + 2 * e + 1]);
          l[c + 2 * e] += x;
          l[c + 2 * e + 1] += y;
          p[e] = pack_f16(x, y);
        }
        sts128(sb + L::OFF_P + (uint32_t)(c / 8) * 2048 + tid * 16, make_uint4(p[0], p[1], p[2], p[3]));
      }
      fence_proxy_async();
      tc_fence_before_sync();
      named_bar_sync(4, 128);
      if (warp == 0 && elect_one()) {
        constexpr uint32_t id_o = instr_desc(128, NCOL, FMT_F16, MAJOR_MN, MAJOR_MN);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) mma_f16(o_col, mdesc<128>(sb, kk), smem_desc(sb + L::OFF_P + kk * 256, 128, 2048, LAYOUT_NONE), id_o, (i | kk) != 0);
        mma_commit(bar_o);
      }
      __syncwarp();
    }

    // ------------------------------------------------------------------------------------------------ outputs
    if (!fail) fail = !wait_bar(bar_o, (count - 1) & 1, s_abort, f.limit);
    if (named_bar_or(3, 128, fail)) break;
    tc_fence_after_sync();
#pragma unroll
    for (int c = 0; c < NCOL; ++c) {
      const float x = warp_sum(l[c]);
      if (lane == 0) s_red[warp * NCOL + c] = x;
    }
    named_bar_sync(3, 128);
    const bool direct = is_whole(w);
    const size_t slot = piece_slot(w, (int)blockIdx.x);
    if (tid < NCOL) {
      float sum = s_red[tid] + s_red[NCOL + tid] + s_red[2 * NCOL + tid] + s_red[3 * NCOL + tid];
      if (s_depth[tid] < 0) sum = 0.f;
      s_sum[tid] = sum;
      const float m = -s_sc[tid / 2 * 4 + 2 + (tid & 1)];
      if (!direct && r0 + tid < R) f.part_ml[slot * f.rows_pad + tid] = make_float2(sum == 0.f ? -INFINITY : m, sum);
    }
    named_bar_sync(3, 128);
    float o[NCOL];
#pragma unroll
    for (int c = 0; c < NCOL; c += 16) tmem_ld16(o_col + lanes + c, o + c);
    tmem_wait_ld();
    const int ch = (tid & ~7) + ((tid & 7) >> 1) + 4 * (tid & 1);   // the lane's channel
#pragma unroll
    for (int c = 0; c < NCOL; ++c) {
      const int r = r0 + c;
      if (r >= R) break;
      const float sum = s_sum[c];
      if (!direct) {
        if (tid < D) f.part_o[(slot * f.rows_pad + c) * D + ch] = o[c] * (1.f / KV_FACTOR);
      } else {
        const float y = sum == 0.f ? 0.f : o[c] / (sum * KV_FACTOR);
        const int node = quot(r, f.group);
        if (tid < D) ((bf16*)a.o)[(((size_t)b * a.N + node) * a.H + w.g * G + rest(r, node, f.group)) * D + ch] = __float2bfloat16_rn(y);
        const uint32_t bad = __ballot_sync(0xffffffffu, tid < D && !isfinite(y)), large = __ballot_sync(0xffffffffu, tid < D && !(fabsf(y) < SMALL));
        if (lane == 0) {
          if (bad) atomicOr(s_bad + c / 32, 1u << (c & 31));
          if (large || sum == 0.f) atomicOr(s_large + c / 32, 1u << (c & 31));
        }
      }
    }
    tc_fence_before_sync();
    named_bar_sync(3, 128);
    if (direct) {
#pragma unroll 1
      for (int c = warp; c < NCOL && r0 + c < R; c += 4)
        if ((s_bad[c / 32] | ~s_large[c / 32]) >> (c & 31) & 1u) {
          const int node = quot(r0 + c, f.group);
          tree_row_again<bf16, D, true>(a, b, node, w.g * G + rest(r0 + c, node, f.group));
        }
      named_bar_sync(3, 128);   // (the flags have been read)
    }
  }
  __syncthreads();
  if (*s_abort) {
    for (int i = 0; i < 100; ++i) __nanosleep(1000);
    if (tid == 0 && f.dev_status) atomicMax(f.dev_status, (int)LAWCAT_ERR_TIMEOUT);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, L::COLS);
}

static int columns(int N, int H, int H_kv) {
  const int R = N * (H / H_kv);
  return R <= 16 ? 16 : R <= 32 ? 32 : 64;
}
template <int NCOL>
static TreePlan cols_plan(const AttnTree& c) {
  const TreeArgs& a = c.a;
  return tree_plan(a.B, a.N, a.H, a.H_kv, a.C, a.W, NCOL, 128, ColLay<128, NCOL>::RESIDENT);
}

template <int D, int NCOL, bool CAP, bool BIAS>
static int tree_quant_tc(const AttnTree& c) {
  using L = ColLay<D, NCOL>;
  const TreeTcArgs f = tree_tc_args(c, cols_plan<NCOL>(c));
  constexpr auto kernel = attn_tree_quant_tc_kernel<D, NCOL, CAP, BIAS>;
  if (int r = grant_smem<kernel>(L::BYTES)) return r;
  LAWCAT_LAUNCH("attn_tree_quant_tc", c.stream, launch_behind(kernel, dim3((unsigned)f.shares), dim3(128), L::BYTES, c.stream, f));
  LAWCAT_CHECK_LAUNCH();
  return f.whole ? (int)LAWCAT_OK : launch_tree_join<D, true, 128, false>(c, f);
}

}  // namespace attn

size_t attn_tree_quant_tc_workspace_bytes(const AttnTree& c) {
  const int n = attn::columns(c.a.N, c.a.H, c.a.H_kv);
  return attn::tree_plan_bytes(n == 16 ? attn::cols_plan<16>(c) : n == 32 ? attn::cols_plan<32>(c) : attn::cols_plan<64>(c), c.d);
}

int launch_attn_tree_quant_tc(const AttnTree& c) {
  const int n = attn::columns(c.a.N, c.a.H, c.a.H_kv);
  auto by = [&](auto cap, auto bias) {
    constexpr bool CAP = decltype(cap)::value, BIAS = decltype(bias)::value;
    if (c.d == 128) return n == 16 ? attn::tree_quant_tc<128, 16, CAP, BIAS>(c) : n == 32 ? attn::tree_quant_tc<128, 32, CAP, BIAS>(c) : attn::tree_quant_tc<128, 64, CAP, BIAS>(c);
    return n == 16 ? attn::tree_quant_tc<64, 16, CAP, BIAS>(c) : n == 32 ? attn::tree_quant_tc<64, 32, CAP, BIAS>(c) : attn::tree_quant_tc<64, 64, CAP, BIAS>(c);
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (c.a.cap > 0.f) return c.a.slopes ? by(yes, yes) : by(yes, no);
  return c.a.slopes ? by(no, yes) : by(no, no);
}

}  // namespace lawcat

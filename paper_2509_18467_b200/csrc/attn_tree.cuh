// Attention of drafted tokens over a cache: what its kernels share.
//
// Row r = node * G + (query head of the group) of a (sequence, key-value head): all rows of a group read the same keys. The keys of a
// sequence are its nodes' own and the cached ones, counted by how far they lie in front of position pos: back = 1 ... n, slot (pos - back) mod C.
// A node of depth e sees a cached key where back + e < W, and a node of its path where the depths differ by less than W.
#pragma once
#include "attn_rows.cuh"

namespace lawcat {
namespace attn {

constexpr int TREE_MAX = 256;   // nodes of a sequence

struct TreeArgs {
  const void *q, *k_t, *v_t;        // [B, N, H, D], [B, N, H_kv, D]
  const void *K, *V;                // [B, C, H_kv, D] in the storage type (not in the 4-bit form)
  const uint8_t *kq, *vq;           // [B, H_kv, C, D / 2]
  const bf16 *kp, *vp;              // [B, H_kv, C, groups, 2]
  const int *pos, *parent;          // [B], [B, N] or null: a chain
  const float* slopes;
  void* o;                          // [B, N, H, D]
  float* part;                      // [B, N, H, parts, D + 2] (maximum in log2 units, sum, weighted values) where parts > 1
  int B, N, H, H_kv, C, W, parts;   // W: the window, or C
  float scale, cap;
};

// cached keys that the least deep node sees
__device__ __forceinline__ int cached_keys(int pos, int W) { return pos < 0 ? 0 : min(pos, W - 1); }

// The nodes of a sequence, in shared memory: the path of each (itself included) as bits, none where it is not there; depth = bits - 1.
struct Paths {
  uint32_t on[TREE_MAX][TREE_MAX / 32];
  int up[TREE_MAX];
};
// Paths by doubling: after step k a node's bits are its nearest 2^k ancestors, `up` the next one. By THREADS threads (their numbers `tid`,
// a named barrier of theirs), which find everything behind the barrier that it ends with.
template <int THREADS>
__device__ __forceinline__ void find_paths(const TreeArgs& a, int b, Paths& s, int tid, int barrier) {
  constexpr int PER = TREE_MAX / THREADS, WORDS = TREE_MAX / 32;
  int up[PER];
  bool climb = false;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int i = tid + p * THREADS;
    up[p] = -1;
    if (i >= a.N) continue;
    up[p] = i - 1;
    if (a.parent) {
      up[p] = a.parent[(size_t)b * a.N + i];
      if (up[p] < -1 || up[p] >= i) up[p] = -2;
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      uint32_t bits = w == i / 32 ? 1u << (i & 31) : 0u;
      if (!a.parent) bits = w < i / 32 ? 0xffffffffu : w == i / 32 ? 0xffffffffu >> (31 - (i & 31)) : 0u;   // (a chain: all in front)
      s.on[i][w] = bits;
    }
    s.up[i] = up[p];
    climb = climb || up[p] >= 0;
  }
  if (a.parent) {
    const int words = (a.N + 31) / 32;
    while (tc::named_bar_or(barrier, THREADS, climb)) {   // (at most eight times: distances double)
      uint32_t more[PER][WORDS];
      int next[PER];
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        next[p] = up[p];
        if (up[p] < 0) continue;
        next[p] = s.up[up[p]];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) more[p][w] = w < words ? s.on[up[p]][w] : 0u;
      }
      tc::named_bar_sync(barrier, THREADS);
      climb = false;
#pragma unroll
      for (int p = 0; p < PER; ++p) {
        if (up[p] < 0) continue;
        const int i = tid + p * THREADS;
#pragma unroll
        for (int w = 0; w < WORDS; ++w)
          if (w < words) s.on[i][w] |= more[p][w];
        s.up[i] = up[p] = next[p];
        climb = climb || up[p] >= 0;
      }
    }
#pragma unroll
    for (int p = 0; p < PER; ++p)
      if (up[p] == -2)
#pragma unroll
        for (int w = 0; w < WORDS; ++w) s.on[tid + p * THREADS][w] = 0u;
  }
  tc::named_bar_sync(barrier, THREADS);
}
__device__ __forceinline__ int node_depth(const Paths& s, int i, int N) {
  int n = -1;
  for (int w = 0; w < (N + 31) / 32; ++w) n += __popc(s.on[i][w]);
  return n;
}

__device__ __forceinline__ float tree_score(const TreeArgs& a, float dot, float slope, int dist) {
  float x = dot * a.scale;
  if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
  return (x - slope * (float)dist) * LOG2E;
}

// one group of channels of a row, as the step reads it: `node` >= 0 a node's own row, else the slot's
template <typename T, int D, bool QUANT>
__device__ __forceinline__ void row_group(const TreeArgs& a, bool v, int b, int g, int node, size_t slot, int c0, float (&x)[quant_group(D)]) {
  constexpr int GS = quant_group(D);
  if (node >= 0 || !QUANT) {
    const T* src = node >= 0 ? (const T*)(v ? a.v_t : a.k_t) + (((size_t)b * a.N + node) * a.H_kv + g) * D + c0
                             : (const T*)(v ? a.V : a.K) + (((size_t)b * a.C + slot) * a.H_kv + g) * D + c0;
#pragma unroll 1
    for (int i = 0; i < GS; ++i) x[i] = ldf<T>(src + i);
    if (!QUANT) return;
    float lo = x[0], hi = x[0], scale, low;
#pragma unroll 1
    for (int i = 1; i < GS; ++i) {
      lo = min_nan(lo, x[i]);
      hi = max_nan(hi, x[i]);
    }
    quant_params(lo, hi, isfinite(lo) && isfinite(hi), scale, low);
    const float inv = __frcp_rn(scale);
#pragma unroll 1
    for (int i = 0; i < GS; ++i) x[i] = fmaf((float)code_bits(quant_code(x[i], scale, low, inv)), scale, low);
  } else {
    const size_t row = ((size_t)b * a.H_kv + g) * a.C + slot;
    const uint8_t* q = (v ? a.vq : a.kq) + row * (D / 2) + c0 / 2;
    const bf16* p = (v ? a.vp : a.kp) + (row * (D / GS) + c0 / GS) * 2;
    const float scale = __bfloat162float(p[0]), low = __bfloat162float(p[1]);
#pragma unroll 1
    for (int i = 0; i < GS; ++i) x[i] = fmaf((float)(q[i / 2] >> (4 * (i & 1)) & 15), scale, low);
  }
}

// One row by one warp, from the keys that it sees alone, 32 at a time: a lane's key for the scores, all lanes' channels for the values.
// (c_first, channels: those that are stored.)
template <typename T, int D, bool QUANT>
__device__ __noinline__ void tree_row_again(const TreeArgs& a, int b, int node, int h, int c_first = 0, int channels = D) {
  constexpr int NC = D / 32 > 0 ? D / 32 : 1, GS = quant_group(D);
  const int lane = threadIdx.x & 31, g = h / (a.H / a.H_kv), pos = a.pos[b];
  const size_t row = ((size_t)b * a.N + node) * a.H + h;
  const T* const q = (const T*)a.q + row * D;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  int depth = 0;
  bool there = pos >= 0;
  for (int i = node; there && i >= 0;) {
    const int p = a.parent ? a.parent[(size_t)b * a.N + i] : i - 1;
    there = p >= -1 && p < i;
    depth += p >= 0;
    i = p;
  }
  const int cached = there ? max(0, min(cached_keys(pos, a.W), a.W - 1 - depth)) : 0;
  const int path = there ? min(depth + 1, a.W) : 0;       // nodes of the path that are near enough, from the row's own on
  float m = -INFINITY, l = 0.f, acc[NC] = {};
  int next = node;                                        // the path's next node
  for (int k0 = 0; k0 < path + cached; k0 += 32) {
    const int k = k0 + lane;
    int mine = -1, dist = k;
    for (int i = 0; i < 32 && k0 + i < path; ++i) {       // (all lanes walk, one keeps)
      if (i == lane) mine = next;
      next = a.parent ? a.parent[(size_t)b * a.N + next] : next - 1;
    }
    size_t slot = 0;
    if (k >= path) {
      const int back = k - path + 1;
      dist = depth + back;
      int s = pos % a.C - back % a.C;
      slot = s < 0 ? s + a.C : s;
    }
    float x = -INFINITY;
    if (k < path + cached) {
      float d = 0.f, u[GS];
      for (int c = 0; c < D; c += GS) {
        row_group<T, D, QUANT>(a, false, b, g, mine, slot, c, u);
        for (int i = 0; i < GS; ++i) d = fmaf(ldf<T>(q + c + i), u[i], d);
      }
      x = tree_score(a, d, slope, dist);
    }
    const float mx = fmaxf(m, warp_max(x)), base = mx == -INFINITY ? 0.f : mx, f = exp2f(m - base);
    const float p = k < path + cached ? exp2f(x - base) : 0.f;
    l = l * f + warp_sum(p);
    m = mx;
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[c] *= f;
    for (int i = 0; i < 32 && k0 + i < path + cached; ++i) {
      const float w = __shfl_sync(0xffffffffu, p, i);
      const int n = __shfl_sync(0xffffffffu, mine, i);
      const size_t s = __shfl_sync(0xffffffffu, (unsigned long long)slot, i);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float y;
        const int ch = D >= 32 ? lane + 32 * c : lane % D;
        if (n >= 0 || !QUANT) {
          y = ldf<T>(n >= 0 ? (const T*)a.v_t + (((size_t)b * a.N + n) * a.H_kv + g) * D + ch : (const T*)a.V + (((size_t)b * a.C + s) * a.H_kv + g) * D + ch);
          if (QUANT) {
            float lo = y, hi = y, scale, low;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {            // (a group is a warp's channels, at width 16 twice the same)
              lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
              hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
            }
            quant_params(lo, hi, isfinite(lo) && isfinite(hi), scale, low);
            y = fmaf((float)code_bits(quant_code(y, scale, low, __frcp_rn(scale))), scale, low);
          }
        } else {
          const size_t r = ((size_t)b * a.H_kv + g) * a.C + s;
          const bf16* pr = a.vp + (r * (D / GS) + ch / GS) * 2;
          y = fmaf((float)(a.vq[r * (D / 2) + ch / 2] >> (4 * (ch & 1)) & 15), __bfloat162float(pr[0]), __bfloat162float(pr[1]));
        }
        acc[c] = fmaf(w, y, acc[c]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (lane + 32 * c < D && lane + 32 * c >= c_first && lane + 32 * c < c_first + channels) stf<T>((T*)a.o + row * D + lane + 32 * c, l == 0.f ? 0.f : acc[c] * inv);
}

}  // namespace attn

// a call's arguments (attn_tree.cu)
struct AttnTree {
  attn::TreeArgs a;
  int d, dtype, exact;
  void* ws;
  int* dev_status;
  cudaStream_t stream;
};
int launch_attn_tree_join(const AttnTree& c);
// the tensor-core kernels (attn_tree_tc.cu): bf16 storage, d = 64 or 128
size_t attn_tree_tc_workspace_bytes(const AttnTree& c);
int launch_attn_tree_tc(const AttnTree& c);
// the same over 4 bits (attn_tree_quant_tc.cu)
size_t attn_tree_quant_tc_workspace_bytes(const AttnTree& c);
int launch_attn_tree_quant_tc(const AttnTree& c);

}  // namespace lawcat

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
// Paths by doubling: after step k a node's bits are its nearest 2^k ancestors, `up` the next one. All threads of a block of at least
// TREE_MAX threads; ends with a barrier.
__device__ __forceinline__ void find_paths(const TreeArgs& a, int b, Paths& s) {
  const int i = threadIdx.x, words = (a.N + 31) / 32;
  int up = -1;
  if (i < a.N) {
    up = i - 1;
    if (a.parent) {
      up = a.parent[(size_t)b * a.N + i];
      if (up < -1 || up >= i) up = -2;
    }
    for (int w = 0; w < words; ++w) {
      uint32_t bits = w == i / 32 ? 1u << (i & 31) : 0u;
      if (!a.parent) bits = w < i / 32 ? 0xffffffffu : w == i / 32 ? 0xffffffffu >> (31 - (i & 31)) : 0u;   // (a chain: all in front)
      s.on[i][w] = bits;
    }
    s.up[i] = up;
  }
  if (a.parent) {
    while (__syncthreads_or(i < a.N && up >= 0)) {   // (at most eight times: distances double)
      uint32_t more[TREE_MAX / 32];
      int next = up;
      if (up >= 0 && i < a.N) {
        next = s.up[up];
#pragma unroll
        for (int w = 0; w < TREE_MAX / 32; ++w) more[w] = w < words ? s.on[up][w] : 0u;
      }
      __syncthreads();
      if (up >= 0 && i < a.N) {
#pragma unroll
        for (int w = 0; w < TREE_MAX / 32; ++w)
          if (w < words) s.on[i][w] |= more[w];
        s.up[i] = up = next;
      }
    }
    if (i < a.N && up == -2)
      for (int w = 0; w < words; ++w) s.on[i][w] = 0u;
  }
  __syncthreads();
}
__device__ __forceinline__ int node_depth(const Paths& s, int i, int N) {
  int n = -1;
  for (int w = 0; w < (N + 31) / 32; ++w) n += __popc(s.on[i][w]);
  return n;
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

}  // namespace lawcat

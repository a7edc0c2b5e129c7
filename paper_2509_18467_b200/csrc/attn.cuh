// Softmax attention beside the linearized layer: what its kernels share.
//   u = scale q.k,  s = cap tanh(u / cap) (cap > 0),  x = s - slope_h |i - j|,  p = softmax(x),  o = p v
// Every mask offered (causal, window, documents, prefix, T != T_k) leaves a query ONE interval of keys [lo, hi), and both ends
// grow with the query; the kernels know nothing else of masks.
#pragma once
#include <atomic>

#include "common.cuh"

namespace lawcat {
namespace attn {

// Every kernel here is launched behind the kernel in front of it on the stream (launch_behind): its launch overlaps that one's end.
// Before the first access to memory, and before tensor memory is taken, which the kernel in front may still be waiting for.
// (512 tokens, 4 heads of 64 in fp32, forward and gradients, six kernels: 79 us without, 69 us so; a step over 32768 slots in 4 bits and its join 39 and 32;
// 77 queries over 8192 keys and their join 37 and 33. With a trigger at the start of kernels that share out their work, 72, 32 and 37.)
__device__ __forceinline__ void behind_last_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

struct Mask {
  int T, T_k;
  int off;           // position of query t: t + off  (T_k - T)
  int causal, window;
  const int2* rows;  // [B, T] (lo, hi) where documents or prefixes are given, else null
  const int2* keys;  // [B, T_k] the other way round, for the gradients (see key_interval)
};

__host__ __device__ __forceinline__ int2 interval(const Mask& m, int b, int t) {
#ifdef __CUDA_ARCH__
  if (m.rows) return __ldg(m.rows + (size_t)b * m.T + t);
#endif
  const int pos = t + m.off;
  int lo = 0, hi = m.T_k;
  if (m.causal) hi = pos + 1 < m.T_k ? pos + 1 : m.T_k;
  if (m.window) {
    if (pos - m.window + 1 > 0) lo = pos - m.window + 1;
    if (pos < m.T_k - m.window) hi = hi < pos + m.window ? hi : pos + m.window;
  }
  return make_int2(lo, hi > lo ? hi : lo);
}

// The other way round: the queries that see key j, one interval as well since both ends of the queries' intervals grow with the
// query. prefix: the keys below it are seen by every query.
__host__ __device__ __forceinline__ int2 key_interval(const Mask& m, int b, int j, int prefix = 0) {
#ifdef __CUDA_ARCH__
  if (m.keys) return __ldg(m.keys + (size_t)b * m.T_k + j);
#endif
  int first = 0, end = m.T;  // (query t has position t + off)
  if (m.causal) {
    if (j >= prefix) first = j - m.off;
  } else if (m.window) {
    first = j - m.off - m.window + 1;
  }
  if (m.window && j - m.off < m.T - m.window) end = j - m.off + m.window;
  first = first < 0 ? 0 : first > m.T ? m.T : first;
  return make_int2(first, end > first ? end : first);
}

// Queries that may see one of the keys [j0, j1): the first with hi > j0 up to the first with lo >= j1 (both ends of the
// intervals grow with t). Called by all threads with the same arguments.
__device__ __forceinline__ int2 queries_of(const Mask& m, int b, int j0, int j1) {
  int l = 0, h = m.T;
  while (l < h) {
    const int mid = (l + h) >> 1;
    if (interval(m, b, mid).y > j0) h = mid; else l = mid + 1;
  }
  const int first = l;
  h = m.T;
  while (l < h) {
    const int mid = (l + h) >> 1;
    if (interval(m, b, mid).x >= j1) h = mid; else l = mid + 1;
  }
  return make_int2(first, l);
}

struct Args {
  const void *q, *k, *v, *dO;
  const void* o_in;
  void *o, *dq, *dk, *dv;
  float* lse;           // [B, T, H] natural logarithm (forward: output; backward: input)
  const float* slopes;  // [H] or null
  float* stat;          // backward: [2, B, H, stat_stride]: -lse log2e, then -D, D = sum_j p_j dO.v_j
  int stat_stride;      // T rounded up to 64
  Mask mask;
  int B, H, H_kv;
  float scale, cap;
  int* dev_status;
};

}  // namespace attn

// Dynamic shared memory of a kernel, granted once per device (the call costs a microsecond, a decode step's launch not many more).
template <auto KERNEL>
int grant_smem(size_t bytes) {
  static std::atomic<unsigned long long> granted{0};
  int dev = 0;
  const bool known = cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 64;
  if (known && (granted.load(std::memory_order_relaxed) >> dev & 1)) return LAWCAT_OK;
  const cudaError_t e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) {
    cudaGetLastError();
    note_cuda_error(e, __FILE__, __LINE__);
    return LAWCAT_ERR_CUDA;
  }
  if (known) granted.fetch_or(1ull << dev, std::memory_order_relaxed);
  return LAWCAT_OK;
}

// a call's arguments, its launchers and scratch
struct AttnCall {
  attn::Args a;
  const int32_t *cu, *prefix;  // HOST arrays of the documents (or null), read during the call alone
  int nseq;
  int d, dtype, exact;
  cudaStream_t stream;
};
// the exact kernels (attn_exact.cu); without scratch no row block's tiles are shared out
size_t attn_fwd_exact_workspace_bytes(const AttnCall& c);
size_t attn_bwd_exact_workspace_bytes(const AttnCall& c);
int launch_attn_fwd_exact(const AttnCall& c, void* ws);
int launch_attn_bwd_exact(const AttnCall& c, void* ws);
// o and lse from [parts, B, H, T, d] weighted values and [parts, B, H, T] (maximum in log2 units, sum)
int launch_attn_fwd_join(const AttnCall& c, int parts, const float* part_o, const float2* part_ml);
// the tensor-core kernels (attn_fwd_tc.cu): bf16 storage, d = 64 or 128
bool attn_tc_supported(int dtype, int d, int exact);
size_t attn_fwd_tc_workspace_bytes(int B, int H, int H_kv, int T, int T_k, int window, int d);
int launch_attn_fwd_tc(const AttnCall& c, void* ws);
int launch_attn_bwd_tc(const AttnCall& c);  // attn_bwd_tc.cu

// one step over a cache, in the storage type (K, V) or in 4 bits (kq, kp, vq, vp); attn_decode.cu
struct AttnDecode {
  const void *q, *k_t, *v_t;
  void *K, *V, *kq, *kp, *vq, *vp;
  const int* pos;
  const float* slopes;
  void *o, *ws;
  int B, H, H_kv, C, window, d, dtype, exact;
  float scale, cap;
  int* dev_status;
  cudaStream_t stream;
};
size_t attn_decode_workspace_bytes(const AttnDecode& c);
int launch_attn_decode(const AttnDecode& c);
// checks of a call's parameters, and of those that name a cache (attn.cu)
int attn_check(const lawcat_attn_params* p);
int attn_check_cache(const lawcat_attn_params* p);
// attention of drafted tokens (attn_tree.cu)
size_t attn_tree_workspace_bytes(const lawcat_attn_params* p);
// T rows per sequence of k_t, v_t into the 4-bit cache, or (write = false) out of it
int launch_attn_quant(const AttnDecode& c, int T, bool write);

}  // namespace lawcat

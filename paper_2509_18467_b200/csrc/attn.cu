// Entry points of softmax attention (the formulas are at the top of attn.cuh): argument checks on the host, the table of the
// queries' key intervals where documents or prefixes are given, then dispatch to the kernels.
#include <cmath>

#include "attn.cuh"

using namespace lawcat;

namespace {

constexpr int MAX_TOKENS = 1 << 30;  // (positions, tile ends and distances stay inside 32 bits)

bool aligned(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; }

int check(const lawcat_attn_params* p) {
  if (!p) return LAWCAT_ERR_INVALID_ARG;
  if (p->B < 0 || p->T < 0 || p->T_k < 0 || p->H <= 0 || p->H_kv <= 0 || p->H % p->H_kv) return LAWCAT_ERR_INVALID_ARG;
  if (p->dtype != LAWCAT_F32 && p->dtype != LAWCAT_BF16) return LAWCAT_ERR_INVALID_ARG;
  if ((p->causal | 1) != 1 || (p->exact | 1) != 1 || p->window < 0) return LAWCAT_ERR_INVALID_ARG;
  if (!std::isfinite(p->scale) || !std::isfinite(p->cap) || p->cap < 0.f) return LAWCAT_ERR_INVALID_ARG;
  // (what the kernels make of them in fp32: scores in units of log2, and the argument of the tanh)
  if (!std::isfinite(p->scale * attn::LOG2E)) return LAWCAT_ERR_INVALID_ARG;
  if (p->cap > 0.f && (!std::isfinite(p->cap * attn::LOG2E) || !std::isfinite(1.f / p->cap) || !std::isfinite(2.f * attn::LOG2E * (p->scale / p->cap))))
    return LAWCAT_ERR_INVALID_ARG;
  if (p->d != 16 && p->d != 32 && p->d != 64 && p->d != 128) return LAWCAT_ERR_UNSUPPORTED;
  if (p->T > MAX_TOKENS || p->T_k > MAX_TOKENS || (long long)p->B * p->H > 0x7fffffffLL / 64) return LAWCAT_ERR_UNSUPPORTED;
  return LAWCAT_OK;
}

// documents and prefixes: HOST arrays of nseq + 1 token offsets and of nseq lengths
int check_docs(const lawcat_attn_params* p, const int32_t* cu, const int32_t* prefix, int nseq) {
  if (!cu && !prefix) return nseq == 0 ? LAWCAT_OK : LAWCAT_ERR_INVALID_ARG;
  if (nseq < 0) return LAWCAT_ERR_INVALID_ARG;
  if (cu) {
    if (p->B != 1 || p->T != p->T_k || cu[0] != 0 || cu[nseq] != p->T) return LAWCAT_ERR_INVALID_ARG;
    for (int i = 0; i < nseq; ++i)
      if (cu[i + 1] < cu[i]) return LAWCAT_ERR_INVALID_ARG;
  } else if (nseq != p->B) {
    return LAWCAT_ERR_INVALID_ARG;
  }
  if (prefix) {
    if (!p->causal || p->window) return LAWCAT_ERR_INVALID_ARG;
    for (int i = 0; i < nseq; ++i)
      if (prefix[i] < 0 || prefix[i] > (cu ? cu[i + 1] - cu[i] : p->T_k)) return LAWCAT_ERR_INVALID_ARG;
  }
  return LAWCAT_OK;
}

// A launch's sequences, by value: what the call passed is read while it is captured, and a replay needs no host memory.
constexpr int TABLE = 256;
struct Sequences {
  int n, first_b, docs;
  int start[TABLE + 1], prefix[TABLE];
};

// rows[b][t] = the keys that query t sees, and keys[b][j] = the queries that see key j
__global__ void attn_rows_kernel(const __grid_constant__ Sequences s, const attn::Mask m, int2* rows, int2* keys) {
  attn::behind_last_kernel();
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (s.docs) {  // one packed batch: the launch's sequences cover tokens [start[0], start[n])
    const int t = s.start[0] + i;
    if (t >= s.start[s.n]) return;
    int lo = 0, hi = s.n - 1;  // the last sequence with start <= t (empty ones in front of it share that start)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s.start[mid] <= t) lo = mid; else hi = mid - 1;
    }
    const int s0 = s.start[lo], len = s.start[lo + 1] - s0;
    attn::Mask md = m;
    md.T = md.T_k = len;
    int2 iv = attn::interval(md, 0, t - s0);
    if (s.prefix[lo] > iv.y) iv.y = s.prefix[lo];
    rows[t] = make_int2(iv.x + s0, iv.y + s0);
    if (keys) {
      iv = attn::key_interval(md, 0, t - s0, s.prefix[lo]);
      keys[t] = make_int2(iv.x + s0, iv.y + s0);
    }
  } else {
    const int b = blockIdx.y;
    if (i < m.T) {
      int2 iv = attn::interval(m, 0, i);
      if (s.prefix[b] > iv.y) iv.y = s.prefix[b];
      rows[(size_t)(s.first_b + b) * m.T + i] = iv;
    }
    if (keys && i < m.T_k) keys[(size_t)(s.first_b + b) * m.T_k + i] = attn::key_interval(m, 0, i, s.prefix[b]);
  }
}

int fill_rows(const lawcat_attn_params* p, const int32_t* cu, const int32_t* prefix, int nseq, attn::Mask& m, int2* rows, int2* keys,
              cudaStream_t stream) {
  Sequences s;
  s.docs = cu != nullptr;
  for (int f = 0; f < nseq; f += TABLE) {
    s.n = nseq - f < TABLE ? nseq - f : TABLE;
    s.first_b = f;
    for (int i = 0; i < s.n; ++i) {
      s.start[i] = cu ? cu[f + i] : 0;
      s.prefix[i] = prefix ? prefix[f + i] : 0;
    }
    s.start[s.n] = cu ? cu[f + s.n] : 0;
    const int tokens = cu ? s.start[s.n] - s.start[0] : keys && m.T_k > m.T ? m.T_k : m.T;
    if (!tokens) continue;
    const dim3 grid((unsigned)((tokens + 255) / 256), cu ? 1u : (unsigned)s.n);
    LAWCAT_LAUNCH("attn_rows", stream, launch_behind(attn_rows_kernel, grid, dim3(256), 0, stream, s, m, rows, keys));
    LAWCAT_CHECK_LAUNCH();
  }
  m.rows = rows;
  m.keys = keys;
  return LAWCAT_OK;
}

size_t rows_bytes(const lawcat_attn_params* p) { return align_up(sizeof(int2) * (size_t)p->B * p->T, 256); }
size_t keys_bytes(const lawcat_attn_params* p) { return align_up(sizeof(int2) * (size_t)p->B * p->T_k, 256); }
int stat_stride(const lawcat_attn_params* p) { return (p->T + 63) / 64 * 64; }
size_t stat_bytes(const lawcat_attn_params* p) { return align_up(2 * sizeof(float) * (size_t)p->B * stat_stride(p) * p->H, 256); }

AttnCall make_call(const lawcat_attn_params* p, const float* slopes, void* stream, int* dev_status) {
  AttnCall c{};
  c.a.B = p->B; c.a.H = p->H; c.a.H_kv = p->H_kv;
  c.a.scale = p->scale; c.a.cap = p->cap;
  c.a.slopes = slopes;
  c.a.dev_status = dev_status;
  // (a window that holds every distance is none: positions plus or minus a window then stay inside 32 bits)
  const int window = p->window > (p->T > p->T_k ? p->T : p->T_k) ? 0 : p->window;
  c.a.mask = attn::Mask{p->T, p->T_k, p->T_k - p->T, p->causal, window, nullptr, nullptr};
  c.d = p->d; c.dtype = p->dtype; c.exact = p->exact;
  c.stream = (cudaStream_t)stream;
  return c;
}

AttnDecode make_decode(const lawcat_attn_params* p, const void* q, const void* k, const void* v, const int* pos, const float* slopes, void* stream,
                       int* dev_status) {
  AttnDecode c{};
  c.dev_status = dev_status;
  c.q = q; c.k_t = k; c.v_t = v;
  c.pos = pos; c.slopes = slopes;
  c.B = p->B; c.H = p->H; c.H_kv = p->H_kv; c.C = p->T_k; c.window = p->window;
  c.d = p->d; c.dtype = p->dtype; c.exact = p->exact;
  c.scale = p->scale; c.cap = p->cap;
  c.stream = (cudaStream_t)stream;
  return c;
}

template <size_t N>
int check_ptrs(const void* const (&req)[N], const void* const* opt, int nopt) {
  for (const void* x : req)
    if (!x || !aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  for (int i = 0; i < nopt; ++i)
    if (!aligned(opt[i])) return LAWCAT_ERR_INVALID_ARG;
  return LAWCAT_OK;
}

int check_cache(const lawcat_attn_params* p) {
  if (p->T_k < 1 || (p->window && p->window > p->T_k)) return LAWCAT_ERR_INVALID_ARG;  // (the window's keys must still be there)
  return LAWCAT_OK;
}

}  // namespace

extern "C" {

size_t lawcat_attn_workspace_bytes(const lawcat_attn_params* p, int op) {
  if (check(p) != LAWCAT_OK) return 0;
  switch (op) {
    case LAWCAT_OP_ATTN_FWD:
      return rows_bytes(p) + (attn_tc_supported(p->dtype, p->d, p->exact)
                                  ? attn_fwd_tc_workspace_bytes(p->B, p->H, p->H_kv, p->T, p->T_k, p->window, p->d)
                                  : attn_fwd_exact_workspace_bytes(make_call(p, nullptr, nullptr, nullptr)));
    case LAWCAT_OP_ATTN_BWD:
      return rows_bytes(p) + keys_bytes(p) + stat_bytes(p) +
             (attn_tc_supported(p->dtype, p->d, p->exact) ? 0 : attn_bwd_exact_workspace_bytes(make_call(p, nullptr, nullptr, nullptr)));
    case LAWCAT_OP_ATTN_DECODE: return align_up(attn_decode_workspace_bytes(make_decode(p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr)), 256);
    default: return 0;
  }
}

int lawcat_attn_fwd(const lawcat_attn_params* p, const int32_t* cu_seqlens, const int32_t* prefix, int32_t nseq, const void* q,
                    const void* k, const void* v, const float* slopes, void* o, float* lse, void* ws, size_t ws_bytes, void* stream,
                    int* dev_status) {
  int r = check(p);
  if (r || (r = check_docs(p, cu_seqlens, prefix, nseq))) return r;
  const bool empty = (size_t)p->B * p->T == 0, none = (size_t)p->B * p->T_k == 0;
  if ((!empty && (!q || !o)) || (!empty && !none && (!k || !v))) return LAWCAT_ERR_INVALID_ARG;
  for (const void* x : {q, k, v, (const void*)slopes, (const void*)o, (const void*)lse, (const void*)ws})
    if (!aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  if (empty) return LAWCAT_OK;
  if (!ws || ws_bytes < lawcat_attn_workspace_bytes(p, LAWCAT_OP_ATTN_FWD)) return LAWCAT_ERR_WORKSPACE_TOO_SMALL;
  AttnCall c = make_call(p, slopes, stream, dev_status);
  c.a.q = q; c.a.k = k; c.a.v = v; c.a.o = o; c.a.lse = lse;
  if (cu_seqlens || prefix) {
    if ((r = fill_rows(p, cu_seqlens, prefix, nseq, c.a.mask, (int2*)ws, nullptr, c.stream))) return r;
  }
  return attn_tc_supported(p->dtype, p->d, p->exact) ? launch_attn_fwd_tc(c, (char*)ws + rows_bytes(p)) : launch_attn_fwd_exact(c, (char*)ws + rows_bytes(p));
}

int lawcat_attn_bwd(const lawcat_attn_params* p, const int32_t* cu_seqlens, const int32_t* prefix, int32_t nseq, const void* q,
                    const void* k, const void* v, const float* slopes, const void* o, const float* lse, const void* dO, void* dq,
                    void* dk, void* dv, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  int r = check(p);
  if (r || (r = check_docs(p, cu_seqlens, prefix, nseq))) return r;
  const bool no_q = (size_t)p->B * p->T == 0, no_k = (size_t)p->B * p->T_k == 0;
  if (!no_q && (!q || !o || !lse || !dO || !dq)) return LAWCAT_ERR_INVALID_ARG;
  if (!no_k && (!k || !v || !dk || !dv)) return LAWCAT_ERR_INVALID_ARG;
  for (const void* x : {q, k, v, (const void*)slopes, o, (const void*)lse, dO, (const void*)dq, (const void*)dk, (const void*)dv, (const void*)ws})
    if (!aligned(x)) return LAWCAT_ERR_INVALID_ARG;
  if (no_q && no_k) return LAWCAT_OK;
  const size_t need = lawcat_attn_workspace_bytes(p, LAWCAT_OP_ATTN_BWD);
  if (need && (!ws || ws_bytes < need)) return LAWCAT_ERR_WORKSPACE_TOO_SMALL;
  AttnCall c = make_call(p, slopes, stream, dev_status);
  c.a.q = q; c.a.k = k; c.a.v = v; c.a.o_in = o; c.a.dO = dO;
  c.a.lse = const_cast<float*>(lse);
  c.a.dq = dq; c.a.dk = dk; c.a.dv = dv;
  int2* const keys = (int2*)((char*)ws + rows_bytes(p));
  c.a.stat = (float*)((char*)keys + keys_bytes(p));
  c.a.stat_stride = stat_stride(p);
  c.cu = cu_seqlens; c.prefix = prefix; c.nseq = nseq;
  if (cu_seqlens || prefix) {
    if ((r = fill_rows(p, cu_seqlens, prefix, nseq, c.a.mask, (int2*)ws, keys, c.stream))) return r;
  }
  return attn_tc_supported(p->dtype, p->d, p->exact) ? launch_attn_bwd_tc(c) : launch_attn_bwd_exact(c, (char*)c.a.stat + stat_bytes(p));
}

int lawcat_attn_decode(const lawcat_attn_params* p, const void* q_t, const void* k_t, const void* v_t, void* K, void* V, const int32_t* pos,
                       const float* slopes, void* o_t, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  int r = check(p);
  if (r || (r = check_cache(p))) return r;
  if (p->B == 0) return LAWCAT_OK;
  const void* const req[] = {q_t, k_t, v_t, K, V, pos, o_t};
  const void* const opt[] = {slopes, ws};
  if ((r = check_ptrs(req, opt, 2))) return r;
  const size_t need = lawcat_attn_workspace_bytes(p, LAWCAT_OP_ATTN_DECODE);
  if (need && (!ws || ws_bytes < need)) return LAWCAT_ERR_WORKSPACE_TOO_SMALL;
  AttnDecode c = make_decode(p, q_t, k_t, v_t, pos, slopes, stream, dev_status);
  c.K = K; c.V = V; c.o = o_t; c.ws = ws;
  return launch_attn_decode(c);
}

int lawcat_attn_decode_quant(const lawcat_attn_params* p, const void* q_t, const void* k_t, const void* v_t, void* kq, void* kp, void* vq,
                             void* vp, const int32_t* pos, const float* slopes, void* o_t, void* ws, size_t ws_bytes, void* stream,
                             int* dev_status) {
  int r = check(p);
  if (r || (r = check_cache(p))) return r;
  if (p->B == 0) return LAWCAT_OK;
  const void* const req[] = {q_t, k_t, v_t, kq, kp, vq, vp, pos, o_t};
  const void* const opt[] = {slopes, ws};
  if ((r = check_ptrs(req, opt, 2))) return r;
  const size_t need = lawcat_attn_workspace_bytes(p, LAWCAT_OP_ATTN_DECODE);
  if (need && (!ws || ws_bytes < need)) return LAWCAT_ERR_WORKSPACE_TOO_SMALL;
  AttnDecode c = make_decode(p, q_t, k_t, v_t, pos, slopes, stream, dev_status);
  c.kq = kq; c.kp = kp; c.vq = vq; c.vp = vp; c.o = o_t; c.ws = ws;
  return launch_attn_decode(c);
}

static int cache_rows(const lawcat_attn_params* p, const void* k, const void* v, void* kq, void* kp, void* vq, void* vp, const int32_t* pos,
                      void* stream, bool write) {
  int r = check(p);
  if (r || (r = check_cache(p))) return r;
  if ((size_t)p->B * p->T == 0) return LAWCAT_OK;
  const void* const req[] = {k, v, kq, kp, vq, vp, pos};
  if ((r = check_ptrs(req, nullptr, 0))) return r;
  AttnDecode c = make_decode(p, nullptr, k, v, pos, nullptr, stream, nullptr);
  c.kq = kq; c.kp = kp; c.vq = vq; c.vp = vp;
  return launch_attn_quant(c, p->T, write);
}

int lawcat_cache_quantize(const lawcat_attn_params* p, const void* k, const void* v, const int32_t* pos, void* kq, void* kp, void* vq,
                          void* vp, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  return cache_rows(p, k, v, kq, kp, vq, vp, pos, stream, true);
}

int lawcat_cache_dequantize(const lawcat_attn_params* p, const void* kq, const void* kp, const void* vq, const void* vp, const int32_t* pos,
                            void* k, void* v, void* ws, size_t ws_bytes, void* stream, int* dev_status) {
  (void)ws; (void)ws_bytes; (void)dev_status;
  return cache_rows(p, k, v, const_cast<void*>(kq), const_cast<void*>(kp), const_cast<void*>(vq), const_cast<void*>(vp), pos, stream, false);
}

}  // extern "C"

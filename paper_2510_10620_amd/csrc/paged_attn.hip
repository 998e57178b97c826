// Attention of one new token per sequence over a paged key-value cache.
#include <cmath>

#include "cache_internal.h"
#include "device_utils.h"

using namespace dcp;

namespace dcp {

struct PagedArgs {
  const char* q;
  char* out;
  float* lse;
  const int32_t* seqs;
  int64_t q_st, q_sh, o_st, o_sh;   // bytes
  int32_t n, hq, group, layer, window, sink;
  float scale_log2e;
};

template <typename T> __device__ __forceinline__ void load8(const char* p, float* x) {
#pragma unroll
  for (int e = 0; e < 8; e++) x[e] = Elem<T>::load((const T*)p + e);
}

// A workgroup takes one query head of one place, D / 8 lanes a key; every group of lanes keeps the running maximum m, the sum l of
// exp(s - m) and the sum of exp(s - m) v of its keys, and the groups meet in LDS.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attn_kernel(KCache c, PagedArgs a) {
  constexpr int kLanes = D / 8, kGroups = 256 / kLanes;
  __shared__ float s_m[kGroups], s_l[kGroups], s_o[kGroups][D];
  const int i = blockIdx.x, h = blockIdx.y, hk = h / a.group;
  const int seq = a.seqs ? a.seqs[i] : i;
  if (!c.is_seq(seq)) return;
  const int len = c.length(seq);
  const int lo = a.window > 0 ? max(len - a.window, 0) : 0, head = a.window > 0 ? min(a.sink, lo) : 0;
  const int32_t* row = c.row(seq);
  const int g = threadIdx.x / kLanes, d0 = (threadIdx.x % kLanes) * 8;
  float q[8], acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, m = -INFINITY, l = 0;
  load8<T>(a.q + i * a.q_st + h * a.q_sh + d0 * sizeof(T), q);
  const char* kb = c.k + a.layer * c.k_sl + hk * c.k_sh + d0 * sizeof(T);
  const char* vb = c.v + a.layer * c.v_sl + hk * c.v_sh + d0 * sizeof(T);
  for (int x = g; x < head + len - lo; x += kGroups) {
    const int j = x < head ? x : x - head + lo;
    const int p = c.page.quot(j), page = row[p];
    if (!c.is_page(page)) continue;
    const int64_t slot = c.page.rem(j, p);
    float k[8], v[8];
    load8<T>(kb + page * c.k_sp + slot * c.k_st, k);
    load8<T>(vb + page * c.v_sp + slot * c.v_st, v);
    float s = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) s = fmaf(q[e], k[e], s);
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1) s += __shfl_xor(s, o);
    s *= a.scale_log2e;
    const float m2 = fmaxf(m, s), base = m2 == -INFINITY ? 0.f : m2;
    const float f = exp2f(m - base), w = exp2f(s - base);
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 8; e++) acc[e] = fmaf(w, v[e], acc[e] * f);
    m = m2;
  }
  if (d0 == 0) { s_m[g] = m; s_l[g] = l; }
#pragma unroll
  for (int e = 0; e < 8; e++) s_o[g][d0 + e] = acc[e];
  __syncthreads();
  float top = -INFINITY, sum = 0;
  for (int x = 0; x < kGroups; x++) top = fmaxf(top, s_m[x]);
  const float base = top == -INFINITY ? 0.f : top;
  for (int x = 0; x < kGroups; x++) sum += s_l[x] * exp2f(s_m[x] - base);
  for (int d = threadIdx.x; d < D; d += 256) {
    float o = 0;
    for (int x = 0; x < kGroups; x++) o += s_o[x][d] * exp2f(s_m[x] - base);
    Elem<T>::store((T*)(a.out + i * a.o_st + h * a.o_sh) + d, sum == 0.f ? 0.f : o / sum);
  }
  if (threadIdx.x == 0) a.lse[(int64_t)h * a.n + i] = sum == 0.f ? -INFINITY : base * 0.6931471805599453f + logf(sum);
}

template <typename T>
static void launch(const KCache& c, const PagedArgs& a, int d, hipStream_t s) {
  const dim3 grid((unsigned)a.n, (unsigned)a.hq);
  if (d == 128) hipLaunchKernelGGL((paged_attn_kernel<T, 128>), grid, dim3(256), 0, s, c, a);
  else if (d == 64) hipLaunchKernelGGL((paged_attn_kernel<T, 64>), grid, dim3(256), 0, s, c, a);
  else hipLaunchKernelGGL((paged_attn_kernel<T, 32>), grid, dim3(256), 0, s, c, a);
}

}  // namespace dcp

extern "C" size_t dcp_paged_attn_workspace_bytes(const dcp_cache_t* cache, int32_t n, int32_t hq) {
  return cache && n > 0 && hq > 0 ? 256 : 0;
}

extern "C" dcp_status_t dcp_paged_attn_fwd(const dcp_cache_t* cache, const dcp_paged_attn_t* args, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  KCache c;
  dcp_status_t st = pack_cache(cache, &c);
  if (st != DCP_OK) return st;
  if (!args) return fail(DCP_ERR_INVALID_ARG, "args is NULL");
  const dcp_paged_attn_t& t = *args;
  if ((st = check_places(c, t.seqs, t.n)) != DCP_OK) return st;
  if (t.hq <= 0) return fail(DCP_ERR_INVALID_ARG, "hq must be positive");
  if (t.hq % c.hkv != 0) return fail(DCP_ERR_UNSUPPORTED, "hq must be a multiple of hkv");
  if (t.layer < 0 || t.layer >= c.n_layers) return fail(DCP_ERR_INVALID_ARG, "layer out of range");
  if (!(t.softmax_scale > 0.f) || !std::isfinite(t.softmax_scale)) return fail(DCP_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
  if (t.window < 0 || t.sink < 0) return fail(DCP_ERR_INVALID_ARG, "window and sink must not be negative");
  if (t.n == 0) return DCP_OK;
  if ((st = check_rows("q", t.q, t.q_stride_t, t.q_stride_h, cache->d)) != DCP_OK) return st;
  if ((st = check_rows("out", t.out, t.o_stride_t, t.o_stride_h, cache->d)) != DCP_OK) return st;
  if (!t.lse || (reinterpret_cast<uintptr_t>(t.lse) & 3u)) return fail(DCP_ERR_INVALID_ARG, "lse is NULL or misaligned");
  if (!workspace || workspace_bytes < dcp_paged_attn_workspace_bytes(cache, t.n, t.hq))
    return fail(DCP_ERR_WORKSPACE, "workspace is NULL or smaller than dcp_paged_attn_workspace_bytes");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return fail(DCP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  const int64_t e = cache->dtype == DCP_BF16 ? 2 : 4;
  {
    const char *q0 = (const char*)t.q, *o0 = (const char*)t.out;
    const char* q1 = q0 + ((t.n - 1) * t.q_stride_t + (t.hq - 1) * t.q_stride_h + cache->d) * e;
    const char* o1 = o0 + ((t.n - 1) * t.o_stride_t + (t.hq - 1) * t.o_stride_h + cache->d) * e;
    if (q0 < o1 && o0 < q1) return fail(DCP_ERR_INVALID_ARG, "out overlaps q");
  }
  const PagedArgs a{(const char*)t.q, (char*)t.out, t.lse, t.seqs, t.q_stride_t * e, t.q_stride_h * e, t.o_stride_t * e, t.o_stride_h * e,
                    t.n, t.hq, t.hq / c.hkv, t.layer, t.window, t.sink, t.softmax_scale * 1.44269504088896340736f};
  ProfScope ps(DCP_K_PAGED_ATTN, (hipStream_t)stream);
  if (cache->dtype == DCP_BF16) launch<bf16_t>(c, a, cache->d, (hipStream_t)stream);
  else launch<float>(c, a, cache->d, (hipStream_t)stream);
  DCP_HIP_TRY(hipGetLastError());
  return DCP_OK;
}

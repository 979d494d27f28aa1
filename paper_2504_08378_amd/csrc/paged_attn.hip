// Attention of new tokens over a paged cache.
//
// Row t of sequence b stands at place p of its cache; it sees key j <= p if there is no window, or j > p - window,
// or j < n_sink.  o = sum_j e^{s_j} v_j / sum_j e^{s_j} over those, s_j = scale q.k_j.
#include <math.h>

#include "paged.h"

struct PagedAttnParams {
  PagedView v;
  const half_t* q;   // [n_rows][q_stride]
  half_t* out;       // [n_rows][out_stride]
  long long q_stride, out_stride;
  int n_heads, window, n_sink;
  float scale2;      // scale * log2(e): the exponentials are powers of two
};

// One query head of one row by one wave, on the vector unit in fp32: the keys one after the other (a group of
// HD / 8 lanes takes each), those that the row does not see are not looked at.
template <int HD>
__device__ __forceinline__ void paged_row(const PagedAttnParams& p, int b, int row, int place, int h) {
  constexpr int LPK = HD / 8, KPW = AF_WAVE / LPK;
  const PagedView& v = p.v;
  const int lane = threadIdx.x & 63, g = lane / LPK, c0 = lane % LPK * 8;
  const int kvh = h / (p.n_heads / v.n_kv);
  const half8 qh = *reinterpret_cast<const half8*>(p.q + (size_t)row * p.q_stride + (size_t)h * HD + c0);
  float q[8], acc[8], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    q[c] = (float)qh[c] * p.scale2;
    acc[c] = 0.f;
  }
  const int lo = p.window > 0 ? max(0, place - p.window + 1) : 0;
  const int sinks = min(p.n_sink, lo), n = place + 1 - lo + sinks;  // seen keys: [0, sinks) and [lo, place]
  bool any = false;
  for (int i0 = 0; i0 < n; i0 += KPW) {
    const int i = i0 + g, j = i < sinks ? i : i - sinks + lo;
    const int page = i < n ? paged_page(v, b, j) : -1;
    float s = -INFINITY;
    half8 vh = {};
    if (page >= 0) {
      const size_t o = paged_offset(v, page, kvh, j, HD) + c0;
      const half8 kh = *reinterpret_cast<const half8*>(v.k + o);
      vh = *reinterpret_cast<const half8*>(v.v + o);
      s = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) s += q[c] * (float)kh[c];
    }
#pragma unroll
    for (int off = 1; off < LPK; off <<= 1) s += __shfl_xor(s, off, AF_WAVE);
    if (page < 0) continue;
    any = true;
    const float mx = fmaxf(m, s), safe = mx == -INFINITY ? 0.f : mx;
    const float corr = exp2f(m - safe), w = exp2f(s - safe);
    m = mx;
    l = l * corr + w;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] = acc[c] * corr + w * (float)vh[c];
  }
  // the groups of lanes
  float M = m;
#pragma unroll
  for (int off = LPK; off < AF_WAVE; off <<= 1) M = fmaxf(M, __shfl_xor(M, off, AF_WAVE));
  const float f = any ? exp2f(m - (M == -INFINITY ? 0.f : M)) : 0.f;
  l *= f;
#pragma unroll
  for (int off = LPK; off < AF_WAVE; off <<= 1) l += __shfl_xor(l, off, AF_WAVE);
  half8 o;
  const bool seen = __any(any);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float a = any ? acc[c] * f : 0.f;
#pragma unroll
    for (int off = LPK; off < AF_WAVE; off <<= 1) a += __shfl_xor(a, off, AF_WAVE);
    o[c] = seen ? (half_t)(a / l) : (half_t)0;
  }
  if (g == 0) *reinterpret_cast<half8*>(p.out + (size_t)row * p.out_stride + (size_t)h * HD + c0) = o;
}

// A wave per row and query head.
template <int HD>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedAttnParams p) {
  const int lane = threadIdx.x & 63;
  const long long item = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= (long long)p.v.n_rows * p.n_heads) return;
  const int row = (int)(item / p.n_heads), h = (int)(item % p.n_heads);
  int b = row;
  if (p.v.q_start) {
    b = -1;
    for (int i = lane; i < p.v.n_seqs; i += AF_WAVE) {
      const PagedSeq s = paged_seq(p.v, i);
      if (s.row0 <= row && row < s.row0 + s.q_len) b = i;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) b = max(b, __shfl_xor(b, off, AF_WAVE));
    if (b < 0) return;
  }
  const PagedSeq s = paged_seq(p.v, b);
  if (s.q_len == 0) return;
  paged_row<HD>(p, b, row, s.len - s.q_len + row - s.row0, h);
}

extern "C" int af_paged_attention(af_ctx* ctx, const af_paged_cache* cache, const af_paged_batch* batch, int n_heads,
                                  float scale, int window, int n_sink, const void* q_f16, long long q_stride,
                                  void* out_f16, long long out_stride) {
  PagedAttnParams p;
  if (!ctx) return AF_ENULL;
  int rc = af_paged_view(cache, batch, n_heads, &p.v);
  if (rc != AF_OK) return rc;
  if ((!q_f16 || !out_f16) && batch->n_rows) return AF_ENULL;
  if (window < 0 || n_sink < 0 || !(fabsf(scale) < INFINITY)) return AF_EINVAL;
  const int hd = cache->head_dim;
  if (!af_paged_rows_ok(q_f16, q_stride, (long long)n_heads * hd) ||
      !af_paged_rows_ok(out_f16, out_stride, (long long)n_heads * hd))
    return AF_ESHAPE;
  if ((rc = af_paged_ready(ctx, &p.v)) != AF_OK) return rc;
  if (batch->n_rows == 0) return AF_OK;
  p.q = (const half_t*)q_f16;
  p.out = (half_t*)out_f16;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.n_heads = n_heads;
  p.window = window;
  p.n_sink = window > 0 ? n_sink : 0;
  p.scale2 = (scale == 0.f ? 1.0f / sqrtf((float)hd) : scale) * 1.44269504088896340736f;
  const long long items = (long long)batch->n_rows * n_heads;
  const dim3 grid((unsigned)((items + 3) / 4)), threads(256);
  if (hd == 128)
    hipLaunchKernelGGL(paged_rows_kernel<128>, grid, threads, 0, ctx->stream, p);
  else
    hipLaunchKernelGGL(paged_rows_kernel<64>, grid, threads, 0, ctx->stream, p);
  AF_LAUNCH_CHECK();
  return AF_OK;
}

// What both forms of the paged attention share: their arguments, and one row on its own.
#pragma once
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

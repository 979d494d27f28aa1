// New tokens into a paged cache: norms of queries and keys for each head, rotary positions, the rows of
// K and V to their pages, the rotated queries beside them, in one pass over q | k | v.
//
// With x one head of a token, g the gain: x <- x rsqrt(mean x^2 + eps) g (where there is a gain), then for
// i < hd/2 and the angle t = pos theta^(-2i/hd): (x_i, x_{i+hd/2}) <- (x_i cos t - x_{i+hd/2} sin t,
// x_{i+hd/2} cos t + x_i sin t).  All of it is fp32 and rounded once, to the fp16 of cache and queries.
// The angle is taken in turns, in fp64, and only what is left of it behind the last whole turn goes
// on in fp32: 2^-25 of a turn at any position.
//
// Bound by memory: the rows are read and written once.  A lane has eight neighbouring elements and the eight
// half a head further, both sides of eight rotations in 16-byte pieces; so a head is 8 lanes (4 at width 64),
// its norm three exchanges inside them.  A wave works for itself: it has one token (or, where there are few tokens, a
// quarter of one's heads), requests its first heads before it looks for the token's sequence and page, forms the
// token's angles with a lane for each, and hands them to the lanes of all heads through LDS.  5348 rows of 80 heads of 128, 109 MB
// each way: 44.0 us, 5.0 TB/s, as a copy of that size (with four tokens a workgroup, looked up before the first load and behind
// three barriers, 51.7; loads that stay in the caches 48.4); one row 3.4 us.
#include <math.h>
#include <string.h>

#include "paged.h"

#define APP_THREADS 256
#define APP_WAVES (APP_THREADS / AF_WAVE)

#define APP_AHEAD 4  // heads of a lane that are requested together

struct AppendParams {
  PagedView v;
  const half_t* qkv;    // [n_rows][qkv_stride]: q | k | v
  half_t* q_out;        // [n_rows][q_stride], or null
  const half_t *q_gain, *k_gain;  // [head_dim] or null
  const int32_t* pos;   // [n_rows] or null: the place in the cache
  long long qkv_stride, q_stride;
  int n_heads;
  float eps;
  double turns[64];     // theta^(-2i/hd) / (2 pi)
};

// WPT: waves that share a token's heads (4: few tokens, 1: many).
template <int HD, int WPT>
__global__ __launch_bounds__(APP_THREADS) void paged_append_kernel(AppendParams p) {
  constexpr int LPH = HD / 16;              // lanes of a head
  constexpr int HPW = AF_WAVE / LPH;        // heads of a wave at a time
  __shared__ __align__(16) float s_cs[APP_WAVES][HD / 2], s_sn[APP_WAVES][HD / 2];
  const PagedView& v = p.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x * (APP_WAVES / WPT) + wave / WPT;
  if (row >= v.n_rows) return;

  const int i0 = lane % LPH * 8, heads = p.n_heads + 2 * v.n_kv;
  const int h0 = wave % WPT * HPW + lane / LPH;  // the lane's first head; the next is WPT * HPW further
  const half_t* src = p.qkv + (size_t)row * p.qkv_stride + i0;
  half8 a[APP_AHEAD], b[APP_AHEAD];
  auto fetch = [&](int h) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < APP_AHEAD; ++u) {
      const size_t o = (size_t)min(h + u * WPT * HPW, heads - 1) * HD;
      a[u] = af_load_once(reinterpret_cast<const half8*>(src + o));
      b[u] = af_load_once(reinterpret_cast<const half8*>(src + o + HD / 2));
    }
  };
  fetch(h0);

  // the row's sequence; numbers that cannot be right are reported by whoever meets them, all by the first wave
  int seq = row;
  PagedSeq s{0, 0, 0};
  if (v.q_start) {
    seq = -1;
    for (int b0 = 0; b0 < v.n_seqs && (seq < 0 || row == 0); b0 += AF_WAVE) {
      PagedSeq c{0, 0, 0};
      if (b0 + lane < v.n_seqs) c = paged_seq(v, b0 + lane);
      const unsigned long long hit = __ballot(c.row0 <= row && row < c.row0 + c.q_len);
      if (hit && seq < 0) {
        const int l = __builtin_ctzll(hit);
        seq = b0 + l;
        s = PagedSeq{__builtin_amdgcn_readlane(c.row0, l), __builtin_amdgcn_readlane(c.q_len, l), __builtin_amdgcn_readlane(c.len, l)};
      }
    }
    if (seq < 0) return;
  } else {
    s = paged_seq(v, row);
  }
  const int at = s.q_len > 0 ? s.len - s.q_len + row - s.row0 : -1;
  if (at < 0) return;  // no token (an empty sequence, or one that cannot be right)
  const int page = paged_page(v, seq, at);
  if (page < 0) return;

  const int pos = p.pos ? p.pos[row] : at;
  if (lane < HD / 2) {
    const double turns = (double)pos * p.turns[lane];
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    s_cs[wave][lane] = cs;
    s_sn[wave][lane] = sn;
  }
  __builtin_amdgcn_wave_barrier();  // a wave's LDS accesses are done in order
  float cs[8], sn[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    cs[c] = s_cs[wave][i0 + c];
    sn[c] = s_sn[wave][i0 + c];
  }
  half_t* const dk = v.k + paged_offset(v, page, 0, at, HD) + i0;
  half_t* const dv = v.v + paged_offset(v, page, 0, at, HD) + i0;
  half_t* const dq = p.q_out ? p.q_out + (size_t)row * p.q_stride + i0 : nullptr;
  for (int h1 = h0;; h1 += APP_AHEAD * WPT * HPW) {
#pragma unroll
    for (int u = 0; u < APP_AHEAD; ++u) {
      const int h = h1 + u * WPT * HPW;
      if (h >= heads) continue;
      half8 ra = a[u], rb = b[u];
      half_t* dst = dq ? dq + (size_t)h * HD : nullptr;
      if (h >= p.n_heads + v.n_kv)
        dst = dv + ((size_t)(h - p.n_heads - v.n_kv) << v.page_shift) * HD;
      else if (h >= p.n_heads)
        dst = dk + ((size_t)(h - p.n_heads) << v.page_shift) * HD;
      if (h < p.n_heads + v.n_kv) {
        float x[8], y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          x[c] = (float)ra[c];
          y[c] = (float)rb[c];
        }
        const half_t* gain = h < p.n_heads ? p.q_gain : p.k_gain;
        if (gain) {
          float sum = 0.f;
#pragma unroll
          for (int c = 0; c < 8; ++c) sum += x[c] * x[c] + y[c] * y[c];
#pragma unroll
          for (int off = 1; off < LPH; off <<= 1) sum += __shfl_xor(sum, off, AF_WAVE);
          const float r = 1.0f / sqrtf(sum * (1.0f / HD) + p.eps);
          const half8 ga = *reinterpret_cast<const half8*>(gain + i0), gb = *reinterpret_cast<const half8*>(gain + i0 + HD / 2);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            x[c] = x[c] * r * (float)ga[c];
            y[c] = y[c] * r * (float)gb[c];
          }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          ra[c] = (half_t)__builtin_fmaf(x[c], cs[c], -(y[c] * sn[c]));
          rb[c] = (half_t)__builtin_fmaf(y[c], cs[c], x[c] * sn[c]);
        }
      }
      if (dst) {
        *reinterpret_cast<half8*>(dst) = ra;
        *reinterpret_cast<half8*>(dst + HD / 2) = rb;
      }
    }
    if (h1 - lane / LPH + APP_AHEAD * WPT * HPW >= heads) break;  // the same for the wave
    fetch(h1 + APP_AHEAD * WPT * HPW);
  }
}

bool af_paged_rows_ok(const void* p, long long stride, long long width) {
  return ((uintptr_t)p & 15u) == 0 && stride >= width && stride % 8 == 0;
}

int af_paged_view(const af_paged_cache* c, const af_paged_batch* b, int n_heads, PagedView* v) {
  if (!c || !b) return AF_ENULL;
  if (!c->k_pages || !c->v_pages || !b->page_table || !b->kv_len) return AF_ENULL;
  if (c->n_pages < 1 || c->n_kv_heads < 1 || n_heads < 1 || n_heads > AF_PAGED_MAX_HEADS) return AF_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return AF_ESHAPE;
  if (n_heads % c->n_kv_heads) return AF_ESHAPE;
  int shift = 0;
  while (shift < 9 && (1 << shift) != c->page_tokens) ++shift;
  if (shift < 4 || shift > 8) return AF_ESHAPE;
  const long long page = (long long)c->n_kv_heads * c->page_tokens * c->head_dim;
  if (c->page_stride < page || c->page_stride % 8) return AF_ESHAPE;
  if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages) & 15u) return AF_ESHAPE;
  if (b->n_seqs < 1 || b->n_seqs > AF_PAGED_MAX_SEQS || b->table_stride < 1) return AF_EINVAL;
  if (((long long)b->table_stride << shift) > AF_PAGED_MAX_TOKENS) return AF_EINVAL;
  if (b->n_rows < 0 || b->n_rows > AF_PAGED_MAX_ROWS || b->max_q_len < 1) return AF_EINVAL;
  if ((long long)b->n_rows * n_heads > 1 << 30) return AF_EINVAL;
  if (!b->q_start && (b->n_rows != b->n_seqs || b->max_q_len != 1)) return AF_EINVAL;
  v->k = (half_t*)c->k_pages;
  v->v = (half_t*)c->v_pages;
  v->page_stride = c->page_stride;
  v->table = b->page_table;
  v->kv_len = b->kv_len;
  v->q_start = b->q_start;
  v->table_stride = b->table_stride;
  v->n_pages = c->n_pages;
  v->page_shift = shift;
  v->n_kv = c->n_kv_heads;
  v->n_seqs = b->n_seqs;
  v->n_rows = b->n_rows;
  v->max_q_len = b->max_q_len;
  v->tickets = nullptr;
  return AF_OK;
}

int af_paged_ready(const af_ctx* ctx, PagedView* v) {
  if (!ctx->ws) return AF_EWORKSPACE;
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return AF_EHIP;
  if (dev != ctx->device) return AF_EINVAL;
  v->tickets = (int*)(ctx->ws + ctx->lay.tickets);
  return AF_OK;
}

extern "C" int af_paged_append(af_ctx* ctx, const af_paged_cache* cache, const af_paged_batch* batch, int n_heads,
                               float rope_theta, const void* q_gain_f16, const void* k_gain_f16, float eps,
                               const int32_t* pos, const void* qkv_f16, long long qkv_stride, void* q_out_f16,
                               long long q_out_stride) {
  AppendParams p;
  if (!ctx) return AF_ENULL;
  int rc = af_paged_view(cache, batch, n_heads, &p.v);
  if (rc != AF_OK) return rc;
  if (!qkv_f16 && batch->n_rows) return AF_ENULL;
  if (!(rope_theta > 0.f) || !(rope_theta < INFINITY) || !(eps >= 0.f) || !(eps < INFINITY)) return AF_EINVAL;
  const int hd = cache->head_dim;
  if (!af_paged_rows_ok(qkv_f16, qkv_stride, (long long)(n_heads + 2 * cache->n_kv_heads) * hd)) return AF_ESHAPE;
  if (q_out_f16 && !af_paged_rows_ok(q_out_f16, q_out_stride, (long long)n_heads * hd)) return AF_ESHAPE;
  if (((uintptr_t)q_gain_f16 | (uintptr_t)k_gain_f16) & 15u) return AF_ESHAPE;
  if ((rc = af_paged_ready(ctx, &p.v)) != AF_OK) return rc;
  if (batch->n_rows == 0) return AF_OK;
  p.qkv = (const half_t*)qkv_f16;
  p.q_out = (half_t*)q_out_f16;
  p.q_gain = (const half_t*)q_gain_f16;
  p.k_gain = (const half_t*)k_gain_f16;
  p.pos = pos;
  p.qkv_stride = qkv_stride;
  p.q_stride = q_out_stride;
  p.n_heads = n_heads;
  p.eps = eps;
  if (ctx->rope_theta != rope_theta || ctx->rope_dim != hd) {  // 64 powers take the host longer than the launch
    for (int i = 0; i < hd / 2; ++i)
      ctx->rope_turns[i] = pow((double)rope_theta, -2.0 * (double)i / (double)hd) / 6.283185307179586476925286766559;
    ctx->rope_theta = rope_theta;
    ctx->rope_dim = hd;
  }
  memcpy(p.turns, ctx->rope_turns, sizeof(p.turns));
  const int rows = batch->n_rows;
  const bool few = rows < 4 * ctx->n_cu;
  const dim3 grid(few ? rows : (rows + APP_WAVES - 1) / APP_WAVES), threads(APP_THREADS);
  if (hd == 128 && few)
    hipLaunchKernelGGL((paged_append_kernel<128, 4>), grid, threads, 0, ctx->stream, p);
  else if (hd == 128)
    hipLaunchKernelGGL((paged_append_kernel<128, 1>), grid, threads, 0, ctx->stream, p);
  else if (few)
    hipLaunchKernelGGL((paged_append_kernel<64, 4>), grid, threads, 0, ctx->stream, p);
  else
    hipLaunchKernelGGL((paged_append_kernel<64, 1>), grid, threads, 0, ctx->stream, p);
  AF_LAUNCH_CHECK();
  return AF_OK;
}

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
// its norm three exchanges inside them.  The angles of a token are formed once, by 64 lanes side by side,
// and go through LDS to the lanes of all heads.
#include <math.h>

#include "paged.h"

#define APP_THREADS 256
#define APP_WAVES (APP_THREADS / AF_WAVE)

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
  constexpr int TOKENS = APP_WAVES / WPT;   // of a workgroup
  __shared__ float s_cs[TOKENS][HD / 2], s_sn[TOKENS][HD / 2];
  __shared__ int s_seq[TOKENS], s_at[TOKENS], s_page[TOKENS], s_pos[TOKENS];
  const PagedView& v = p.v;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = blockIdx.x * TOKENS;
  if (tid < TOKENS) s_seq[tid] = -1;
  __syncthreads();
  // the sequences of this workgroup's rows
  if (v.q_start) {
    for (int b = tid; b < v.n_seqs; b += APP_THREADS) {
      const PagedSeq s = paged_seq(v, b);
      for (int t = max(s.row0, first); t < min(s.row0 + s.q_len, first + TOKENS); ++t) s_seq[t - first] = b;
    }
    __syncthreads();
  } else if (tid < TOKENS && first + tid < v.n_rows) {
    s_seq[tid] = first + tid;
  }
  if (tid < TOKENS) {
    const int b = s_seq[tid];
    int at = -1, page = -1;
    if (b >= 0) {
      const PagedSeq s = paged_seq(v, b);
      const int i = first + tid - s.row0;
      if (i >= 0 && i < s.q_len) at = s.len - s.q_len + i;  // -1: no token (an empty sequence)
      if (at >= 0) page = paged_page(v, b, at);
    }
    s_at[tid] = at;
    s_page[tid] = page;
    s_pos[tid] = at >= 0 && p.pos ? p.pos[first + tid] : at;
  }
  __syncthreads();
  for (int e = tid; e < TOKENS * (HD / 2); e += APP_THREADS) {
    const int t = e / (HD / 2), i = e % (HD / 2);
    const double turns = (double)s_pos[t] * p.turns[i];
    float sn, cs;
    sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
    s_cs[t][i] = cs;
    s_sn[t][i] = sn;
  }
  __syncthreads();

  const int t = wave / WPT, row = first + t;
  if (s_page[t] < 0) return;
  const int lk = lane % LPH, i0 = lk * 8;
  const half_t* src = p.qkv + (size_t)row * p.qkv_stride + i0;
  const int heads = p.n_heads + 2 * v.n_kv;
  for (int h = (wave % WPT) * HPW + lane / LPH; h < heads; h += WPT * HPW) {
    half8 a = *reinterpret_cast<const half8*>(src + (size_t)h * HD);
    half8 b = *reinterpret_cast<const half8*>(src + (size_t)h * HD + HD / 2);
    half_t* dst;
    if (h < p.n_heads)
      dst = p.q_out ? p.q_out + (size_t)row * p.q_stride + (size_t)h * HD : nullptr;
    else if (h < p.n_heads + v.n_kv)
      dst = v.k + paged_offset(v, s_page[t], h - p.n_heads, s_at[t], HD);
    else
      dst = v.v + paged_offset(v, s_page[t], h - p.n_heads - v.n_kv, s_at[t], HD);
    if (h < p.n_heads + v.n_kv) {
      float x[8], y[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        x[c] = (float)a[c];
        y[c] = (float)b[c];
      }
      const half_t* gain = h < p.n_heads ? p.q_gain : p.k_gain;
      if (gain) {
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) s += x[c] * x[c] + y[c] * y[c];
#pragma unroll
        for (int off = 1; off < LPH; off <<= 1) s += __shfl_xor(s, off, AF_WAVE);
        const float r = 1.0f / sqrtf(s * (1.0f / HD) + p.eps);
        const half8 ga = *reinterpret_cast<const half8*>(gain + i0), gb = *reinterpret_cast<const half8*>(gain + i0 + HD / 2);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          x[c] = x[c] * r * (float)ga[c];
          y[c] = y[c] * r * (float)gb[c];
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float cs = s_cs[t][i0 + c], sn = s_sn[t][i0 + c];
        a[c] = (half_t)__builtin_fmaf(x[c], cs, -(y[c] * sn));
        b[c] = (half_t)__builtin_fmaf(y[c], cs, x[c] * sn);
      }
    }
    if (dst) {
      *reinterpret_cast<half8*>(dst + i0) = a;
      *reinterpret_cast<half8*>(dst + i0 + HD / 2) = b;
    }
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
  if ((long long)b->n_rows * n_heads > 0x7FFFFFFF) return AF_EINVAL;
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
  for (int i = 0; i < hd / 2; ++i)
    p.turns[i] = pow((double)rope_theta, -2.0 * (double)i / (double)hd) / 6.283185307179586476925286766559;
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

// Attention of new tokens over a paged cache: the launches.
//
// Row t of sequence b stands at place p of its cache; it sees key j <= p if there is no window, or j > p - window,
// or j < n_sink.  o = sum_j e^{s_j} v_j / sum_j e^{s_j} over those, s_j = scale q.k_j.
//
// Sequences with at most 16 rows a key head (query heads x new tokens), and all with a single token, are bound by the read of
// their keys and values and go to paged_split.h, longer ones to the matrix cores of paged_prompt.h.  A batch that may hold both
// is one launch: its first workgroups, one per compute unit, take the former while the others fill the units.
#include <math.h>

#include "paged_prompt.h"
#include "paged_split.h"

template <int HD>
__global__ __launch_bounds__(SPL_THREADS, 2) void paged_split_kernel(PagedSplitParams p) {
  extern __shared__ __align__(16) unsigned long long s_first[];
  __shared__ __align__(16) float s_acc[SPL_WAVES][SPL_ROWS * (HD + 4)];
  float* const acc[SPL_WAVES] = {s_acc[0], s_acc[1], s_acc[2], s_acc[3]};
  paged_split_body<HD>(p, blockIdx.x, gridDim.x, acc, s_first);
}

template <int HD, bool FINE>
__global__ __launch_bounds__(SPL_THREADS, 2) void paged_mixed_kernel(PagedSplitParams p, PagedPieces pieces, int wgs, int longs) {
  static_assert(SPL_THREADS == PRM_WAVES * AF_WAVE && SPL_ROWS * (HD + 4) * sizeof(float) <= PRM_TILE * HD * sizeof(half_t), "LDS shared");
  extern __shared__ __align__(16) unsigned long long s_first[];
  __shared__ __align__(16) half_t s_k0[PRM_TILE * HD], s_k1[PRM_TILE * HD], s_v0[PRM_TILE * HD], s_v1[PRM_TILE * HD];
  if ((int)blockIdx.x < wgs) {
    float* const acc[SPL_WAVES] = {(float*)s_k0, (float*)s_k1, (float*)s_v0, (float*)s_v1};
    paged_split_body<HD>(p, blockIdx.x, wgs, acc, s_first);
  } else {
    const unsigned wg = blockIdx.x - (unsigned)wgs;
    const int piece = pieces.most > 1 ? (int)(wg / (unsigned)longs) : 0;
    paged_prompt_body<HD, FINE>(p.a, pieces, p.short_q, wg - (unsigned)(piece * longs), piece, s_k0, s_k1, s_v0, s_v1);
  }
}

template <int HD>
static int launch_attention(af_ctx* ctx, const PagedAttnParams& a) {
  const int rep = a.n_heads / a.v.n_kv, short_q = rep < SPL_ROWS ? SPL_ROWS / rep : 1;
  const bool mixed = a.v.max_q_len > short_q && a.v.n_rows > short_q;
  PagedSplitParams p;
  p.a = a;
  p.part = (float*)(ctx->ws + ctx->lay.partials);
  p.tickets = (int*)(ctx->ws + ctx->lay.tickets) + AF_TICKET_ATTN;
  p.slot_rows = rep >= SPL_ROWS ? SPL_ROWS : rep * (a.v.max_q_len < short_q ? a.v.max_q_len : short_q);
  p.short_q = short_q;
  const size_t floats = (ctx->lay.attn_part + ctx->lay.attn_floats * sizeof(float) - ctx->lay.partials) / sizeof(float);
  const size_t fit = floats / ((size_t)2 * p.slot_rows * (HD + 2));
  long long wgs = (mixed ? 1 : 2) * (long long)ctx->n_cu;
  if (wgs > (long long)fit) wgs = (long long)fit;
  if (wgs > SPL_MAX_WGS) wgs = SPL_MAX_WGS;
  if (wgs < 1) return AF_EWORKSPACE;
  const size_t lds = paged_split_lds(a.v.n_seqs);
  if (!mixed) {
    hipLaunchKernelGGL(paged_split_kernel<HD>, dim3((unsigned)wgs), dim3(SPL_THREADS), lds, ctx->stream, p);
    AF_LAUNCH_CHECK();
    return AF_OK;
  }
  // as many workgroups for the long ones as any division of the rows among the sequences can need
  const long long longer = a.v.n_rows / (short_q + 1);
  const long long longs = ((long long)a.v.n_rows * rep / PRM_ROWS + (a.v.n_seqs < longer ? a.v.n_seqs : longer)) * a.v.n_kv;
  // In pieces where they would not fill the chip, two a unit, and the keys may be many (us, whole / in pieces, 32 query heads on 8:
  // 32 tokens behind 8000 195 / 43, 256 behind 30000 712 / 252, two times 64 behind 2000 57.0 / 29.0; 16 on 1, 100 behind 60000 1398 / 119;
  // where the keys are few there is one piece: 500 tokens 19.8).
  PagedPieces pieces{};
  pieces.tickets = p.tickets;
  pieces.ticket0 = 2 * SPL_MAX_WGS;
  pieces.part = p.part + (size_t)2 * wgs * p.slot_rows * (HD + 2);
  pieces.most = 1;
  if (longs <= ctx->n_cu && longs <= AF_TICKET_ATTN - pieces.ticket0) {
    const long long room = (long long)((floats - (size_t)2 * wgs * p.slot_rows * (HD + 2)) / PRM_PIECE_FLOATS(HD));
    const long long tiles = ((long long)a.v.table_stride << a.v.page_shift) / PRM_TILE;
    long long most = 2 * ctx->n_cu / longs;
    if (most > PRM_MAX_PIECES) most = PRM_MAX_PIECES;
    if (most > tiles / PRM_PIECE_TILES) most = tiles / PRM_PIECE_TILES;
    if (most > room / longs) most = room / longs;
    if (most > 1) pieces.most = (int)most;
  }
  // (some 10^7 workgroups at most: n_rows * n_heads <= 2^30)
  const dim3 grid((unsigned)(wgs + longs * pieces.most)), threads(SPL_THREADS);
  if (ctx->paged_f16_weights)
    hipLaunchKernelGGL((paged_mixed_kernel<HD, false>), grid, threads, lds, ctx->stream, p, pieces, (int)wgs, (int)longs);
  else
    hipLaunchKernelGGL((paged_mixed_kernel<HD, true>), grid, threads, lds, ctx->stream, p, pieces, (int)wgs, (int)longs);
  AF_LAUNCH_CHECK();
  return AF_OK;
}

extern "C" int af_paged_attention(af_ctx* ctx, const af_paged_cache* cache, const af_paged_batch* batch, int n_heads,
                                  float scale, int window, int n_sink, const void* q_f16, long long q_stride,
                                  void* out_f16, long long out_stride) {
  PagedAttnParams p;
  if (!ctx) return AF_ENULL;
  int rc = af_paged_view(cache, batch, n_heads, &p.v);
  if (rc != AF_OK) return rc;
  if ((!q_f16 || !out_f16) && batch->n_rows) return AF_ENULL;
  const int hd = cache->head_dim;
  p.scale2 = (scale == 0.f ? 1.0f / sqrtf((float)hd) : scale) * 1.44269504088896340736f;
  if (window < 0 || n_sink < 0 || !(fabsf(p.scale2) < INFINITY)) return AF_EINVAL;
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
  return hd == 128 ? launch_attention<128>(ctx, p) : launch_attention<64>(ctx, p);
}

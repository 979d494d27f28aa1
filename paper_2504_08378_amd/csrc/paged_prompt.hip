// Attention of prompts over a paged cache: many rows of a sequence at a time, on the matrix cores.
//
// A workgroup has 128 rows, (token, query head) pairs that share a key head, and goes through the keys that any of
// them sees, 64 at a time; a wave has 32 of the rows.
//   scores   S^T[key][row] = K Q^T, 32 x 32 per instruction: a row's scores lie in the registers of two lanes, so its
//            maximum and sum run along registers and one exchange;
//   values   O^T[dim][row] = V^T P^T: which eight keys a lane supplies per instruction is free as long as both operands
//            agree, so it supplies those whose weights it has; V comes out of LDS transposed.
// Pages go to LDS by direct loads, two tiles deep: the next tile is on its way while this one is used.  LDS rows
// hold their 16-byte pieces in an order that depends on the row, so that the lanes of a read, which stand in one
// column of up to 16 rows, lie in different banks; the loads pick the pieces from memory in that order.
#include <math.h>

#include "paged_attn.h"

#define PRM_THREADS 256
#define PRM_ROWS 128
#define PRM_TILE 64

typedef float prm_f16 __attribute__((ext_vector_type(16)));
typedef half_t prm_h4 __attribute__((ext_vector_type(4)));
typedef __fp16 prm_fp16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void prm_lds;
typedef __attribute__((address_space(1))) const void prm_glb;

template <int HD>
__global__ __launch_bounds__(PRM_THREADS, 2) void paged_prompt_kernel(PagedAttnParams p, int short_q) {
  constexpr int KS = HD / 16;        // contraction steps of the scores
  constexpr int DB = HD / 32;        // blocks of 32 dimensions
  constexpr int CH = HD / 8;         // 16-byte pieces of a row
  constexpr int RPI = AF_WAVE / CH;  // rows of a load instruction
  constexpr int NI = 16 / RPI;       // load instructions of a wave per tile, for its 16 keys
  __shared__ __align__(16) half_t s_k0[PRM_TILE * HD], s_k1[PRM_TILE * HD], s_v0[PRM_TILE * HD], s_v1[PRM_TILE * HD];
  __shared__ __align__(16) int s_bad[2][4];

  const PagedView& v = p.v;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int rep = p.n_heads / v.n_kv, window = p.window, n_sink = p.n_sink;
  const int kvh = (int)(blockIdx.x % (unsigned)v.n_kv);

  // which sequence, and which of its 128 rows: the last ones first, they see most
  int b = -1, tile = (int)(blockIdx.x / (unsigned)v.n_kv);
  PagedSeq seq{0, 0, 0};
  for (int b0 = 0; b0 < v.n_seqs && b < 0; b0 += AF_WAVE) {
    PagedSeq s{0, 0, 0};
    if (b0 + lane < v.n_seqs) s = paged_seq(v, b0 + lane);
    const int tiles = s.q_len > short_q ? (int)(((long long)s.q_len * rep + PRM_ROWS - 1) / PRM_ROWS) : 0;
    const int incl = (int)af_wave_incl_scan((unsigned)tiles);
    const unsigned long long hit = __ballot(tile < incl);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      b = b0 + l;
      tile = __builtin_amdgcn_readlane(incl, l) - 1 - tile;
      seq = PagedSeq{__builtin_amdgcn_readlane(s.row0, l), __builtin_amdgcn_readlane(s.q_len, l), __builtin_amdgcn_readlane(s.len, l)};
    } else {
      tile -= __builtin_amdgcn_readlane(incl, 63);
    }
  }
  if (b < 0) return;
  const int p0 = seq.len - seq.q_len, last = seq.len - 1, rows_all = seq.q_len * rep;
  const int r0 = tile * PRM_ROWS, r1 = min(r0 + PRM_ROWS, rows_all) - 1;  // rows of the workgroup
  const int wr0 = min(r0 + wave * 32, r1), wr1 = min(r0 + wave * 32 + 31, r1);
  const int r = min(r0 + wave * 32 + n, r1), tok = r / rep, head = kvh * rep + (r - tok * rep), place = p0 + tok;
  const int wp0 = p0 + wr0 / rep, wp1 = p0 + wr1 / rep;  // places of the wave's rows
  const PagedTiles tl = paged_tiles<PRM_TILE>(p0 + r0 / rep, p0 + r1 / rep, window, n_sink);

  half8 q[KS];
  const half_t* qsrc = p.q + (size_t)(seq.row0 + tok) * p.q_stride + (size_t)head * HD + h * 8;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    q[s] = *reinterpret_cast<const half8*>(qsrc + s * 16);
    if (p.scale2 < 0.f) q[s] = -q[s];  // so that the largest product is the largest score
  }
  const float scale2 = fabsf(p.scale2);

  // loads: row 16 wave + i RPI + lane / CH of the tile, the piece that belongs where the lane writes
  const int lr = lane / CH, lc = lane % CH;
  const int32_t* table = v.table + (size_t)b * v.table_stride;
  const int mask = (1 << v.page_shift) - 1;
  int id = 0;
  auto page_of = [&](int t) __attribute__((always_inline)) {
    id = table[min(paged_tile_start<PRM_TILE>(tl, min(t, tl.n - 1)) + wave * 16, last) >> v.page_shift];
  };
  auto fetch = [&](int t, half_t* sk, half_t* sv, int* sb) __attribute__((always_inline)) {
    const int pg = __builtin_amdgcn_readfirstlane(id);
    const bool bad = !paged_page_ok(v, pg);
    if (lane == 0) {
      sb[wave] = bad;
      if (bad) paged_report(v);
    }
    const size_t base = (size_t)(bad ? 0 : pg) * (size_t)v.page_stride + ((size_t)kvh << v.page_shift) * HD;
    const int k0 = paged_tile_start<PRM_TILE>(tl, t) + wave * 16;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = i * RPI + lr;
      const unsigned o = (unsigned)(min(k0 + row, last) & mask) * HD;
      const int ck = lc ^ (row & (CH - 1)), cv = lc ^ (HD == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2);
      __builtin_amdgcn_global_load_lds((prm_glb*)(v.k + base + o + ck * 8), (prm_lds*)(sk + (wave * 16 + i * RPI) * HD), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((prm_glb*)(v.v + base + o + cv * 8), (prm_lds*)(sv + (wave * 16 + i * RPI) * HD), 16, 0, 0);
    }
  };
  // reads: a key's row for the scores; four keys of one dimension for the values
  const int i16 = lane & 15;
  const int kat = n * HD, kx = h ^ (lane & (CH - 1));
  const int vrow = 4 * h + (i16 >> 2), vx = HD == 128 ? i16 >> 2 : i16 >> 3;
  const int vlow = ((lane >> 4) & 1) * 16 + (i16 & 3) * 4;

  prm_f16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = prm_f16{};
  float m = -INFINITY, l = 0.f;

  auto compute = [&](int t, const half_t* sk, const half_t* sv, const int* sb) __attribute__((always_inline)) {
    const int k0 = paged_tile_start<PRM_TILE>(tl, t);
    if (!(k0 <= wp1 && (window <= 0 || k0 + PRM_TILE - 1 > wp0 - window || k0 < n_sink))) return;
    // Reads run ahead of the products that use them: both blocks of keys before the first product, the first
    // values under the second block's, each block of values under the one before.
    auto keys = [&](half8 (&a)[KS], int kb) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[ks] = *reinterpret_cast<const half8*>(sk + kb * 32 * HD + kat + ((ks * 2) ^ kx) * 8);
    };
    auto values = [&](half8 (&a)[4], int d) __attribute__((always_inline)) {
#pragma unroll
      for (int s4 = 0; s4 < 4; ++s4) {
        const half_t* at = sv + (vrow + 16 * s4) * HD + ((d ^ vx) * 32 + vlow);
        const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) prm_fp16x4*)at);
        const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) prm_fp16x4*)(at + 8 * HD));
        a[s4] = __builtin_shufflevector(__builtin_bit_cast(prm_h4, lo), __builtin_bit_cast(prm_h4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    const int4 bad = *reinterpret_cast<const int4*>(sb);
    prm_f16 s[2] = {prm_f16{}, prm_f16{}};
    half8 a0[KS], a1[KS], v0[4], v1[4];
    keys(a0, 0);
    keys(a1, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a0[ks], q[ks], s[0], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    values(v0, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a1[ks], q[ks], s[1], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (!(k0 + PRM_TILE - 1 <= wp0 && (window <= 0 || k0 > wp1 - window || k0 + PRM_TILE <= n_sink))) {
      const int end = place - k0 - 4 * h, from = (window > 0 ? place - window + 1 : 0) - k0 - 4 * h, first = n_sink - k0 - 4 * h;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = kb * 32 + (i & 3) + 8 * (i >> 2);
          s[kb][i] = (row <= end) & ((row >= from) | (row < first)) ? s[kb][i] : -INFINITY;
        }
    }
    if (bad.x | bad.y | bad.z | bad.w) {
      const int gone[4] = {bad.x, bad.y, bad.z, bad.w};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = gone[kb * 2 + (i >> 3)] ? -INFINITY : s[kb][i];
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, AF_WAVE)) * scale2;
    if (__any(mx > m)) {
      mx = fmaxf(mx, m);
      const float corr = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
      m = mx;
      l *= corr;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= corr;
    }
    // Weights times 2^15 (in the range of fp16), each to the nearest of its 11 bits: one more rounding of the size of the
    // result's own, and independent from key to key.
    const float off = (m == -INFINITY ? 0.f : -m) + 15.f;
    half8 w[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], scale2, off));
        l += e;
        w[kb * 2 + (i >> 3)][i & 7] = (half_t)e;
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int d = 0; d < DB; d += 2) {
      values(v1, d + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s4 = 0; s4 < 4; ++s4) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v0[s4], w[s4], o[d], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (d + 2 < DB) values(v0, d + 2);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s4 = 0; s4 < 4; ++s4) o[d + 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1[s4], w[s4], o[d + 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // every wave's loads are in LDS (the barrier alone does not wait for loads that go there directly)
  auto landed = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
  };

  page_of(0);
  fetch(0, s_k0, s_v0, s_bad[0]);
  page_of(1);
  for (int t = 0; t < tl.n; t += 2) {
    landed();
    if (t + 1 < tl.n) {
      fetch(t + 1, s_k1, s_v1, s_bad[1]);
      page_of(t + 2);
    }
    compute(t, s_k0, s_v0, s_bad[0]);
    if (t + 1 >= tl.n) break;
    landed();
    if (t + 2 < tl.n) {
      fetch(t + 2, s_k0, s_v0, s_bad[0]);
      page_of(t + 3);
    }
    compute(t + 1, s_k1, s_v1, s_bad[1]);
  }

  if (r0 + wave * 32 > r1) return;
  l += __shfl_xor(l, 32, AF_WAVE);
  const bool mine = r0 + wave * 32 + n <= r1;
  const float inv = 1.0f / l;
  bool odd = false;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      o[d][i] *= inv;
      odd |= o[d][i] != o[d][i];
    }
  // A result that is not a number (an infinity among what was read, seen or not; nothing seen) is formed again key by key.
  const unsigned long long again = __ballot(odd && mine);
  unsigned todo = (unsigned)again | (unsigned)(again >> 32);
  if (mine && !(todo >> n & 1)) {
    half_t* dst = p.out + (size_t)(seq.row0 + tok) * p.out_stride + (size_t)head * HD + 4 * h;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<prm_h4*>(dst + d * 32 + i * 8) =
            prm_h4{(half_t)o[d][i * 4], (half_t)o[d][i * 4 + 1], (half_t)o[d][i * 4 + 2], (half_t)o[d][i * 4 + 3]};
  }
  while (todo) {
    const int k = __builtin_ctz(todo);
    todo &= todo - 1;
    const int rr = r0 + wave * 32 + k, tt = rr / rep;
    paged_row<HD>(p, b, seq.row0 + tt, p0 + tt, kvh * rep + (rr - tt * rep));
  }
}

int af_launch_paged_prompt(af_ctx* ctx, const PagedAttnParams& a, int head_dim, int short_q) {
  // as many workgroups as any division of the rows among the sequences can need
  const long long rep = a.n_heads / a.v.n_kv, rows = (long long)a.v.n_rows * rep;
  const long long longer = a.v.n_rows / (short_q + 1), seqs = a.v.n_seqs < longer ? a.v.n_seqs : longer;
  const long long wgs = (rows / PRM_ROWS + seqs) * a.v.n_kv;
  if (wgs > 0x7FFFFFFF) return AF_EINVAL;
  if (wgs == 0) return AF_OK;
  if (head_dim == 128)
    hipLaunchKernelGGL(paged_prompt_kernel<128>, dim3((unsigned)wgs), dim3(PRM_THREADS), 0, ctx->stream, a, short_q);
  else
    hipLaunchKernelGGL(paged_prompt_kernel<64>, dim3((unsigned)wgs), dim3(PRM_THREADS), 0, ctx->stream, a, short_q);
  AF_LAUNCH_CHECK();
  return AF_OK;
}

// Attention of prompts over a paged cache: many rows of a sequence at a time, on the matrix cores.
//
// A workgroup has 128 rows, (token, query head) pairs that share a key head, and goes through the keys that any of
// them sees, 64 at a time (four sixteens, each in one page: the first tokens and a window make one list); a wave has 32 of
// the rows.
//   scores   S^T[key][row] = K Q^T, 32 x 32 per instruction: a row's scores lie in the registers of two lanes;
//   values   O^T[dim][row] = V^T P^T: which eight keys a lane supplies per instruction is free as long as both operands
//            agree, so it supplies those whose weights it has; V comes out of LDS transposed.
// Pages go to LDS by direct loads, two tiles deep: the next tile is on its way while this one is used.  LDS rows
// hold their 16-byte pieces in an order that depends on the row, so that the lanes of a read, which stand in one
// column of up to 16 rows, lie in different banks (the conflict counter reads 0); the loads pick the pieces from memory in
// that order.
//
// The weights enter the value products as two fp16 values, 22 bits, so these are formed twice: 1.5 times the matrix work of weights
// rounded to fp16, which leave the results up to 2.6e-4 from 64 bits where their own rounding leaves 2.0e-4.  The caller may choose
// those (FINE false).
//
// What bounds it, 8192 tokens of 32 heads on 32, causal, 550 GFLOP and 275 more for the second value products: 762 us, 1080 TFLOP/s; the
// matrix unit is busy 64 % of the cycles, and the clock is the 1.58 GHz that power allows.  Rounded weights: 581 us, 51 % at 1.73 GHz.  (A
// loop of nothing but these instructions on random data runs at 1.6 GHz, 1650 TFLOP/s, and at 2.1 GHz on zeros.)  In the other cycles
// neither of the two waves of a SIMD has products ready.  On the way, us, with rounded weights: all loads of a tile issued in a row at its
// start, where a wave waits until the memory path has taken them, and each read next to its product 669; a maximum per tile and an
// exchange between the lanes 655; loads between the products, with reads that the compiler could not tell from the loads' buffers (it
// waited for them) 667; this form 573.  Eight waves on one pair of tiles, half of them a phase behind the others, 573; without the
// waves' priorities 587.
#pragma once
#include <type_traits>

#include "paged_attn.h"

#define PRM_WAVES 4
#define PRM_ROWS (32 * PRM_WAVES)
#define PRM_SPAN 16                        // keys that a wave loads of a tile: never in two pages
#define PRM_TILE (PRM_WAVES * PRM_SPAN)
typedef float prm_f16 __attribute__((ext_vector_type(16)));
typedef float prm_f2 __attribute__((ext_vector_type(2)));
typedef half_t prm_h2 __attribute__((ext_vector_type(2)));
typedef half_t prm_h4 __attribute__((ext_vector_type(4)));
typedef __fp16 prm_fp16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void prm_lds;
typedef __attribute__((address_space(1))) const void prm_glb;

// Where few workgroups would go through many keys, several share the rows of one, each with a piece of its tiles:
// their maxima, sums and values meet in memory, and the one that finishes last joins them, in order.
struct PagedPieces {
  float* part;   // [workgroup][most][PRM_PIECE_FLOATS]
  int* tickets;  // of the workgroups, zero between launches
  int ticket0, most;
};
#define PRM_MAX_PIECES 16
#define PRM_PIECE_TILES 8  // tiles of a piece, at least
#define PRM_PIECE_FLOATS(HD) ((size_t)PRM_WAVES * AF_WAVE * ((HD) / 2 + 2))
PAGED_HD int paged_pieces(int tiles, int most) {
  const int n = tiles / PRM_PIECE_TILES;
  return n < 1 ? 1 : n < most ? n : most;
}

// s_k0 .. s_v1: LDS of PRM_TILE * HD elements each, objects of their own.  piece: which of a workgroup's pieces.
// FINE: weights of 22 bits, else of 11.
template <int HD, bool FINE>
__device__ __forceinline__ void paged_prompt_body(const PagedAttnParams& p, const PagedPieces& pieces, const int short_q,
                                                  const unsigned wg, const int piece, half_t* s_k0, half_t* s_k1, half_t* s_v0,
                                                  half_t* s_v1) {
  constexpr int KS = HD / 16;        // contraction steps of the scores
  constexpr int DB = HD / 32;        // blocks of 32 dimensions
  constexpr int CH = HD / 8;         // 16-byte pieces of a row
  constexpr int RPI = AF_WAVE / CH;  // rows of a load instruction
  constexpr int NI = PRM_SPAN / RPI; // load instructions of a wave per tile
  __shared__ int s_gone;  // a page of this workgroup does not exist
  __shared__ int s_ticket;

  const PagedView& v = p.v;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int rep = p.n_heads / v.n_kv, window = p.window, n_sink = p.n_sink;
  const int kvh = (int)(wg % (unsigned)v.n_kv);

  // which sequence, and which of its 128 rows: the last ones first, they see most
  int b = -1, tile = (int)(wg / (unsigned)v.n_kv);
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
  const PagedTiles tl = paged_tiles<PRM_SPAN>(p0 + r0 / rep, p0 + r1 / rep, window, n_sink);
  const int tiles = (tl.n + PRM_WAVES - 1) / PRM_WAVES, shares = paged_pieces(tiles, pieces.most);
  if (piece >= shares) return;
  const int t0 = (int)((long long)tiles * piece / shares), t1 = (int)((long long)tiles * (piece + 1) / shares);

  // loads: row 16 wave + i RPI + lane / CH of the tile, the piece that belongs where the lane writes
  const int lr = lane / CH, lc = lane % CH;
  const int32_t* table = v.table + (size_t)b * v.table_stride;
  const int mask = (1 << v.page_shift) - 1;
  // where the page of the keys and of the values that are fetched next begins, and the number of the one behind them
  size_t page_k, page_v;
  int id_next;
  auto page_of = [&](int t) __attribute__((always_inline)) {
    return table[paged_tile_start<PRM_SPAN>(tl, min(t * PRM_WAVES + wave, tl.n - 1)) >> v.page_shift];
  };
  auto turn_page = [&]() __attribute__((always_inline)) {
    int id = __builtin_amdgcn_readfirstlane(id_next);
    if (!paged_page_ok(v, id)) {  // the first page is read in its place, and hidden
      id = 0;
      s_gone = 1;
      paged_report(v);
    }
    page_v = page_k;
    page_k = (size_t)id * (size_t)v.page_stride + ((size_t)kvh << v.page_shift) * HD;
  };
  // Load instruction i of tile t's, and behind the last keys of those once more.
  auto fetch = [&](const half_t* page, int t, half_t* to, int i, bool keys) __attribute__((always_inline)) {
    const int row = i * RPI + lr, k0 = paged_tile_start<PRM_SPAN>(tl, min(t * PRM_WAVES + wave, tl.n - 1));
    const unsigned o = (unsigned)(min(k0 + row, last) & mask) * HD;
    const int c = lc ^ (keys ? row & (CH - 1) : HD == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2);
    __builtin_amdgcn_global_load_lds((prm_glb*)(page + (o + c * 8)), (prm_lds*)(to + (wave * PRM_SPAN + i * RPI) * HD), 16, 0, 0);
  };
  auto sync = []() __attribute__((always_inline)) {  // lgkmcnt(0) and the barrier: loads stay in flight over it
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };

  // The first tile's keys and values and the second's keys are requested together; the first step waits for the first keys only
  // (8932 rows that see 1028 keys each, rounded weights, us: with only the keys at first 181.4, so 178.3).
  if (tid == 0) s_gone = 0;
  id_next = page_of(t0);
  const int id_second = page_of(t0 + 1);
  sync();
  page_k = 0;
  turn_page();
#pragma unroll
  for (int i = 0; i < NI; ++i) fetch(v.k + page_k, t0, s_k0, i, true);
  asm volatile("" ::: "memory");
  half8 q[KS];
  const half_t* qsrc = p.q + (size_t)(seq.row0 + tok) * p.q_stride + (size_t)head * HD + h * 8;
#pragma unroll
  for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const half8*>(qsrc + s * 16);
  asm volatile("" ::: "memory");
  id_next = id_second;
  turn_page();
#pragma unroll
  for (int i = 0; i < NI; ++i) fetch(v.v + page_v, t0, s_v0, i, false);
#pragma unroll
  for (int i = 0; i < NI; ++i) fetch(v.k + page_k, t0 + 1, s_k1, i, true);
  asm volatile("" ::: "memory");
  const float scale2 = fabsf(p.scale2);

  // Reads: a key's row for the scores; four keys of one dimension for the values.  The lane's places are kept as numbers that
  // the compiler does not look into: it takes reads whose address it cannot trace to one buffer for reads of what is being
  // loaded, and waits for the loads.
  const int i16 = lane & 15, kx = h ^ (lane & (CH - 1)), vx = HD == 128 ? i16 >> 2 : i16 >> 3;
  int kat[KS], vat[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kat[ks] = n * HD + ((ks * 2) ^ kx) * 8;
    asm volatile("" : "+v"(kat[ks]));
  }
#pragma unroll
  for (int d = 0; d < DB; ++d) {
    vat[d] = (4 * h + (i16 >> 2)) * HD + (d ^ vx) * 32 + ((lane >> 4) & 1) * 16 + (i16 & 3) * 4;
    asm volatile("" : "+v"(vat[d]));
  }
  auto key = [&](const half_t* sk, int kb, int ks) __attribute__((always_inline)) {
    return *reinterpret_cast<const half8*>(&sk[kat[ks] + kb * 32 * HD]);
  };
  auto value = [&](const half_t* sv, int d, int s4) __attribute__((always_inline)) {
    const auto lo = __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) prm_fp16x4*)&sv[vat[d] + 16 * s4 * HD]);
    const auto hi = __builtin_amdgcn_ds_read_tr16_b64_v4f16((__attribute__((address_space(3))) prm_fp16x4*)&sv[vat[d] + (16 * s4 + 8) * HD]);
    return (half8)__builtin_shufflevector(__builtin_bit_cast(prm_h4, lo), __builtin_bit_cast(prm_h4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
  };

  prm_f16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = prm_f16{};
  float m = -INFINITY, l = 0.f;

  // Scores that a row does not see, behind the products of tile t.
  auto hide = [&](int t, prm_f16 (&s)[2]) __attribute__((always_inline)) {
    const int first = t * PRM_WAVES, k0 = paged_tile_start<PRM_SPAN>(tl, first);
    const bool whole = first >= tl.sinks || first + PRM_WAVES <= tl.sinks;  // 64 neighbours
    if (!(whole && k0 + PRM_TILE - 1 <= wp0 && (window <= 0 || k0 > wp1 - window || k0 + PRM_TILE <= n_sink))) {
      const int from = window > 0 ? max(0, place - window + 1) : 0, sinks = min(n_sink, from);
      const unsigned span = (unsigned)(place - from);  // seen: from .. place, and what is below sinks
#pragma unroll
      for (int g = 0; g < PRM_WAVES; ++g) {
        const int k = paged_tile_start<PRM_SPAN>(tl, first + g) + 4 * h, above = k - from, sink = sinks - k;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int row = (i & 3) + 8 * (i >> 2), e = (g & 1) * 8 + i;
          s[g >> 1][e] = (((unsigned)(above + row) <= span) | (row < sink)) ? s[g >> 1][e] : -INFINITY;
        }
      }
    }
    if (s_gone) {
#pragma unroll
      for (int g = 0; g < PRM_WAVES; ++g) {
        const int k = paged_tile_start<PRM_SPAN>(tl, first + g);
        if (k <= last && paged_page_ok(v, __builtin_amdgcn_readfirstlane(table[k >> v.page_shift]))) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[g >> 1][(g & 1) * 8 + i] = -INFINITY;
      }
    }
  };
  half8 w[4], wr[FINE ? 4 : 1];  // the weights' rounded values, and what the rounding left
  // The matrix unit's half of a step: the values of tile t - 1 (sv) by its weights, the scores of tile t (keys sk).
  prm_f16 s[2];
  auto products = [&](auto first, const half_t* sk, const half_t* sv, auto&& between) __attribute__((always_inline)) {
    constexpr int AHEAD = FINE ? 3 : 4, RING = FINE ? 4 : 8;
    half8 x[RING], a[2][KS];
    // Every read of values stands AHEAD of its products (three pairs or four), every read of keys a block; the compiler would move
    // it next to them.
    if constexpr (!first.value) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) x[i] = value(sv, 0, i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
#pragma unroll
        for (int s4 = 0; s4 < 4; ++s4) {
          const int now = d * 4 + s4, next = now + AHEAD;
          if (next < DB * 4) x[next % RING] = value(sv, next >> 2, next & 3);
          if (d + 1 == DB && s4 * 2 < KS) {
            a[0][s4 * 2] = key(sk, 0, s4 * 2);
            a[0][s4 * 2 + 1] = key(sk, 0, s4 * 2 + 1);
          }
          if constexpr (FINE) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[now % RING], wr[s4], o[d], 0, 0, 0);
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[now % RING], w[s4], o[d], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        between(d);
      }
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[0][ks] = key(sk, 0, ks);
#pragma unroll
      for (int d = 0; d < DB; ++d) between(d);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) s[kb] = prm_f16{};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      a[1][ks] = key(sk, 1, ks);
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0][ks], q[ks], s[0], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1][ks], q[ks], s[1], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // The vector unit's half: the scores to weights, times 2^7, each to the nearest of its 11 bits and, FINE, what is left to the
  // nearest of another 11 (below 2^-32 of the row's largest weight there are none).  Without the rest each is off by 2^-11 of itself
  // at most, independent from key to key: the caller's choice.  Returns their sum, without the rest that of the rounded ones.
  auto weigh = [&]() __attribute__((always_inline)) {
    const float off = (m == -INFINITY ? 0.f : -m) + 7.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float x = s[i >> 4][i & 15], y = s[i >> 4][(i & 15) + 1];
      const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale2, off)), e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(y, scale2, off));
      const prm_h2 hi = __builtin_convertvector((prm_f2{e0, e1}), prm_h2);
      w[i >> 3][i & 7] = hi[0];
      w[i >> 3][(i & 7) + 1] = hi[1];
      if constexpr (FINE) {
        const prm_h2 rest = __builtin_convertvector((prm_f2{e0 - (float)hi[0], e1 - (float)hi[1]}), prm_h2);
        sum += e0 + e1;
        wr[i >> 3][i & 7] = rest[0];
        wr[i >> 3][(i & 7) + 1] = rest[1];
      } else {
        sum = __builtin_amdgcn_fdot2(hi, prm_h2{(half_t)1, (half_t)1}, sum, false);
      }
    }
    return sum;
  };
  // m is the largest score of the tiles up to the one that set it.  While the weights of a tile stay in range (the largest below
  // 2^9 times that score's, or the sum would not be), it need not follow; if a row's do not, or it has seen nothing so far, it
  // does, and what has been summed is scaled.  So most tiles need no maximum and no exchange between lanes.  The first tile begins
  // with its maximum.
  auto weights = [&](auto first, int t) __attribute__((always_inline)) {
    hide(t, s);
    float sum = 0.f;
    if constexpr (!first.value) sum = weigh();
    if (first.value || !__all(sum <= 65504.f && m > -INFINITY)) {
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) mx = fmaxf(mx, s[i >> 4][i & 15]);
      mx = fmaxf(fmaxf(mx, __shfl_xor(mx, 32, AF_WAVE)) * scale2, m);
      if constexpr (!first.value) {
        const float corr = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mx);
        l *= corr;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= corr;
      }
      m = mx;
      sum = weigh();
    }
    l += sum;
    __builtin_amdgcn_sched_barrier(0);
  };
  auto wait_loads = [&]() __attribute__((always_inline)) {  // vmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);
    turn_page();
  };

  // Step t: products (values of t - 1, scores of t), then weights of t.  Keys of t and values of t - 1 are read in one step; the
  // next ones, keys of t + 1 and values of t, are fetched meanwhile to the other buffers, which the step before has read.
  // A barrier alone does not wait for loads that go to LDS directly.
  auto step = [&](auto first, int t, half_t* k_now, half_t* k_next, half_t* v_before, half_t* v_now) __attribute__((always_inline)) {
    __builtin_amdgcn_s_setprio(1);  // of the two waves of a SIMD, the one with products goes first
    products(first, k_now, v_before, [&](int d) __attribute__((always_inline)) {
      constexpr int PER = (2 * NI + DB - 1) / DB;
#pragma unroll
      for (int i = d * PER; i < (d + 1) * PER && i < 2 * NI; ++i) {
        if constexpr (first.value) break;  // requested already
        if (i < NI)
          fetch(v.v + page_v, t, v_now, i, false);
        else
          fetch(v.k + page_k, t + 1, k_next, i - NI, true);
      }
      if (d == DB - 1) id_next = page_of(t + 2);
      __builtin_amdgcn_sched_barrier(0);
    });
    __builtin_amdgcn_s_setprio(0);
    weights(first, t);
    wait_loads();
    sync();
  };
  __builtin_amdgcn_s_waitcnt(0x0F70 | 2 * NI);  // vmcnt(2 NI): the first keys are there, and the queries
  sync();
  if (p.scale2 < 0.f) {  // so that the largest product is the largest score
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = -q[s];
  }
  step(std::true_type{}, t0, s_k0, s_k1, s_v1, s_v0);
  for (int t = t0 + 1; t < t1; t += 2) {
    step(std::false_type{}, t, s_k1, s_k0, s_v0, s_v1);
    if (t + 1 < t1) step(std::false_type{}, t + 1, s_k0, s_k1, s_v1, s_v0);
  }
  auto finish = [&](const half_t* sv) __attribute__((always_inline)) {  // the last values
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int s4 = 0; s4 < 4; ++s4) {
        const half8 x = value(sv, d, s4);
        if constexpr (FINE) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, wr[s4], o[d], 0, 0, 0);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, w[s4], o[d], 0, 0, 0);
      }
  };
  if ((t1 - t0) & 1)
    finish(s_v0);
  else
    finish(s_v1);

  const bool rows = r0 + wave * 32 <= r1;  // this wave has any
  if (shares > 1) {
    // a thread's pairs of values, 512 bytes of a wave next to each other: (m, l), then o
    auto at = [&](int z, int k) __attribute__((always_inline)) {
      return pieces.part + ((size_t)wg * pieces.most + z) * PRM_PIECE_FLOATS(HD) + ((size_t)k * PRM_WAVES * AF_WAVE + tid) * 2;
    };
    if (rows) {
      af_store_agent2(at(piece, 0), m, l);
#pragma unroll
      for (int k = 0; k < HD / 4; ++k) af_store_agent2(at(piece, 1 + k), o[k >> 3][2 * k & 15], o[k >> 3][(2 * k & 15) + 1]);
    }
    af_stores_done();
    __syncthreads();
    if (tid == 0) {
      int* ticket = &pieces.tickets[af_ticket_of(pieces.ticket0 + (int)wg)];
      s_ticket = af_ticket_take(ticket);
      if (s_ticket == shares - 1) af_ticket_reset(ticket);
    }
    __syncthreads();
    if (s_ticket != shares - 1 || !rows) return;
    m = -INFINITY;
    for (int z = 0; z < shares; ++z) m = fmaxf(m, af_load_agent2(at(z, 0))[0]);
    const float safe = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = prm_f16{};
    for (int z = 0; z < shares; ++z) {
      const af_float2 ml = af_load_agent2(at(z, 0));
      af_float2 x[HD / 4];
#pragma unroll
      for (int k = 0; k < HD / 4; ++k) x[k] = af_load_agent2(at(z, 1 + k));
      const float f = __builtin_amdgcn_exp2f(ml[0] - safe);
      l += f * ml[1];
#pragma unroll
      for (int k = 0; k < HD / 4; ++k) {
        o[k >> 3][2 * k & 15] += f * x[k][0];
        o[k >> 3][(2 * k & 15) + 1] += f * x[k][1];
      }
    }
  }
  if (!rows) return;
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

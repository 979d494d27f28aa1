// Attention of few rows over a paged cache: single tokens (or a few) per sequence, one pass over the keys, split over
// their length.
//
// Up to 16 rows, (token, query head) pairs that share a key head, are the columns of 16 x 16 x 32 products; every key and value is read
// once for all of them.  A wave takes 32 keys at a time, straight to registers, and keeps a running softmax of its own:
//   scores   D[key][row] = K Q^T: a lane supplies eight dimensions of one key, which is the load it has made;
//   values   D[dim][row] = V^T P^T: a lane supplies the eight keys whose weights it has, picked out of the rows by byte permutation.
// The page numbers of the next step travel with the rows of this one.
// What bounds it: the read of the cache, 6.4 TB/s of the 6.7 of a plain read while all workgroups read (131070 keys of 8 key heads: 84 us, and 9
// for the joins; 64 sequences of up to 8190: 108 and 5), latency where there is little (512 keys of 32 heads 7.9: 5.9 to the sums of a
// workgroup, 2.0 for the join).  Two workgroups a compute unit (211 registers): three, with 168, 118 for the 95 that it took then, four
// launched 127; loads that stay in the caches 112; one of eight waves 91, but 512 keys of 32 heads 10.5 for 9.2.
#pragma once
#include "paged_attn.h"

#define SPL_THREADS 256
#define SPL_WAVES (SPL_THREADS / AF_WAVE)
#define SPL_STEP 32                      // keys of a wave at a time
#define SPL_ROWS 16                      // rows (query heads x tokens that share a key head) of a workgroup
#define SPL_RW (SPL_ROWS / SPL_WAVES)    // of them a wave's, in the sums
#define SPL_JOIN 16                      // partial results that are joined at once
#define SPL_MAX_WGS 1024                 // workgroups: SPL_JOIN sets of them, at most 64, are joined by one wave

typedef float spl_f4 __attribute__((ext_vector_type(4)));
typedef half_t spl_h2 __attribute__((ext_vector_type(2)));

struct PagedSplitParams {
  PagedAttnParams a;
  float* part;       // [2 wgs][slot_rows][HD + 2]
  int* tickets;      // two per workgroup, zero between launches
  int slot_rows;     // most rows of a group
  int short_q;       // sequences with more new tokens are the other kernel's
};

PAGED_HD int paged_split_units(const PagedTiles& t) { return t.n > SPL_WAVES ? (t.n + SPL_WAVES - 1) / SPL_WAVES : 1; }
static inline size_t paged_split_lds(int n_seqs) {
  return ((size_t)n_seqs + 1) * sizeof(unsigned long long) + (size_t)n_seqs * sizeof(PagedSeq);
}

// The work of the launch is a line of units, a step of each of the four waves for one group of rows, in the order sequence, key
// head, group, key; every workgroup takes an equal stretch of it.  A group whose units lie in several stretches is joined by the
// workgroup that finishes last.  (Stretches of single steps balanced better under a window, 35.3 for the 36.8 us of then, but cut more
// groups and put short ones on single waves: eight sequences of up to 517 keys 15.6 for 10.4, 256 of up to 1500 106 for 95.)
// wg of wgs workgroups; acc: LDS for a wave's sums each, [SPL_ROWS][HD + 4]; s_first: LDS of paged_split_lds() bytes.
template <int HD>
__device__ __forceinline__ void paged_split_body(const PagedSplitParams& p, const int wg, const int wgs,
                                                 float* const (&acc_lds)[SPL_WAVES], unsigned long long* s_first) {
  constexpr int TT = HD / 32;   // contraction steps of the scores
  constexpr int VC = HD / 16;   // value columns of a lane
  typedef half_t vrow __attribute__((ext_vector_type(VC)));
  typedef unsigned vwords __attribute__((ext_vector_type(VC / 2)));
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  typedef unsigned long long u64;
  PagedSeq* s_seq = reinterpret_cast<PagedSeq*>(s_first + p.a.v.n_seqs + 1);  // s_first[n_seqs + 1]: first unit of each
  __shared__ float2 s_ml[SPL_WAVES][SPL_ROWS];
  __shared__ u64 s_sum[SPL_WAVES];
  __shared__ int s_b, s_last;

  const PagedView& v = p.a.v;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int rep = p.a.n_heads / v.n_kv, window = p.a.window, n_sink = p.a.n_sink;

  // Units of the sequences, summed.  Up to 64 sequences: by every wave for itself, a lane has one (0.3 us less than the other way,
  // at any length); more: in LDS.
  const bool few = v.n_seqs <= AF_WAVE;
  const int per = (v.n_seqs + SPL_THREADS - 1) / SPL_THREADS;
  PagedSeq own{0, 0, 0};
  u64 mine = 0, total = 0, before = 0;
  unsigned units_own = 0;  // of a group of the lane's sequence
  auto units_of = [&](const PagedSeq& s) __attribute__((always_inline)) -> u64 {
    if (s.q_len <= 0 || s.q_len > p.short_q) return 0;
    units_own = paged_split_units(paged_tiles<SPL_STEP>(s.len - s.q_len, s.len - 1, window, n_sink));
    return (u64)((s.q_len * rep + SPL_ROWS - 1) / SPL_ROWS) * (unsigned)v.n_kv * (u64)units_own;
  };
  auto of_lane = [](u64 x, int l) __attribute__((always_inline)) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, l);
  };
  u64 ends = 0;
  if (few) {
    if (lane < v.n_seqs) {
      own = paged_seq(v, lane);
      mine = units_of(own);
    }
    ends = af_wave_incl_scan(mine);
    total = of_lane(ends, AF_WAVE - 1);
  } else {
    for (int b = tid * per; b < min(tid * per + per, v.n_seqs); ++b) {
      const PagedSeq s = paged_seq(v, b);
      s_seq[b] = s;
      s_first[b] = mine;
      mine += units_of(s);
    }
    ends = af_wave_incl_scan(mine);
    if (lane == 63) s_sum[wave] = ends;
    __syncthreads();
    before = ends - mine;
#pragma unroll
    for (int w = 0; w < SPL_WAVES; ++w) {
      if (w < wave) before += s_sum[w];
      total += s_sum[w];
    }
  }
  const u64 share = total >> 31 ? (total + (unsigned)wgs - 1) / (unsigned)wgs : ((unsigned)total + wgs - 1) / (unsigned)wgs;
  // If every group can begin with a stretch of its own, it does: a workgroup then has one piece and at most one join (32 windows of
  // 1028 keys 35.2 -> 32.2 us, 8 sequences of up to 4000 20.0 -> 19.2; 13 of up to 12102, one key head, 23.3 -> 24.3, and 0.3 to find that
  // they cannot).
  bool apart = false;
  if (few && share > 1 && !(total >> 31) && (long long)v.n_seqs * v.n_kv <= wgs) {
    const unsigned padded = (units_own + (unsigned)share - 1) / (unsigned)share * (unsigned)share;
    const u64 wide = units_own ? mine / units_own * padded : 0;
    const u64 up_to = af_wave_incl_scan(wide), all = of_lane(up_to, AF_WAVE - 1);
    if (all <= (u64)wgs * share) {
      apart = true;
      mine = wide;
      ends = up_to;
      total = all;
    }
  }
  const u64 u0 = (u64)wg * share, u1 = min(u0 + share, total);
  if (u0 >= u1) return;
  int b = 0;
  if (!few) {
    for (int b = tid * per; b < min(tid * per + per, v.n_seqs); ++b) {
      const u64 a = before + s_first[b], e = b + 1 < min(tid * per + per, v.n_seqs) ? before + s_first[b + 1] : before + mine;
      s_first[b] = a;
      if (a <= u0 && u0 < e) s_b = b;
    }
    if (tid == 0) s_first[v.n_seqs] = total;
    __syncthreads();
    b = s_b;
  }

  for (u64 u = u0; u < u1;) {
    PagedSeq seq;
    u64 first_unit;
    if (few) {
      b = __builtin_ctzll(__ballot(u < ends));
      seq = PagedSeq{__builtin_amdgcn_readlane(own.row0, b), __builtin_amdgcn_readlane(own.q_len, b), __builtin_amdgcn_readlane(own.len, b)};
      first_unit = of_lane(ends - mine, b);
    } else {
      while (u >= s_first[b + 1]) ++b;
      seq = s_seq[b];
      first_unit = s_first[b];
    }
    const int p0 = seq.len - seq.q_len, p1 = seq.len - 1, rows_all = seq.q_len * rep, groups = (rows_all + SPL_ROWS - 1) / SPL_ROWS;
    const PagedTiles tl = paged_tiles<SPL_STEP>(p0, p1, window, n_sink);
    const int units = paged_split_units(tl);
    const u64 local = u - first_unit;
    const unsigned span = apart ? ((unsigned)units + (unsigned)share - 1) / (unsigned)share * (unsigned)share : (unsigned)units;
    const unsigned hg = local >> 32 ? (unsigned)(local / span) : (unsigned)local / span;
    const int t0 = (int)(local - (u64)hg * span), t1 = (int)min((u64)units, t0 + (u1 - u));
    const int kvh = groups == 1 ? (int)hg : (int)(hg / (unsigned)groups), grp = (int)hg - kvh * groups;
    const int r0 = grp * SPL_ROWS, rows = min(SPL_ROWS, rows_all - r0);

    // the row of this lane's column: token r / rep, query head r % rep of the key head's
    const int r = r0 + min(n, rows - 1), tok = rep == 1 ? r : r / rep, head = kvh * rep + (r - tok * rep);
    const int place = p0 + tok;
    half8 q[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t)
      q[t] = *reinterpret_cast<const half8*>(p.a.q + (size_t)(seq.row0 + tok) * p.a.q_stride + (size_t)head * HD + t * 32 + g * 8);

    const int32_t* table = v.table + (size_t)b * v.table_stride;
    const int mask = (1 << v.page_shift) - 1, last = seq.len - 1, end = min(t1 * SPL_WAVES, tl.n);  // steps up to here
    int id[2];
    bool bad[2];
    half8 kr[2][TT];
    vrow vr[8];
    // pages of the two 16 keys of a step (what lies behind the sequence's end is read as its last row and masked)
    auto ids = [&](int t) __attribute__((always_inline)) {
      const int k = paged_tile_start<SPL_STEP>(tl, min(t, end - 1));
#pragma unroll
      for (int i = 0; i < 2; ++i) id[i] = table[max(0, min(k + i * 16, last)) >> v.page_shift];
    };
    auto fetch = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int pg = __builtin_amdgcn_readfirstlane(id[i]);
        bad[i] = !paged_page_ok(v, pg);
        const size_t base = (size_t)(bad[i] ? 0 : pg) * (size_t)v.page_stride + ((size_t)kvh << v.page_shift) * HD;
        const half_t *Kc = v.k + base, *Vc = v.v + base;
        const unsigned o = (unsigned)(min(k0 + i * 16 + n, last) & mask) * HD + g * 8;
#pragma unroll
        for (int t = 0; t < TT; ++t) kr[i][t] = af_load_once(reinterpret_cast<const half8*>(Kc + o + t * 32));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned ov = (unsigned)(min(k0 + i * 16 + g * 4 + j, last) & mask) * HD + n * VC;
          vr[i * 4 + j] = af_load_once(reinterpret_cast<const vrow*>(Vc + ov));
        }
      }
    };

    float m = -INFINITY, l = 0.f;
    spl_f4 acc[VC];
    const spl_f4 zero4 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < VC; ++c) acc[c] = zero4;
    int t = t0 * SPL_WAVES + wave, k0 = paged_tile_start<SPL_STEP>(tl, t);
    ids(t);
    if (t < end) fetch(k0);
    ids(t + SPL_WAVES);
    for (; t < end; t += SPL_WAVES) {
      // scores of keys k0 + 16 i + 4 g + e, row n
      float sc[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        spl_f4 d = zero4;
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kr[i][tt], q[tt], d, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[i * 4 + e] = d[e] * p.a.scale2;
      }
      const bool inside = k0 + SPL_STEP - 1 <= p0 && (window <= 0 || k0 > p1 - window || k0 + SPL_STEP <= n_sink);
      if (!inside || bad[0] || bad[1]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)  // (a step may hold keys that no row sees, with or without a page)
          if (bad[i] && paged_span_seen(k0 + i * 16, p0, p1, window, n_sink)) paged_report(v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (bad[j >> 2] || !paged_seen(k0 + (j >> 2) * 16 + g * 4 + (j & 3), place, window, n_sink)) sc[j] = -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) mx = fmaxf(mx, sc[j]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, AF_WAVE));
      mx = fmaxf(mx, __shfl_xor(mx, 32, AF_WAVE));
      mx = fmaxf(mx, m);
      const float safe = mx == -INFINITY ? 0.f : mx;
      if (__any(m != mx)) {
        const float corr = __builtin_amdgcn_exp2f(m - safe);
        l *= corr;
#pragma unroll
        for (int c = 0; c < VC; ++c) acc[c] *= corr;
      }
      m = mx;
      // weights times 2^15 (in the range of fp16) as a rounded value and a rest: 22 bits
      u32x4 ph, pl;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e0 = __builtin_amdgcn_exp2f(sc[2 * i] - safe) * 32768.f, e1 = __builtin_amdgcn_exp2f(sc[2 * i + 1] - safe) * 32768.f;
        l += e0 + e1;
        const spl_h2 hi = {(half_t)e0, (half_t)e1};
        const spl_h2 lo = {(half_t)(e0 - (float)hi[0]), (half_t)(e1 - (float)hi[1])};
        ph[i] = __builtin_bit_cast(unsigned, hi);
        pl[i] = __builtin_bit_cast(unsigned, lo);
      }
      vwords vw[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) vw[j] = __builtin_bit_cast(vwords, vr[j]);
#pragma unroll
      for (int c = 0; c < VC; ++c) {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[i] = __builtin_amdgcn_perm(vw[2 * i + 1][c / 2], vw[2 * i][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
        const half8 a8 = __builtin_bit_cast(half8, a);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a8, __builtin_bit_cast(half8, pl), acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a8, __builtin_bit_cast(half8, ph), acc[c], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);  // with the products and the next rows' addresses mixed, registers spill
      if (t + SPL_WAVES < end) {
        k0 = paged_tile_start<SPL_STEP>(tl, t + SPL_WAVES);
        fetch(k0);
        ids(t + 2 * SPL_WAVES);
      }
    }
    l += __shfl_xor(l, 16, AF_WAVE);
    l += __shfl_xor(l, 32, AF_WAVE);

    // the waves' sums
    if (n < rows) {
      float* to = (wave == 0 ? acc_lds[0] : wave == 1 ? acc_lds[1] : wave == 2 ? acc_lds[2] : acc_lds[3]) + n * (HD + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c) to[(g * 4 + e) * VC + c] = acc[c][e];
      if (g == 0) s_ml[wave][n] = make_float2(m, l);
    }
    __syncthreads();
    const u64 start = u - (u64)t0;
    const bool whole = t1 - t0 == units;
    // A result that is not a number (an infinity among what was read, seen or not; nothing seen) is formed again key by key.
    auto store = [&](int rr, float v0, float v1, float L) __attribute__((always_inline)) {
      const int ra = r0 + rr, ta = ra / rep, ha = kvh * rep + (ra - ta * rep), d = lane * 2;
      const float o0 = v0 / L, o1 = v1 / L;
      if (__any(d < HD && (o0 != o0 || o1 != o1)))
        paged_row<HD>(p.a, b, seq.row0 + ta, p0 + ta, ha);
      else if (d < HD)
        *reinterpret_cast<half2v*>(p.a.out + (size_t)(seq.row0 + ta) * p.a.out_stride + (size_t)ha * HD + d) = half2v{(half_t)o0, (half_t)o1};
    };
    // partial result of this group's piece in workgroup w: [rows][maximum, sum, values]
    auto slot = [&](int w) __attribute__((always_inline)) {
      return p.part + (size_t)(2 * w + (start > (u64)w * share ? 1 : 0)) * p.slot_rows * (HD + 2);
    };
    const int d = min(lane * 2, HD - 2);
    float M[SPL_RW], L[SPL_RW], v0[SPL_RW], v1[SPL_RW];  // of rows wave, wave + 4, ...
    auto put = [&](float* to) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < SPL_RW; ++i)
        if (wave + i * SPL_WAVES < rows) {
          float* at = to + (wave + i * SPL_WAVES) * (HD + 2);
          if (lane * 2 < HD) af_store_agent2(at + 2 + d, v0[i], v1[i]);
          if (lane == 0) af_store_agent2(at, M[i], L[i]);
        }
    };
    // The sum of `cnt` partial results, at from(i): lane i has the maximum and the sum of the i-th.  They come from other XCDs, so
    // two rows' are requested together, in fours: sixteen whatever their number, the last one again, cost four pieces of a row 0.7 us
    // and five of eight rows 0.5 (sixteen pieces of sixteen rows gain 0.3 by it), twos and eights 0.1 to 0.3.
    auto join = [&](int cnt, auto&& from) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < SPL_RW; i += 2) {
        if (wave + i * SPL_WAVES >= rows) continue;
        const bool two = wave + (i + 1) * SPL_WAVES < rows;
        const int ra = (wave + i * SPL_WAVES) * (HD + 2), rb = ra + SPL_WAVES * (HD + 2);
        const float* mine = from(min(lane, cnt - 1));
        af_float2 ml[2] = {af_load_agent2(mine + ra), af_float2{0.f, 0.f}};
        if (two) ml[1] = af_load_agent2(mine + rb);
        float f[2];
        for (int c0 = 0; c0 < cnt; c0 += SPL_JOIN) {
          af_float2 av[2][SPL_JOIN];
#pragma unroll
          for (int e0 = 0; e0 < SPL_JOIN; e0 += 4) {
            if (c0 + e0 >= cnt) break;
#pragma unroll
            for (int e = e0; e < e0 + 4; ++e) {
              const float* at = from(min(c0 + e, cnt - 1)) + 2 + d;
              av[0][e] = af_load_agent2(at + ra);
              if (two) av[1][e] = af_load_agent2(at + rb);
            }
          }
          if (c0 == 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              if (k && !two) continue;
              float mx = lane < cnt ? ml[k][0] : -INFINITY;
              mx = af_wave_max(mx);
              f[k] = lane < cnt ? __builtin_amdgcn_exp2f(ml[k][0] - (mx == -INFINITY ? 0.f : mx)) : 0.f;
              M[i + k] = mx;
              L[i + k] = af_wave_sum(lane < cnt ? f[k] * ml[k][1] : 0.f);
              v0[i + k] = v1[i + k] = 0.f;
            }
          }
#pragma unroll
          for (int e = 0; e < SPL_JOIN; ++e)
            if (c0 + e < cnt) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                if (k && !two) continue;
                const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f[k]), c0 + e));
                v0[i + k] += w * av[k][e][0];
                v1[i + k] += w * av[k][e][1];
              }
            }
        }
      }
    };
    // last of `cnt` workgroups at ticket t
    auto last_of = [&](int cnt, int t) __attribute__((always_inline)) {
      af_stores_done();
      __syncthreads();
      if (tid == 0) {
        s_last = af_ticket_take(&p.tickets[af_ticket_of(t)]) == cnt - 1;
        if (s_last) af_ticket_reset(&p.tickets[af_ticket_of(t)]);
      }
      __syncthreads();
      return s_last != 0;
    };
#pragma unroll
    for (int i = 0; i < SPL_RW; ++i) {
      const int rr = wave + i * SPL_WAVES;
      if (rr >= rows) break;
      M[i] = -INFINITY;
      L[i] = v0[i] = v1[i] = 0.f;
#pragma unroll
      for (int w = 0; w < SPL_WAVES; ++w) M[i] = fmaxf(M[i], s_ml[w][rr].x);
      const float safe = M[i] == -INFINITY ? 0.f : M[i];
#pragma unroll
      for (int w = 0; w < SPL_WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(s_ml[w][rr].x - safe);
        L[i] += f * s_ml[w][rr].y;
        v0[i] += f * acc_lds[w][rr * (HD + 4) + d];
        v1[i] += f * acc_lds[w][rr * (HD + 4) + d + 1];
      }
    }
    bool done = whole;
    if (!whole) {
      // Workgroups w0 .. w1 have the group's pieces.  Sixteen neighbours join theirs, and where there are more of them, the
      // sixteens' sums are joined after that: a single workgroup would go through 64 pieces of eight rows for 17 us.
      const int w0 = (int)(start / share), w1 = (int)((start + (u64)units - 1) / share);
      const int first = w0 + (wg - w0) / SPL_JOIN * SPL_JOIN, cnt = min(SPL_JOIN, w1 - first + 1);
      const int sets = (w1 - w0) / SPL_JOIN + 1;
      done = true;
      put(slot(wg));
      if (cnt > 1) {  // alone, it may be the first of another group: the ticket is that one's
        done = last_of(cnt, first);
        if (done) {
          join(cnt, [&](int i) __attribute__((always_inline)) { return slot(first + i); });
          if (sets > 1) put(slot(first));
        }
      }
      if (done && sets > 1) {
        done = last_of(sets, SPL_MAX_WGS + w0);
        if (done) join(sets, [&](int i) __attribute__((always_inline)) { return slot(w0 + i * SPL_JOIN); });
      }
    }
    if (done) {
#pragma unroll
      for (int i = 0; i < SPL_RW; ++i)
        if (wave + i * SPL_WAVES < rows) store(wave + i * SPL_WAVES, v0[i], v1[i], L[i]);
    }
    u = apart ? u1 : u + (u64)(t1 - t0);
    if (u < u1) __syncthreads();  // the sums in LDS are read; the next stretch writes them
  }
}

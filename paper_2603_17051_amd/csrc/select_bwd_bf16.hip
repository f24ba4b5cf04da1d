// Backward of the attention over selected blocks with the cache detached, bf16 MFMA with fp32 accumulation:
//   P_ij = exp(<Q~_i, K~_j> / sqrt(D) - lse_i),  dS_ij = P_ij (<dO_i, V_j> - <dO_i, O_i>),  j in S_i (see the forward)
//   dQ~_i = sum over j in S_i of dS_ij K~_j / sqrt(D)       dK~_j = sum over i that see j of dS_ij Q~_i / sqrt(D)
//   dV_j  = sum over i that see j of P_ij dO_i              (j a chunk row; dQ~ and dK~ are turned back)
// Gradients go out in fp32 and carry 16 bits: every operand that is not bf16 by itself (rotated queries and chunk keys, P, dS)
// enters its products as two bf16 halves, the halves' small products left out (2^-17).  With one rounded half each the
// gradients were 3.8e-3 off, now 6.7e-6 at the keys as they are cached; the price is 5 products instead of 3 per cached key, and 7 + 9
// instead of 3 + 4 per chunk key: two clips of 4680 rows, 24 pairs of 128, 2816 cached keys 2080 to 2160 us instead of 1139.  Bound by the
// products, 1.2 PFLOP/s.  Calls of few rows take three pieces in the scores (select_rules.hpp) and all four products of halves of dS with Q~ and K~.
// Two launches, no atomics: the query side walks a group's tiles as the forward does and leaves the rows' terms (lse, <dO, O>),
// the key side walks the queries for 64 chunk keys; every chunk row is a key of all queries that see it, whatever those selected.
#include "select_rules.hpp"
#include "select_walk.hpp"

namespace astro {
namespace {

constexpr int kWaves = 4;

struct SelectBwdParams {
  SelectStaged staged;
  const __bf16 *v_chunk, *k_cache, *v_cache, *out, *dout;
  const float* lse;
  float *neg_delta, *neg_lse2;  // [B][H][Nq]: -<dO, O>, -lse * log2(e)
  float *dq, *dk, *dv;          // [B, Nq, H, D]
  // key ranges of the query side: range `split` leaves its sums in its part, which a merge launch adds up and turns back
  int splits;
  float* dq_part;  // [splits][B, Nq, H, D]
  RotaryTables rot;
  int H, Nq, BH, tiles, group, block_rows;
  bool by_xcd;
  int64_t cache_rows;
  float scale;
  StreamInts hist_rows;
};

// ---- query side: 16 * QS queries of a wave, lane (i = lane % 16, g = lane / 16) owns queries 16 * qs + i ----------------
template <int D, int QS, bool kFine>
struct SelectDqWave {
  static constexpr int KS = D / 32, DT = D / 16;
  bf16x8 qh[QS][KS], ql[QS][KS], qr[kFine ? QS : 1][KS], doreg[QS][KS];
  f32x4 neg_lse2[QS], neg_delta[QS];  // four copies: the accumulators of S and dP start from them
  f32x4 dq[DT][QS];
  OperandAddr16<D> addr;
  int g;

  __device__ __forceinline__ void load(const SelectBwdParams& p, int b, int h, int q_wave, int lane, bool leave_terms) {
    g = lane >> 4;
    addr.init(lane);
    const int64_t bh = (int64_t)b * p.H + h;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      const int q = q_wave + 16 * qs + (lane & 15), row = q < p.Nq ? q : p.Nq - 1;
      const int64_t at = (bh * p.Nq + row) * D + g * 8, token = (((int64_t)b * p.Nq + row) * p.H + h) * D + g * 8;
      float d = 0.f;
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        qh[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_hi + at + st * 32);
        ql[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_lo + at + st * 32);
        if constexpr (kFine) qr[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_rest + at + st * 32);
        doreg[qs][st] = *reinterpret_cast<const bf16x8*>(p.dout + token + st * 32);
        const bf16x8 o = *reinterpret_cast<const bf16x8*>(p.out + token + st * 32);
#pragma unroll
        for (int j = 0; j < 8; ++j) d = fmaf((float)doreg[qs][st][j], (float)o[j], d);
      }
      d = sum_quarters(d);
      const float l = -p.lse[bh * p.Nq + row] * kLog2e;
      neg_lse2[qs] = f32x4{l, l, l, l};
      neg_delta[qs] = f32x4{-d, -d, -d, -d};
      if (leave_terms && q < p.Nq && g == 0) {
        p.neg_delta[bh * p.Nq + q] = -d;
        p.neg_lse2[bh * p.Nq + q] = l;
      }
    }
    clear();
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dq[dt][qs] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ bool not_numbers_yet() const {
    bool x = false;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) x = x || not_numbers(dq[dt][qs]);
    return x;
  }

  template <bool kChunk, bool kCare>  // as in the forward
  __device__ __forceinline__ void tile(const char* stage, const int (&live)[QS], int fewest, bool ring) {
    const char *ks = stage, *vs = stage + kSelectTile * D * 2, *lo = vs + kSelectTile * D * 2;
    f32x4 s[2][QS], dp[2][QS], start[2][QS];
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) start[kh][qs] = neg_lse2[qs];
    if constexpr (kFine)
      scores_from_thirds<D, QS, kCare>(ks, lo, lo + kSelectTile * D * 2, !ring, addr, qh, ql, qr, start, s);
    else if constexpr (kCare)
      scores_of_any<D, QS>(ks, lo, !ring, addr, qh, ql, start, s);
    else
      scores_from_halves<D, QS, kChunk>(ks, lo, addr, qh, ql, start, s);
    // keys that do not count get a score that makes P and dS exactly 0
    if (kCare || fewest < kSelectTile) {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int qs = 0; qs < QS; ++qs)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[kh][qs][r] = 16 * kh + 4 * g + r >= live[qs] ? kNegBig : s[kh][qs][r];
    }
    // dP - <dO, O>, with the exponentials of the scores between its products
    bf16x8 v[KS][2];
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int kh = 0; kh < 2; ++kh) v[st][kh] = read_rows16<D>(vs, addr.row[st], 16 * kh);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) dp[kh][qs] = mfma16(v[st][kh], doreg[qs][st], st == 0 ? neg_delta[qs] : dp[kh][qs]);
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int qs = 0; qs < QS; ++qs)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[kh][qs][r] = fast_exp2(s[kh][qs][r]);
          if constexpr (kCare) dp[kh][qs][r] = 16 * kh + 4 * g + r >= live[qs] ? 0.f : dp[kh][qs][r];
        }
    bf16x8 a[2][4], c[2][4];  // of dQ~'s columns, four at a time, so that products on one accumulator lie apart
    if constexpr (!kCare) read_quad<D>(ks, addr, 0, a[0]);
    if constexpr (kChunk && !kCare) read_quad<D>(lo, addr, 0, c[0]);
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 hi[QS], small[QS];
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int r = 0; r < 4; r += 2) {
          const f32x2 ds = {s[kh][qs][r] * dp[kh][qs][r], s[kh][qs][r + 1] * dp[kh][qs][r + 1]};
          const HalfPairs x = kCare ? halves_of_any(ds) : halves(ds);
          hi[qs][4 * kh + r] = x.hi[0], hi[qs][4 * kh + r + 1] = x.hi[1];
          small[qs][4 * kh + r] = x.lo[0], small[qs][4 * kh + r + 1] = x.lo[1];
        }
    if constexpr (kCare) {
#pragma unroll
      for (int qs = 0; qs < QS; ++qs)
        each_bound(live[qs], [&](int bound, bool mine) __attribute__((always_inline)) {
          const u32x4 mask = rows_between(g, 0, bound), low_mask = rows_between(g, 0, ring ? 0 : bound);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bf16x8 x = only(mask, read_cols16<D>(ks, addr.tr[dt], 0));
            const f32x4 big = mfma16(x, hi[qs], dq[dt][qs]);
            f32x4 to = mfma16(x, small[qs], big);
            const bf16x8 y = only(low_mask, read_cols16<D>(lo, addr.tr[dt], 0));
            to = mfma16(y, hi[qs], to);
            if constexpr (kFine) to = mfma16(y, small[qs], to);
            dq[dt][qs] = either(mine, with_small(big, to), dq[dt][qs]);
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      return;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int quad = 0; quad < DT / 4; ++quad) {
      if (quad + 1 < DT / 4) {
        read_quad<D>(ks, addr, quad + 1, a[(quad + 1) & 1]);
        if constexpr (kChunk) read_quad<D>(lo, addr, quad + 1, c[(quad + 1) & 1]);
      }
      auto product = [&](const bf16x8 (&x)[4], const bf16x8 (&y)[QS]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int qs = 0; qs < QS; ++qs) dq[4 * quad + i][qs] = mfma16(x[i], y[qs], dq[4 * quad + i][qs]);
      };
      product(a[quad & 1], hi);
      product(a[quad & 1], small);
      if constexpr (kChunk) product(c[quad & 1], hi);
      if constexpr (kChunk && kFine) product(c[quad & 1], small);
    }
  }
};

template <int D, int QS, int kStages, int OCC, bool kFine>
__global__ void __launch_bounds__(kWaves * 64, OCC) select_bwd_dq_kernel(SelectBwdParams p, SelectLists lists) {
  using Wave = SelectDqWave<D, QS, kFine>;
  using Walk = SelectWalk<D, kWaves, kFine>;
  using Stages = SelectStages<D, kWaves, kStages, kFine>;
  constexpr int kAhead = kStages - 1, kQueries = kWaves * 16 * QS;
  __shared__ __attribute__((aligned(1024))) char lds[Stages::kBytes];
  __shared__ TileList tile_list;

  const WorkItem item = work_item(p.tiles, p.BH * p.splits, p.by_xcd);
  if (!item.valid) return;
  const int split = item.bh % p.splits;
  const PairIndex pair = split_pair(item.bh / p.splits, p.H, p.group);
  const int b = pair.b, h = pair.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t bh = (int64_t)b * p.H + h;
  const int q_wg = item.tile * kQueries, q_wave = q_wg + wave * 16 * QS, q_last = p.Nq - 1;
  if (wave == 0)
    fill_tile_list(lists, lists.blocks + (bh * lists.groups + q_wg / lists.query_block) * lists.n_select, p.hist_rows.v[pair.cache_b] / lists.T,
                   &tile_list);
  const int vis_wave = visible_chunk_rows(q_wave < q_last ? q_wave : q_last, p.Nq, p.block_rows);
  const int vis_last = visible_chunk_rows(q_wg + kQueries - 1 < q_last ? q_wg + kQueries - 1 : q_last, p.Nq, p.block_rows);
  Wave w;
  w.load(p, b, h, q_wave, lane, split == 0);
  wait_vmem();  // (see the forward)
  __syncthreads();
  Walk walk;
  walk.init(&tile_list, vis_last);
  walk.k_ring = segment_words(p.k_cache + (int64_t)pair.cache_bh * p.cache_rows * D, D, 1, D);
  walk.v_ring = segment_words(p.v_cache + (int64_t)pair.cache_bh * p.cache_rows * D, D, 1, D);
  walk.k_hi = segment_words((const __bf16*)p.staged.k_hi + bh * p.Nq * D, D, p.Nq, D);
  walk.k_lo = segment_words((const __bf16*)p.staged.k_lo + bh * p.Nq * D, D, p.Nq, D);
  if constexpr (kFine) walk.k_rest = segment_words((const __bf16*)p.staged.k_rest + bh * p.Nq * D, D, p.Nq, D);
  walk.v_chunk = segment_words(p.v_chunk + ((int64_t)b * p.Nq * p.H + h) * D, (int64_t)p.H * D, p.Nq, D);
  walk.v_chunk_stride = p.H * D * 2;
  const int t_begin = (int)((int64_t)split * walk.tiles / p.splits), t_end = (int)((int64_t)(split + 1) * walk.tiles / p.splits);

  // (invariant at the top of tile t as in the forward)
  auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < kAhead; ++t)
      if (t_begin + t < t_end) walk.issue(t_begin + t, walk.entry(t_begin + t), Stages::of(lds, t));
    if (kAhead > 1)
      walk.wait_all_but(t_begin + kAhead - 1, t_end);
    else
      wait_vmem();
    __syncthreads();
  };
  begin();
  auto step = [&](int t, auto chunk_c, auto care_c) __attribute__((always_inline)) {
    constexpr bool kChunk = decltype(chunk_c)::value, kCare = decltype(care_c)::value;
    const char* stage = Stages::of(lds, t - t_begin);
    if (t + kAhead < t_end) walk.issue(t + kAhead, walk.entry(t + kAhead), Stages::of(lds, t - t_begin + kAhead));
    const bool ring = kCare ? t < walk.ring_tiles : !kChunk;
    const int row0 = (t - walk.ring_tiles) * kSelectTile, fewest = ring ? walk.rows_of(t) : vis_wave - row0;
    int live[QS];
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      live[qs] = fewest;
      if (!ring && (kCare || (p.block_rows != 0 && fewest < kSelectTile))) {
        const int q = q_wave + 16 * qs + (lane & 15);
        live[qs] = min(max(visible_chunk_rows(q < q_last ? q : q_last, p.Nq, p.block_rows) - row0, 0), kSelectTile);
      }
    }
    w.template tile<kChunk, kCare>(stage, live, fewest, ring);
    if (kAhead > 1)
      walk.wait_all_but(t + kAhead, t_end);
    else
      wait_vmem();
    __syncthreads();
  };
  {
    int t = t_begin;
    for (; t < t_end && t < walk.ring_tiles; ++t) step(t, std::false_type{}, std::false_type{});
    for (; t < t_end; ++t) step(t, std::true_type{}, std::false_type{});
  }
  if (walk.again(&tile_list, w.not_numbers_yet())) {
    w.clear();
    begin();
    for (int t = t_begin; t < t_end; ++t) step(t, std::true_type{}, std::true_type{});
  }

  const bool rope = p.rot.n_t + p.rot.n_h + p.rot.n_w != 0;
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int q = q_wave + 16 * qs + (lane & 15);
    if (q >= p.Nq) continue;
    const int64_t at = (((int64_t)b * p.Nq + q) * p.H + h) * D + 4 * w.g;
    if (p.splits > 1) {
      float* part = p.dq_part + (int64_t)split * p.BH * p.Nq * D + at;
#pragma unroll
      for (int dt = 0; dt < Wave::DT; ++dt) *reinterpret_cast<f32x4*>(part + 16 * dt) = w.dq[dt][qs];
      continue;
    }
    float* row = p.dq + at;
    TokenTables tt{};
    if (rope) tt = token_tables(p.rot, b, q);
#pragma unroll
    for (int dt = 0; dt < Wave::DT; ++dt) {
      f32x4 x = w.dq[dt][qs] * p.scale;
      if (rope) x = unrotate_quad(p.rot, tt, 4 * dt + w.g, x);
      *reinterpret_cast<f32x4*>(row + 16 * dt) = x;
    }
  }
}

// dQ = R(phi)^T (the ranges' sums) / sqrt(D): bytes only
template <int D>
__global__ void __launch_bounds__(256) select_dq_merge_kernel(SelectBwdParams p, uint32_t n_rows) {
  constexpr uint32_t CPR = D / 4;
  const uint32_t row = blockIdx.x * (256 / CPR) + threadIdx.x / CPR;  // (b * Nq + q) * H + h
  if (row >= n_rows) return;
  const uint32_t c = threadIdx.x % CPR, bq = row / (uint32_t)p.H, b = bq / (uint32_t)p.Nq;
  f32x4 x[kMaxSelectSplits], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (uint32_t s = 0; s < kMaxSelectSplits; ++s) {  // (the first part again for those that are not there: no branch between loads)
    const uint32_t from = s < (uint32_t)p.splits ? s : 0;
    x[s] = *reinterpret_cast<const f32x4*>((const char*)p.dq_part + ((from * n_rows + row) * CPR + c) * 16u);
  }
#pragma unroll
  for (int s = 0; s < kMaxSelectSplits; ++s) sum += s < p.splits ? x[s] : f32x4{0.f, 0.f, 0.f, 0.f};
  sum *= p.scale;
  if (p.rot.n_t + p.rot.n_h + p.rot.n_w != 0) sum = unrotate_quad(p.rot, token_tables(p.rot, b, bq - b * p.Nq), c, sum);
  *reinterpret_cast<f32x4*>(p.dq + (int64_t)row * D + c * 4) = sum;
}

// ---- key side: 16 chunk keys of a wave, lane (i, g) owns key i; tiles of 32 queries -----------------------------------------
template <int D, int OCC, bool kFine>
__global__ void __launch_bounds__(kWaves * 64, OCC) select_bwd_dkv_kernel(SelectBwdParams p) {
  constexpr int KS = D / 32, DT = D / 16, kStages = 2, kAhead = kStages - 1, kKeys = kWaves * 16;
  using Stream = SharedStream<D, kWaves>;
  using Stages = SelectStages<D, kWaves, kStages, kFine>;
  constexpr int kTileBytes = Stages::kTileBytes;
  __shared__ __attribute__((aligned(1024))) char lds[Stages::kBytes];
  __shared__ __attribute__((aligned(1024))) float terms[kStages][2][kSelectTile];  // -lse * log2(e), -<dO, O>
  __shared__ int again;

  const WorkItem item = work_item(p.tiles, p.BH, p.by_xcd);
  if (!item.valid) return;
  const int b = item.bh / p.H, h = item.bh - b * p.H;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int64_t bh = (int64_t)b * p.H + h;
  const int j_wg = item.tile * kKeys, j = j_wg + wave * 16 + i16, j_last = p.Nq - 1;
  OperandAddr16<D> addr;
  addr.init(lane);
  bf16x8 kh[1][KS], kl[1][KS], kr[1][KS], v[KS];
  {
    const int row = j < p.Nq ? j : j_last;
    const int64_t at = (bh * p.Nq + row) * D + g * 8, token = (((int64_t)b * p.Nq + row) * p.H + h) * D + g * 8;
#pragma unroll
    for (int st = 0; st < KS; ++st) {
      kh[0][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.k_hi + at + st * 32);
      kl[0][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.k_lo + at + st * 32);
      if constexpr (kFine) kr[0][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.k_rest + at + st * 32);
      v[st] = *reinterpret_cast<const bf16x8*>(p.v_chunk + token + st * 32);
    }
  }
  f32x4 dk[DT], dv[DT];
  // queries from the first that sees any key of the workgroup; `first`: that sees this lane's key, last_first: all of the wave's
  const int j_wave = j_wg + wave * 16;
  const int first = first_query_row_seeing(j < p.Nq ? j : j_last, p.block_rows);
  const int last_first = first_query_row_seeing(j_wave + 15 < p.Nq ? j_wave + 15 : j_last, p.block_rows);
  const int t_begin = __builtin_amdgcn_readfirstlane(first_query_row_seeing(j_wg, p.block_rows) / kSelectTile), t_end = (p.Nq + kSelectTile - 1) / kSelectTile;

  Stream stream;
  stream.init();
  const u32x4 q_hi = segment_words((const __bf16*)p.staged.q_hi + bh * p.Nq * D, D, p.Nq, D);
  const u32x4 q_lo = segment_words((const __bf16*)p.staged.q_lo + bh * p.Nq * D, D, p.Nq, D);
  const u32x4 q_rest = kFine ? segment_words((const __bf16*)p.staged.q_rest + bh * p.Nq * D, D, p.Nq, D) : u32x4{};
  const u32x4 dout = segment_words(p.dout + ((int64_t)b * p.Nq * p.H + h) * D, (int64_t)p.H * D, p.Nq, D);
  // a row behind the last query has zeros for Q~ and dO, and a term that makes its P exactly 0 (exp2 of any lse may be infinite)
  const float* const term_rows = (wave & 1 ? p.neg_delta : p.neg_lse2) + bh * p.Nq;
  auto issue = [&](int t) __attribute__((always_inline)) {
    char* stage = Stages::of(lds, t - t_begin);
    stream.issue(q_hi, D * 2, t * kSelectTile, stage);
    stream.issue(dout, p.H * D * 2, t * kSelectTile, stage + kTileBytes);
    stream.issue(q_lo, D * 2, t * kSelectTile, stage + 2 * kTileBytes);
    if constexpr (kFine) stream.issue(q_rest, D * 2, t * kSelectTile, stage + 3 * kTileBytes);
  };
  float term = 0.f;  // of the tile ahead: waves 0 and 1 bring them
  auto take_term = [&](int t) __attribute__((always_inline)) {
    const int q = t * kSelectTile + (lane & 31);
    if (wave < 2 && t < t_end) term = q < p.Nq ? term_rows[q] : kNegBig;
  };
  auto leave_term = [&](int t) __attribute__((always_inline)) {
    if (wave < 2 && lane < kSelectTile && t < t_end) terms[(t - t_begin) % kStages][wave][lane] = term;
  };
  auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      if (t_begin + t < t_end) issue(t_begin + t);
      take_term(t_begin + t);
      leave_term(t_begin + t);
    }
    wait_vmem();
    __syncthreads();
  };
  auto step = [&](int t, auto care_c) __attribute__((always_inline)) {
    constexpr bool kCare = decltype(care_c)::value;
    const char *qs = Stages::of(lds, t - t_begin), *dos = qs + kTileBytes, *lo = qs + 2 * kTileBytes;
    if (t + kAhead < t_end) issue(t + kAhead);
    take_term(t + kAhead);
    const float(*row_terms)[kSelectTile] = terms[(t - t_begin) % kStages];
    f32x4 s[2][1], dp[2], start[2][1];
#pragma unroll
    for (int qh = 0; qh < 2; ++qh) {
      start[qh][0] = *reinterpret_cast<const f32x4*>(&row_terms[0][16 * qh + 4 * g]);
      dp[qh] = *reinterpret_cast<const f32x4*>(&row_terms[1][16 * qh + 4 * g]);
    }
    // of the tile's queries: this lane's key is a key of [from, to)
    const int from = min(max(first - t * kSelectTile, 0), kSelectTile), to = min(p.Nq - t * kSelectTile, kSelectTile);
    if constexpr (kFine)
      scores_from_thirds<D, 1, kCare>(qs, lo, lo + kTileBytes, true, addr, kh, kl, kr, start, s);
    else if constexpr (kCare)
      scores_of_any<D, 1>(qs, lo, true, addr, kh, kl, start, s);
    else
      scores_from_halves<D, 1, true>(qs, lo, addr, kh, kl, start, s);
    if (kCare || t * kSelectTile < last_first) {
#pragma unroll
      for (int qh = 0; qh < 2; ++qh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * qh + 4 * g + r;
          s[qh][0][r] = row < from || (kCare && row >= to) ? kNegBig : s[qh][0][r];
        }
    }
    bf16x8 dor[KS][2];
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int qh = 0; qh < 2; ++qh) dor[st][qh] = read_rows16<D>(dos, addr.row[st], 16 * qh);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int qh = 0; qh < 2; ++qh) dp[qh] = mfma16(dor[st][qh], v[st], dp[qh]);
#pragma unroll
    for (int qh = 0; qh < 2; ++qh)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[qh][0][r] = fast_exp2(s[qh][0][r]);
    if constexpr (kCare) {
#pragma unroll
      for (int qh = 0; qh < 2; ++qh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 16 * qh + 4 * g + r;
          dp[qh][r] = row < from || row >= to ? 0.f : dp[qh][r];
        }
    }
    bf16x8 a[2][4], c[2][4];  // of the gradients' columns, four at a time, so that products on one accumulator lie apart
    if constexpr (!kCare) read_quad<D>(dos, addr, 0, a[0]);
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 p_hi, p_lo, ds_hi, ds_lo;
#pragma unroll
    for (int qh = 0; qh < 2; ++qh)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const f32x2 pr = {s[qh][0][r], s[qh][0][r + 1]};
        const f32x2 ds = {pr[0] * dp[qh][r], pr[1] * dp[qh][r + 1]};
        const HalfPairs x = kCare ? halves_of_any(pr) : halves(pr), y = kCare ? halves_of_any(ds) : halves(ds);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          p_hi[4 * qh + r + i] = x.hi[i], p_lo[4 * qh + r + i] = x.lo[i];
          ds_hi[4 * qh + r + i] = y.hi[i], ds_lo[4 * qh + r + i] = y.lo[i];
        }
      }
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kQuads = DT / 4;
    if constexpr (kCare) {
      each_bound(from, [&](int bound, bool mine) __attribute__((always_inline)) {
        const u32x4 mask = rows_between(g, bound, to);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bf16x8 x = only(mask, read_cols16<D>(dos, addr.tr[dt], 0)), y = only(mask, read_cols16<D>(qs, addr.tr[dt], 0));
          const f32x4 big_v = mfma16(x, p_hi, dv[dt]), big_k = mfma16(y, ds_hi, dk[dt]);
          dv[dt] = either(mine, with_small(big_v, mfma16(x, p_lo, big_v)), dv[dt]);
          const bf16x8 z = only(mask, read_cols16<D>(lo, addr.tr[dt], 0));
          f32x4 all_k = mfma16(z, ds_hi, mfma16(y, ds_lo, big_k));
          if constexpr (kFine) all_k = mfma16(z, ds_lo, all_k);
          dk[dt] = either(mine, with_small(big_k, all_k), dk[dt]);
          __builtin_amdgcn_sched_barrier(0);
        }
      });
    } else {
#pragma unroll
      for (int quad = 0; quad < kQuads; ++quad) {
        if (quad + 1 < kQuads) {
          read_quad<D>(dos, addr, quad + 1, a[(quad + 1) & 1]);
        } else {
          read_quad<D>(qs, addr, 0, a[kQuads & 1]);
          read_quad<D>(lo, addr, 0, c[0]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dv[4 * quad + i] = mfma16(a[quad & 1][i], p_hi, dv[4 * quad + i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) dv[4 * quad + i] = mfma16(a[quad & 1][i], p_lo, dv[4 * quad + i]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int quad = 0; quad < kQuads; ++quad) {
        if (quad + 1 < kQuads) {
          read_quad<D>(qs, addr, quad + 1, a[(quad + 1 + kQuads) & 1]);
          read_quad<D>(lo, addr, quad + 1, c[(quad + 1) & 1]);
        }
        const auto& x = a[(quad + kQuads) & 1];
#pragma unroll
        for (int i = 0; i < 4; ++i) dk[4 * quad + i] = mfma16(x[i], ds_hi, dk[4 * quad + i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) dk[4 * quad + i] = mfma16(x[i], ds_lo, dk[4 * quad + i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) dk[4 * quad + i] = mfma16(c[quad & 1][i], ds_hi, dk[4 * quad + i]);
        if constexpr (kFine)
#pragma unroll
          for (int i = 0; i < 4; ++i) dk[4 * quad + i] = mfma16(c[quad & 1][i], ds_lo, dk[4 * quad + i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    leave_term(t + kAhead);
    wait_vmem();
    __syncthreads();
  };
  again = 0;
  begin();
  for (int t = t_begin; t < t_end; ++t) {
    asm volatile("" : "+s"(t));  // (beside the second walk's the compiler counts this loop in vector registers: 3 % of the launch)
    step(t, std::false_type{});
  }
  {  // (see each_bound)
    bool not_numbers_yet = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) not_numbers_yet = not_numbers_yet || not_numbers(dk[dt]) || not_numbers(dv[dt]);
    if (__any(not_numbers_yet)) again = 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(again)) {
      begin();
      for (int t = t_begin; t < t_end; ++t) step(t, std::true_type{});
    }
  }
  if (j >= p.Nq) return;
  const bool rope = p.rot.n_t + p.rot.n_h + p.rot.n_w != 0;
  const int64_t row = (((int64_t)b * p.Nq + j) * p.H + h) * D + 4 * g;
  TokenTables tt{};
  if (rope) tt = token_tables(p.rot, b, j);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    f32x4 x = dk[dt] * kLn2;  // the staged queries carry log2(e) / sqrt(D)
    if (rope) x = unrotate_quad(p.rot, tt, 4 * dt + g, x);
    *reinterpret_cast<f32x4*>(p.dk + row + 16 * dt) = x;
    *reinterpret_cast<f32x4*>(p.dv + row + 16 * dt) = dv[dt];
  }
}

template <int D, int QS, int kStages, int OCC, bool kFine>
void launch_dq(const DevGeom& g, const AttnOperands& op, const SelectLists& lists, SelectBwdParams p, hipStream_t stream) {
  p.tiles = blocks_of(op.Nq, kWaves * 16 * QS);
  const CallShape shape = select_call_shape(g, op, lists);
  if (p.dq_part)
    p.splits = select_splits(select_dq_cost(D), g.n_cus, p.tiles * p.BH, mean_keys(shape) / kSelectTile,
                             (double)p.BH * op.Nq * D * sizeof(float));
  const int items = work_grid_size(p.tiles, p.BH * p.splits);
  p.by_xcd = order_by_xcd(shape, items);
  {
    ProfileScope prof("select_attn_bwd_dq_bf16", stream);
    select_bwd_dq_kernel<D, QS, kStages, OCC, kFine><<<dim3(items), kWaves * 64, 0, stream>>>(p, lists);
  }
  if (p.splits > 1) {
    const uint32_t n_rows = (uint32_t)p.BH * op.Nq;
    constexpr uint32_t kRows = 256 / (D / 4);
    ProfileScope prof("select_attn_bwd_dq_merge", stream);
    select_dq_merge_kernel<D><<<dim3((n_rows + kRows - 1) / kRows), 256, 0, stream>>>(p, n_rows);
  }
}

template <int D, int OCC, bool kFine>
void launch_dkv(const AttnOperands& op, SelectBwdParams p, hipStream_t stream) {
  p.tiles = blocks_of(op.Nq, kWaves * 16);
  p.by_xcd = true;
  ProfileScope prof("select_attn_bwd_dkv_bf16", stream);
  select_bwd_dkv_kernel<D, OCC, kFine><<<dim3(work_grid_size(p.tiles, p.BH)), kWaves * 64, 0, stream>>>(p);
}

}  // namespace

size_t select_bwd_bytes(const DevGeom& g, int Nq) {
  const size_t rows = (size_t)g.B * g.H * Nq;
  return ((2 * rows + 3) / 4 * 4 + (select_may_split(g.n_cus, g.B * g.H, Nq) ? kMaxSelectSplits * rows * g.D : 0)) * sizeof(float);
}

hipError_t launch_select_bwd_bf16(const DevGeom& g, const AttnOperands& op, const SelectStaged& staged, const SelectLists& lists,
                                  const void* out, const float* lse, const void* dout, float* dq, float* dk, float* dv, float* scratch,
                                  hipStream_t stream) {
  SelectBwdParams p;
  p.staged = staged;
  p.v_chunk = (const __bf16*)op.v_chunk;
  p.k_cache = (const __bf16*)op.k_cache;
  p.v_cache = (const __bf16*)op.v_cache;
  p.out = (const __bf16*)out;
  p.dout = (const __bf16*)dout;
  p.lse = lse;
  p.neg_delta = scratch;
  p.neg_lse2 = scratch + (size_t)g.B * g.H * op.Nq;
  p.splits = 1;
  p.dq_part = select_may_split(g.n_cus, g.B * g.H, op.Nq) ? scratch + (2 * (size_t)g.B * g.H * op.Nq + 3) / 4 * 4 : nullptr;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.rot = RotaryTables{staged.tab_t, g.tab_h, g.tab_w, g.n_t, g.n_h, g.n_w, g.gw, g.T, op.Nq / g.T};
  p.H = g.H;
  p.Nq = op.Nq;
  p.BH = g.B * g.H;
  p.tiles = 0;
  p.group = op.group;
  p.block_rows = op.block_rows;
  p.by_xcd = true;
  p.cache_rows = (int64_t)g.C * g.T;
  p.scale = 1.0f / sqrtf((float)g.D);
  p.hist_rows = op.hist_rows;
  if (staged.q_rest) {  // a few workgroups, each alone on its CU
    if (g.D == 128) {
      launch_dq<128, 1, 2, 1, true>(g, op, lists, p, stream);
      launch_dkv<128, 1, true>(op, p, stream);
    } else {
      launch_dq<64, 1, 3, 1, true>(g, op, lists, p, stream);
      launch_dkv<64, 1, true>(op, p, stream);
    }
  } else if (g.D == 128) {
    launch_dq<128, 1, 2, 3, false>(g, op, lists, p, stream);
    launch_dkv<128, 2, false>(op, p, stream);
  } else {
    if (lists.query_block % 128 == 0)
      launch_dq<64, 2, 3, 2, false>(g, op, lists, p, stream);
    else
      launch_dq<64, 1, 3, 3, false>(g, op, lists, p, stream);
    launch_dkv<64, 3, false>(op, p, stream);
  }
  return hipGetLastError();
}

}  // namespace astro

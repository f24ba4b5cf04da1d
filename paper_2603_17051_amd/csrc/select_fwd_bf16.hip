// Attention of the chunk over selected blocks of the ring and over the chunk itself, bf16 MFMA with fp32 accumulation:
//   out_i = sum over j in S_i of P_ij V_j,  P = softmax of <Q~_i, K~_j> / sqrt(D) over S_i,
//   S_i = rows of the blocks listed for i's group of queries, and the chunk rows that i sees.
// One pass over the keys with a running reference and sum, everything transposed so that a lane owns queries:
//   S^T[key][q] = K (Q_hi + Q_lo)^T  (+ K_lo Q_hi^T for the chunk's keys; cached keys are bf16 by definition)
//   O^T[d][q]  += V^T P^T            (B = P^T straight from the accumulators of S^T)
// The scores keep 16 bits of the rotated queries and keys (24 for few rows, see select_rules.hpp), because the log-sum-exp goes out in fp32 and
// the backward takes probabilities from it; with operands rounded once it was up to 1e-4 off at 64 keys, now 1e-7 (and the pass 360 us where
// it is 516 now, 4680 queries of 12 heads of 128 over 7168 cached and 4680 chunk keys).  Only P is rounded (the output is bf16): the
// log-sum-exp is of what it was before, the output's weights are the rounded ones over their sum, so that they sum to 1.  Bound by the
// products, 3 per cached and 4 per chunk key and query: 578 GFLOP there in 490 us behind the staging, 1180 TFLOP/s.
// A workgroup owns queries of ONE group, turns the group's list into a list of tiles in LDS, and fetches tile after tile
// through it, two ahead.
#include "select_rules.hpp"
#include "select_walk.hpp"

namespace astro {
namespace {

constexpr int kWaves = 4, kStages = 3;
constexpr float kSumLimit = 0x1p44f, kTiny = 0x1p-60f;  // what a row's probabilities may sum to before its reference moves

struct SelectFwdParams {
  SelectStaged staged;
  const __bf16 *v_chunk, *k_cache, *v_cache;
  __bf16* out;
  float* lse;
  // key ranges: workgroup (pair, split, tile) walks the split's share of its tiles and leaves its normalised output and
  // log-sum-exp in part `split`; a merge launch combines them
  int splits;
  float *out_part, *lse_part;  // [splits][B, Nq, H, D], [splits][B][H][Nq]
  int H, Nq, BH, q_tiles, group, block_rows;
  bool by_xcd;
  int64_t cache_rows;
  StreamInts hist_rows;
};

// 16 * QS queries of a wave: lane (i = lane % 16, g = lane / 16) owns queries 16 * qs + i.
template <int D, int QS, bool kFine>
struct SelectFwdWave {
  static constexpr int KS = D / 32, DT = D / 16;
  bf16x8 qh[QS][KS], ql[QS][KS], qr[kFine ? QS : 1][KS];
  f32x4 o[DT][QS];
  float ref[QS], sum[QS], weight[QS];  // softmax reference in log2 units, this lane's parts of the row's sum before and after P is rounded
  OperandAddr16<D> addr;
  int g;

  __device__ __forceinline__ void init(int lane) {
    g = lane >> 4;
    addr.init(lane);
    clear();
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      ref[qs] = 0.f;
      sum[qs] = weight[qs] = 0.f;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][qs] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  __device__ __forceinline__ bool not_numbers_yet() const {
    bool x = false;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) x = x || not_numbers(o[dt][qs]);
    return x;
  }

  // The rare path: scores s and their parts of the sums relative to the references, which move for the rows that need it.
  template <typename Probabilities>
  __device__ __forceinline__ void move_reference(const f32x4 (&s)[2][QS], const float (&part)[QS], const Probabilities& probabilities) {
    float total[QS], less[QS];
    bool needed[QS], any = false;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {  // (a lane alone may have seen nothing but masked keys)
      total[qs] = sum_quarters(sum[qs]);
      const float here = sum_quarters(part[qs]);
      needed[qs] = !(here <= kSumLimit) || !(total[qs] + here >= kTiny);
      any = any || needed[qs];
    }
    if (!__any(any)) return;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      float mx = kNegBig;
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[kh][qs][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      // to the larger of this tile's largest score and of what has been summed; nothing seen yet: to the former, or not at all
      if (total[qs] > 0.f)
        less[qs] = fmaxf(fmaxf(mx, __log2f(total[qs])), -120.f);
      else
        less[qs] = mx > -1.0e28f ? mx : 0.f;
      if (!needed[qs]) less[qs] = 0.f;  // a row's result does not depend on its neighbours
      const float alpha = total[qs] > 0.f ? fast_exp2(-less[qs]) : 0.f;
      sum[qs] *= alpha;
      weight[qs] *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt][qs] = o[dt][qs] * alpha;
      ref[qs] += less[qs];
    }
    probabilities(less);
  }

  // One tile of 32 keys, of which the first live[qs] count for this lane's query qs (fewest, wave-uniform, for any of the wave).
  // kCare: with care (see each_bound()), for tiles of both kinds (`ring`: which; a second instance of the careful code moved the registers
  // of the backward's first walk, 1080 -> 1270 us); else what the tile holds has to be finite.
  template <bool kChunk, bool kCare>
  __device__ __forceinline__ void tile(const char* stage, const int (&live)[QS], int fewest, bool ring) {
    const char *vs = stage + kSelectTile * D * 2, *lo = vs + kSelectTile * D * 2;
    f32x4 s[2][QS], start[2][QS];  // the scores come out relative to the reference
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) start[kh][qs] = f32x4{-ref[qs], -ref[qs], -ref[qs], -ref[qs]};
    if constexpr (kFine)
      scores_from_thirds<D, QS, kCare>(stage, lo, lo + kSelectTile * D * 2, !ring, addr, qh, ql, qr, start, s);
    else if constexpr (kCare)
      scores_of_any<D, QS>(stage, lo, !ring, addr, qh, ql, start, s);
    else
      scores_from_halves<D, QS, kChunk>(stage, lo, addr, qh, ql, start, s);
    bf16x8 v[2][4];  // of the output's columns, four at a time: the first under the softmax
    if constexpr (!kCare) read_quad<D>(vs, addr, 0, v[0]);
    if (kCare || fewest < kSelectTile) {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int qs = 0; qs < QS; ++qs)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[kh][qs][r] = 16 * kh + 4 * g + r >= live[qs] ? kNegBig : s[kh][qs][r];
    }
    __builtin_amdgcn_sched_barrier(0);
    // Probabilities relative to the current reference, which starts at 0 and moves only when a row needs it: its probabilities
    // outgrow it (a huge or infinite sum), or all it has seen are so small that they may vanish.  fp32 sums and bf16's
    // exponents hold what lies between.
    float part[QS], rounded[QS];
    bf16x8 pb[QS];
    auto probabilities = [&](const float (&less)[QS]) __attribute__((always_inline)) {
#pragma unroll
      for (int qs = 0; qs < QS; ++qs) {
        part[qs] = rounded[qs] = 0.f;
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int r = 0; r < 4; r += 2) {
            const f32x2 e = {fast_exp2(s[kh][qs][r] - less[qs]), fast_exp2(s[kh][qs][r + 1] - less[qs])};
            part[qs] += e[0] + e[1];
            const bf16x2 x = __builtin_convertvector(e, bf16x2);
            rounded[qs] = add_pair(x, rounded[qs]);
            pb[qs][4 * kh + r] = x[0];
            pb[qs][4 * kh + r + 1] = x[1];
          }
      }
    };
    const float none[QS] = {};
    probabilities(none);
    bool look = false;
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) look = look || !(part[qs] <= kSumLimit) || !(sum[qs] + part[qs] >= kTiny);
    if (__builtin_expect(__any(look), 0)) move_reference(s, part, probabilities);
#pragma unroll
    for (int qs = 0; qs < QS; ++qs) {
      sum[qs] += part[qs];
      weight[qs] += rounded[qs];
    }
    if constexpr (kCare) {
#pragma unroll
      for (int qs = 0; qs < QS; ++qs)
        each_bound(live[qs], [&](int bound, bool mine) __attribute__((always_inline)) {
          const u32x4 mask = rows_between(g, 0, bound);
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            o[dt][qs] = either(mine, mfma16(only(mask, read_cols16<D>(vs, addr.tr[dt], 0)), pb[qs], o[dt][qs]), o[dt][qs]);
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      return;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int quad = 0; quad < DT / 4; ++quad) {
      if (quad + 1 < DT / 4) read_quad<D>(vs, addr, quad + 1, v[(quad + 1) & 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int qs = 0; qs < QS; ++qs) o[4 * quad + i][qs] = mfma16(v[quad & 1][i], pb[qs], o[4 * quad + i][qs]);
    }
  }
};

template <int D, int QS, int OCC, bool kFine>
__global__ void __launch_bounds__(kWaves * 64, OCC) select_fwd_kernel(SelectFwdParams p, SelectLists lists) {
  using Wave = SelectFwdWave<D, QS, kFine>;
  using Walk = SelectWalk<D, kWaves, kFine>;
  using Stages = SelectStages<D, kWaves, kStages, kFine>;
  constexpr int kAhead = kStages - 1, kQueries = kWaves * 16 * QS;
  __shared__ __attribute__((aligned(1024))) char lds[Stages::kBytes];
  __shared__ TileList tile_list;

  const WorkItem item = work_item(p.q_tiles, p.BH * p.splits, p.by_xcd);
  if (!item.valid) return;
  const int split = item.bh % p.splits;
  const PairIndex pair = split_pair(item.bh / p.splits, p.H, p.group);
  const int b = pair.b, h = pair.h;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int64_t bh = (int64_t)b * p.H + h;
  const int q_wg = item.tile * kQueries, q_wave = q_wg + wave * 16 * QS, q_last = p.Nq - 1;
  if (wave == 0)
    fill_tile_list(lists, lists.blocks + (bh * lists.groups + q_wg / lists.query_block) * lists.n_select, p.hist_rows.v[pair.cache_b] / lists.T,
                   &tile_list);
  const int vis_wave = visible_chunk_rows(q_wave < q_last ? q_wave : q_last, p.Nq, p.block_rows);
  const int vis_last = visible_chunk_rows(q_wg + kQueries - 1 < q_last ? q_wg + kQueries - 1 : q_last, p.Nq, p.block_rows);

  Wave w;
  w.init(lane);
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const int q = q_wave + 16 * qs + i16;
    const int64_t at = (bh * p.Nq + (q < p.Nq ? q : q_last)) * D + g * 8;
#pragma unroll
    for (int st = 0; st < Wave::KS; ++st) {
      w.qh[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_hi + at + st * 32);
      w.ql[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_lo + at + st * 32);
      if constexpr (kFine) w.qr[qs][st] = *reinterpret_cast<const bf16x8*>((const __bf16*)p.staged.q_rest + at + st * 32);
    }
  }
  // The queries have to be here before the first tile is asked for: the compiler does not count the walk's loads, and would wait
  // for the queries inside the loop, which is for all of the loads in flight there, on every tile (D = 64, 64 queries: 0.89 us a tile, 0.68 without).
  wait_vmem();
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

  // Invariant at the top of tile t: it has landed and is visible to every wave, the tile behind it may be in flight, and the
  // stage of tile t + kAhead (= that of tile t - 1) is free.
  auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < kAhead; ++t)
      if (t_begin + t < t_end) walk.issue(t_begin + t, walk.entry(t_begin + t), Stages::of(lds, t));
    walk.wait_all_but(t_begin + kAhead - 1, t_end);
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
        const int q = q_wave + 16 * qs + i16;
        live[qs] = min(max(visible_chunk_rows(q < q_last ? q : q_last, p.Nq, p.block_rows) - row0, 0), kSelectTile);
      }
    }
    w.template tile<kChunk, kCare>(stage, live, fewest, ring);
    walk.wait_all_but(t + kAhead, t_end);
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

  // normalise, write O [B, Nq, H, D] and LSE [B, H, Nq] (of this split's keys)
#pragma unroll
  for (int qs = 0; qs < QS; ++qs) {
    const float l_tot = sum_quarters(w.sum[qs]);
    // a key range in which a query sees nothing reports zeros and a log-sum-exp of -inf, weight 0 in the merge; a sum that is not a number
    // stays one
    const bool nothing = p.splits > 1 && l_tot == 0.f;
    const float inv = nothing ? 0.f : 1.f / sum_quarters(w.weight[qs]), lse = w.ref[qs] * kLn2 + __logf(l_tot);
    const int q = q_wave + 16 * qs + i16;
    if (q >= p.Nq) continue;
    const int64_t row = (((int64_t)b * p.Nq + q) * p.H + h) * D + 4 * g;
    if (p.splits > 1) {
      float* part = p.out_part + (int64_t)split * p.BH * p.Nq * D + row;
#pragma unroll
      for (int dt = 0; dt < Wave::DT; ++dt) *reinterpret_cast<f32x4*>(part + 16 * dt) = w.o[dt][qs] * inv;
      if (g == 0) p.lse_part[(int64_t)split * p.BH * p.Nq + bh * p.Nq + q] = lse;
    } else {
#pragma unroll
      for (int dt = 0; dt < Wave::DT; ++dt) {
        bf16x4 x;
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = (__bf16)(w.o[dt][qs][c] * inv);
        *reinterpret_cast<bf16x4*>(p.out + row + 16 * dt) = x;
      }
      if (g == 0) p.lse[bh * p.Nq + q] = lse;
    }
  }
}

// Softmax over the union of the ranges' keys: their outputs weighted by exp(lse_s - lse).  Bound by the parts' bytes; all of a
// row's are in flight before the first is used.  (Parts are below 2^32 bytes, see select_may_split().)
template <int D>
__global__ void __launch_bounds__(256) select_merge_kernel(SelectFwdParams p, uint32_t n_rows) {
  constexpr uint32_t CPR = D / 4;
  const uint32_t row = blockIdx.x * (256 / CPR) + threadIdx.x / CPR;  // (b * Nq + q) * H + h
  if (row >= n_rows) return;
  const uint32_t c = threadIdx.x % CPR, bq = row / (uint32_t)p.H, b = bq / (uint32_t)p.Nq;
  const uint32_t lse_at = (b * p.H + (row - bq * p.H)) * p.Nq + (bq - b * p.Nq);
  float m = kNegBig, l[kMaxSelectSplits];  // (m: over no number; one that is none makes its weight none)
  f32x4 o[kMaxSelectSplits];
#pragma unroll
  for (uint32_t s = 0; s < kMaxSelectSplits; ++s) {  // (the first part again for those that are not there: no branch between loads)
    const uint32_t from = s < (uint32_t)p.splits ? s : 0;
    o[s] = *reinterpret_cast<const f32x4*>((const char*)p.out_part + ((from * n_rows + row) * CPR + c) * 16u);
    l[s] = p.lse_part[from * n_rows + lse_at];
  }
#pragma unroll
  for (int s = 0; s < kMaxSelectSplits; ++s) m = fmaxf(m, l[s]);
  float tot = 0.f;
  f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kMaxSelectSplits; ++s) {
    const float w = s < p.splits ? __expf(l[s] - m) : 0.f;
    tot += w;
    a += s < p.splits ? o[s] * w : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bf16x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (__bf16)(a[i] / tot);
  *reinterpret_cast<bf16x4*>(p.out + (int64_t)row * D + c * 4) = x;
  if (c == 0) p.lse[lse_at] = m + __logf(tot);
}

template <int D, int QS, int OCC, bool kFine>
hipError_t launch(const DevGeom& g, const AttnOperands& op, const SelectStaged& staged, const SelectLists& lists, void* out, float* lse,
                  float* parts, hipStream_t stream) {
  SelectFwdParams p;
  p.staged = staged;
  p.v_chunk = (const __bf16*)op.v_chunk;
  p.k_cache = (const __bf16*)op.k_cache;
  p.v_cache = (const __bf16*)op.v_cache;
  p.out = (__bf16*)out;
  p.lse = lse;
  p.H = g.H;
  p.Nq = op.Nq;
  p.BH = g.B * g.H;
  p.q_tiles = blocks_of(op.Nq, kWaves * 16 * QS);
  p.group = op.group;
  p.block_rows = op.block_rows;
  p.cache_rows = (int64_t)g.C * g.T;
  p.hist_rows = op.hist_rows;
  const CallShape shape = select_call_shape(g, op, lists);
  p.splits = parts ? select_splits(select_fwd_cost(D, kWaves * 16 * QS), g.n_cus, p.q_tiles * p.BH, mean_keys(shape) / kSelectTile,
                                   (double)p.BH * op.Nq * D * sizeof(float))
                   : 1;
  p.by_xcd = order_by_xcd(shape, p.q_tiles * p.BH * p.splits);
  const int64_t n_rows = (int64_t)p.BH * op.Nq;
  p.out_part = parts;
  p.lse_part = parts ? parts + p.splits * n_rows * D : nullptr;
  {
    ProfileScope prof("select_attn_fwd_bf16", stream);
    select_fwd_kernel<D, QS, OCC, kFine><<<dim3(work_grid_size(p.q_tiles, p.BH * p.splits)), kWaves * 64, 0, stream>>>(p, lists);
  }
  if (p.splits > 1) {
    ProfileScope prof("select_attn_fwd_merge", stream);
    constexpr int kRows = 256 / (D / 4);
    select_merge_kernel<D><<<dim3((unsigned)((n_rows + kRows - 1) / kRows)), 256, 0, stream>>>(p, (uint32_t)n_rows);
  }
  return hipGetLastError();
}

}  // namespace

size_t select_fwd_split_bytes(const DevGeom& g, int Nq) {
  if (!select_may_split(g.n_cus, g.B * g.H, Nq)) return 0;
  return (size_t)kMaxSelectSplits * g.B * g.H * Nq * (g.D + 1) * sizeof(float);
}

hipError_t launch_select_fwd_bf16(const DevGeom& g, const AttnOperands& op, const SelectStaged& staged, const SelectLists& lists, void* out,
                                  float* lse, float* parts, hipStream_t stream) {
  const bool wide = lists.query_block % 128 == 0;
  auto run = [&](auto f) { return f(g, op, staged, lists, out, lse, parts, stream); };
  if (staged.q_rest) {  // a few workgroups, each alone on its CU
    if (g.D == 128) return wide ? run(launch<128, 2, 1, true>) : run(launch<128, 1, 1, true>);
    return wide ? run(launch<64, 2, 1, true>) : run(launch<64, 1, 1, true>);
  }
  if (g.D == 128) return wide ? run(launch<128, 2, 2, false>) : run(launch<128, 1, 2, false>);
  return wide ? run(launch<64, 2, 3, false>) : run(launch<64, 1, 3, false>);
}

}  // namespace astro

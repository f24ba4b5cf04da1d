// The walk over the keys that a group of queries attends to: the selected blocks of the ring, then the chunk's own rows.
#pragma once

#include "kernels.hpp"
#include "mfma_common.hpp"

namespace astro {

constexpr int kSelectTile = 32;  // key rows of a tile
static_assert(ASTRO_MAX_SELECT_ROWS % kSelectTile == 0, "whole tiles");
constexpr int kMaxSelectTiles = ASTRO_MAX_SELECT_ROWS / kSelectTile;

// The ring tiles of a list, in LDS: full tiles from the front, those that a frame's end cuts short from the back, so that a
// walk takes all full ones without a test.  An entry is first row * 32 + rows - 1.
struct TileList {
  uint32_t entry[kMaxSelectTiles];
  int full, partial;
  int again;  // see each_bound()
};

// One wave fills the list.  A number counts if it is larger than every one before it in the list and the number of a
// block of a resident frame: a block is taken once however often it is listed, and nothing that a list may hold
// leads outside the resident rows.
__device__ __forceinline__ void fill_tile_list(const SelectLists& s, const int32_t* list, int resident_frames, TileList* to) {
  const int lane = threadIdx.x & 63;
  int top = -1, full = 0, partial = 0;
  for (int e0 = 0; e0 < s.n_select; e0 += 64) {
    const int x = e0 + lane < s.n_select ? list[e0 + lane] : -1;
    int most = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(most, d);
      if (lane >= d && y > most) most = y;
    }
    int before = __shfl_up(most, 1);
    if (lane == 0 || before < top) before = top;
    const bool counts = x > before && x < resident_frames * s.frame_blocks;
    const int last = __shfl(most, 63);
    top = last > top ? last : top;
    const int frame = counts ? x / s.frame_blocks : 0, first = counts ? (x - frame * s.frame_blocks) * s.key_block : 0;
    const int left = s.T - first, rows = counts ? (left < s.key_block ? left : s.key_block) : 0;
    const uint32_t row0 = (uint32_t)(frame * s.T + first);
    const int tiles = rows / kSelectTile, rest = rows % kSelectTile;
    int upto = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    for (int i = 0; i < tiles; ++i) to->entry[full + upto - tiles + i] = (row0 + i * kSelectTile) * kSelectTile + kSelectTile - 1;
    const uint64_t cut = __ballot(rest != 0);
    if (rest) to->entry[kMaxSelectTiles - 1 - (partial + __popcll(cut & ((1ull << lane) - 1)))] = (row0 + tiles * kSelectTile) * kSelectTile + rest - 1;
    full += __shfl(upto, 63);
    partial += __popcll(cut);
  }
  if (lane == 0) {
    to->full = full;
    to->partial = partial;
    to->again = 0;
  }
}

// A [32 rows][D] tile that WAVES waves fill together by direct-to-LDS loads, 16 bytes per lane; rows past the end of the
// source read as zeros.  The loads are issued from assembly, as PrivateStream's (see there): the compiler waits for all
// of its own before the next LDS read, which here belongs to another stage, and would end the prefetch of two tiles.
template <int D, int WAVES>
struct SharedStream {
  static constexpr int CPR = D / 8, kRowsPerInst = 64 / CPR, kInsts = kSelectTile / (kRowsPerInst * WAVES);
  static_assert(kInsts * kRowsPerInst * WAVES == kSelectTile, "the tile divides over the waves");
  static constexpr int kPatterns = 16 % (kRowsPerInst * WAVES) == 0 ? 16 / (kRowsPerInst * WAVES) : 1;  // the swizzle repeats every 16 rows
  uint32_t lane_row, chunk[kPatterns];
  uint32_t wave_at;

  __device__ __forceinline__ void init() {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    lane_row = wave * kRowsPerInst + lane / CPR;
    wave_at = wave * 1024;
#pragma unroll
    for (int u = 0; u < kPatterns; ++u) chunk[u] = ((lane % CPR) ^ swizzle16<CPR>(u * WAVES * kRowsPerInst + (int)lane_row)) * 16;
  }
  __device__ __forceinline__ void issue(const u32x4 rsrc, uint32_t stride_bytes, uint32_t row0, const char* lds_tile) const {
    typedef const char __attribute__((address_space(3))) * lds_ptr;
    const uint32_t dst = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)lds_tile) + wave_at;
#pragma unroll
    for (int u = 0; u < kInsts; ++u) {
      const uint32_t off = (row0 + u * WAVES * kRowsPerInst + lane_row) * stride_bytes + chunk[u % kPatterns];
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst + u * WAVES * 1024), "v"(off), "s"(rsrc)
                   : "memory", "m0");
    }
  }
};

// The workgroup's LDS ring of tile stages: K rows, V rows, and for chunk tiles what the rounding of the rotated keys left: a second piece
// and, if kFine, a third.
template <int D, int WAVES, int STAGES, bool kFine>
struct SelectStages {
  static constexpr int kTileBytes = kSelectTile * D * 2, kTiles = kFine ? 4 : 3, kBytes = STAGES * kTiles * kTileBytes;
  static __device__ __forceinline__ char* of(char* lds, int t) { return lds + (t % STAGES) * kTiles * kTileBytes; }
};

// What a workgroup walks: tiles [0, ring_tiles) from the list, then the chunk's rows in order, 32 to a tile, as far as its last
// query sees them.
template <int D, int WAVES, bool kFine>
struct SelectWalk {
  static constexpr int kTileBytes = kSelectTile * D * 2, kInsts = SharedStream<D, WAVES>::kInsts;
  SharedStream<D, WAVES> stream;
  const TileList* list;
  u32x4 k_ring, v_ring, k_hi, k_lo, k_rest, v_chunk;
  uint32_t v_chunk_stride;
  int full, ring_tiles, tiles;

  // after the list is there for all; vis_last: chunk rows that the workgroup's last query sees
  __device__ __forceinline__ void init(const TileList* l, int vis_last) {
    list = l;
    full = __builtin_amdgcn_readfirstlane(l->full);
    ring_tiles = full + __builtin_amdgcn_readfirstlane(l->partial);
    tiles = ring_tiles + (vis_last + kSelectTile - 1) / kSelectTile;
    stream.init();
  }
  // where tile t lies (any entry for a chunk tile)
  __device__ __forceinline__ uint32_t entry(int t) const {
    return list->entry[t < full ? t : t < ring_tiles ? kMaxSelectTiles - 1 - (t - full) : 0];
  }
  // rows of ring tile t
  __device__ __forceinline__ int rows_of(int t) const {
    return t < full ? kSelectTile : (int)(__builtin_amdgcn_readfirstlane(entry(t)) % kSelectTile) + 1;
  }
  __device__ __forceinline__ void issue(int t, uint32_t entry_of_t, char* stage) const {
    if (t < ring_tiles) {
      const uint32_t e = __builtin_amdgcn_readfirstlane(entry_of_t), row0 = e / kSelectTile, rows = e % kSelectTile + 1;
      u32x4 k = k_ring, v = v_ring;
      k.z = v.z = (row0 + rows) * (D * 2);  // past its last row a tile reads zeros, whatever the next frame holds
      stream.issue(k, D * 2, row0, stage);
      stream.issue(v, D * 2, row0, stage + kTileBytes);
    } else {
      const uint32_t row0 = (uint32_t)(t - ring_tiles) * kSelectTile;
      stream.issue(k_hi, D * 2, row0, stage);
      stream.issue(v_chunk, v_chunk_stride, row0, stage + kTileBytes);
      stream.issue(k_lo, D * 2, row0, stage + 2 * kTileBytes);
      if constexpr (kFine) stream.issue(k_rest, D * 2, row0, stage + 3 * kTileBytes);
    }
  }
  // whether any wave of the workgroup has to walk again
  __device__ __forceinline__ bool again(TileList* l, bool wave_has_to) const {
    if (__any(wave_has_to)) l->again = 1;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(l->again) != 0;
  }
  // until no more than tile `newest` (if it exists) is in flight
  __device__ __forceinline__ void wait_all_but(int newest, int end) const {
    if (newest >= end)
      wait_vmem();
    else if (newest < ring_tiles)
      wait_vmem_except<2 * kInsts>();
    else
      wait_vmem_except<(kFine ? 4 : 3) * kInsts>();
  }
};

// x = hi + lo, two bf16 each that hold 16 bits of it: products of the halves keep 2^-17 where a rounded operand keeps 2^-9.
struct HalfPairs {
  bf16x2 hi, lo;
};
__device__ __forceinline__ HalfPairs halves(f32x2 x) {
  const bf16x2 hi = __builtin_convertvector(x, bf16x2);
  return HalfPairs{hi, __builtin_convertvector(x - __builtin_convertvector(hi, f32x2), bf16x2)};
}

// The same where x may be infinite: no small half then, which would be inf - inf.
__device__ __forceinline__ HalfPairs halves_of_any(f32x2 x) {
  const bf16x2 hi = __builtin_convertvector(x, bf16x2);
  const f32x2 big = __builtin_convertvector(hi, f32x2), rest = x - big;
  return HalfPairs{hi, __builtin_convertvector(f32x2{__builtin_isfinite(big[0]) ? rest[0] : 0.f, __builtin_isfinite(big[1]) ? rest[1] : 0.f}, bf16x2)};
}
// of a sum without and with its products of small halves: the former where it is infinite or not a number (a small half has a sign of its own or is 0)
__device__ __forceinline__ f32x4 with_small(const f32x4& without, const f32x4& with) {
  f32x4 x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __builtin_isfinite(without[i]) ? with[i] : without[i];
  return x;
}

// The scores of 16 rows of the other side in fp32 from halves: S = start + A (B_hi + B_lo)^T (+ A_lo B_hi^T), where A comes from an
// LDS tile and B is held, N sub-blocks of 16 rows of it.  An MFMA takes its result's place in the next but one at the earliest:
// products on one accumulator are kept four apart, for N = 1 by an accumulator of their own for the small ones.
// Operands are read ahead of the products: read where they were used, each waited for the LDS (alone on its CU, a forward tile of 128
// columns took 1.1 us, of which its products are 0.3).
template <int D, int N, bool kLow>
__device__ __forceinline__ void scores_from_halves(const char* tile, const char* low, const OperandAddr16<D>& addr, const bf16x8 (&hi)[N][D / 32],
                                                   const bf16x8 (&lo)[N][D / 32], const f32x4 (&start)[2][N], f32x4 (&s)[2][N]) {
  constexpr int KS = D / 32;
  f32x4 small[2];
  bf16x8 a[KS][2], c[2][2];  // all of A at once; of A_lo a step ahead
#pragma unroll
  for (int st = 0; st < KS; ++st)
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) a[st][kh] = read_rows16<D>(tile, addr.row[st], 16 * kh);
#pragma unroll
  for (int kh = 0; kh < 2; ++kh) {
    if constexpr (kLow) c[0][kh] = read_rows16<D>(low, addr.row[0], 16 * kh);
    small[kh] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < N; ++n) s[kh][n] = start[kh][n];
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int st = 0; st < KS; ++st) {
    if constexpr (kLow)
      if (st + 1 < KS)
#pragma unroll
        for (int kh = 0; kh < 2; ++kh) c[(st + 1) & 1][kh] = read_rows16<D>(low, addr.row[st + 1], 16 * kh);
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int n = 0; n < N; ++n) s[kh][n] = mfma16(a[st][kh], hi[n][st], s[kh][n]);
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        f32x4& to = N == 1 ? small[kh] : s[kh][n];
        to = mfma16(a[st][kh], lo[n][st], to);
      }
    if constexpr (kLow) {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int n = 0; n < N; ++n) {
          f32x4& to = N == 1 ? small[kh] : s[kh][n];
          to = mfma16(c[st & 1][kh], hi[n][st], to);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if constexpr (N == 1)
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) s[kh][0] += small[kh];
}

// The same, bit for bit, where the sums without small halves are numbers; where operands may be infinite.  with_low: whether there is an A_lo.
template <int D, int N>
__device__ __forceinline__ void scores_of_any(const char* tile, const char* low, bool with_low, const OperandAddr16<D>& addr, const bf16x8 (&hi)[N][D / 32],
                                              const bf16x8 (&lo)[N][D / 32], const f32x4 (&start)[2][N], f32x4 (&s)[2][N]) {
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      f32x4 big = start[kh][n], all = big, small = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < D / 32; ++st) {
        const bf16x8 a = read_rows16<D>(tile, addr.row[st], 16 * kh);
        bf16x8 c{};
        if (with_low) c = read_rows16<D>(low, addr.row[st], 16 * kh);
        big = mfma16(a, hi[n][st], big);
        if constexpr (N == 1) {  // in the order of the products above
          small = mfma16(c, hi[n][st], mfma16(a, lo[n][st], small));
        } else {
          all = mfma16(c, hi[n][st], mfma16(a, lo[n][st], mfma16(a, hi[n][st], all)));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      s[kh][n] = with_small(big, N == 1 ? big + small : all);
    }
}

// Scores from three pieces each: A B^T but for the three smallest products, 24 bits.  rest: A's third pieces; with_low: whether A has more pieces
// than one.  kCare: as in scores_of_any().
template <int D, int N, bool kCare>
__device__ __forceinline__ void scores_from_thirds(const char* tile, const char* low, const char* rest, bool with_low, const OperandAddr16<D>& addr,
                                                   const bf16x8 (&hi)[N][D / 32], const bf16x8 (&lo)[N][D / 32], const bf16x8 (&third)[N][D / 32],
                                                   const f32x4 (&start)[2][N], f32x4 (&s)[2][N]) {
  constexpr int KS = D / 32;
  f32x4 of_b[2][N], of_a[2][N];  // small products, by whose pieces are small: sums of their own, so that fewer wait for one another
  bf16x8 a[KS][2], c[KS][2], e[KS][2];
#pragma unroll
  for (int st = 0; st < KS; ++st)
#pragma unroll
    for (int kh = 0; kh < 2; ++kh) {
      a[st][kh] = read_rows16<D>(tile, addr.row[st], 16 * kh);
      if (with_low) {
        c[st][kh] = read_rows16<D>(low, addr.row[st], 16 * kh);
        e[st][kh] = read_rows16<D>(rest, addr.row[st], 16 * kh);
      } else {
        c[st][kh] = e[st][kh] = bf16x8{};
      }
    }
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[kh][n] = start[kh][n];
      of_a[kh][n] = of_b[kh][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int st = 0; st < KS; ++st) {
    auto product = [&](const bf16x8 (&x)[2], const bf16x8 (&y)[N][KS], f32x4 (&to)[2][N]) __attribute__((always_inline)) {
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int n = 0; n < N; ++n) to[kh][n] = mfma16(x[kh], y[n][st], to[kh][n]);
    };
    product(a[st], hi, s);
    product(a[st], lo, of_b);
    if (with_low) product(c[st], hi, of_a);
    product(a[st], third, of_b);
    if (with_low) {
      product(c[st], lo, of_a);
      product(e[st], hi, of_a);
    }
  }
#pragma unroll
  for (int kh = 0; kh < 2; ++kh)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const f32x4 all = s[kh][n] + (of_a[kh][n] + of_b[kh][n]);
      s[kh][n] = kCare ? with_small(s[kh][n], all) : all;
    }
}

// Operands of the products that contract over a tile's 32 rows: columns 16 (4 quad) .. 16 (4 quad + 3) + 15 of it.
template <int D>
__device__ __forceinline__ void read_quad(const char* tile, const OperandAddr16<D>& addr, int quad, bf16x8 (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = read_cols16<D>(tile, addr.tr[4 * quad + i], 0);
}

// Values that are not finite.  A probability of 0 does not keep a row that a query does not see (behind the end of a causal block) out of a
// matrix product whose element there is infinite or not a number: 0 * inf.  And products of small halves turn an infinite sum into inf - inf.  A
// workgroup whose result is not a number therefore walks again, with care: tiles go through the products once for every distinct
// bound of a wave's lanes, with the rows behind the bound (or before it) as zeros, a lane takes the result of its own, and sums
// that are infinite without small halves stay as they are.  Done so at once, the passes at frames of 391 rows of D = 64 took a quarter to a half longer.
template <typename F>
__device__ __forceinline__ void each_bound(int bound, F f) {
  uint64_t left = ~0ull;
  while (left != 0) {
    const int x = __builtin_amdgcn_readlane(bound, __ffsll((unsigned long long)left) - 1);
    f(x, bound == x);
    left &= ~__ballot(bound == x);
  }
}
// of the operands of read_quad(): the elements of rows [from, to)
__device__ __forceinline__ u32x4 rows_between(int g, int from, int to) {
  u32x4 m;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int row = 16 * (w / 2) + 4 * g + 2 * (w % 2);
    m[w] = (row >= from && row < to ? 0xffffu : 0u) | (row + 1 >= from && row + 1 < to ? 0xffff0000u : 0u);
  }
  return m;
}
__device__ __forceinline__ bf16x8 only(const u32x4& mask, const bf16x8& x) {
  return __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, x) & mask);
}
__device__ __forceinline__ bool not_numbers(const f32x4& x) { return !(x[0] == x[0] && x[1] == x[1] && x[2] == x[2] && x[3] == x[3]); }
__device__ __forceinline__ f32x4 either(bool first, const f32x4& x, const f32x4& y) { return first ? x : y; }

}  // namespace astro

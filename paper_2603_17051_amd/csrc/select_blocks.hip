// Which blocks of the cache a group of queries attends to: means of the keys of every block, kept by the append, and the
// selection of the blocks whose mean has the largest product with the mean query of the group.
//   kbar[j] = (1/n_j) sum of the block's keys, as they were handed in (before rotation), rounded to fp32
//   qbar[g] = the same over the group's queries
//   score   = <qbar[g], kbar[j]>, rounded to fp32; NaN counts as -inf; the n_select largest, ties to the lower number
// Sums and products are 64 bits: a selection is a set of integers, and in 32 bits its last member would depend on the
// order of the sums.  (bf16 values have 8 bits, so their 64-bit sums over a block are as good as exact in any order.)
// Means of what was handed in do not depend on positions: they stay right when sinks are rotated again.
#include "cached_key.hpp"
#include "kernels.hpp"
#include "mfma_common.hpp"
#include "ring_state.hpp"

namespace astro {
namespace {

constexpr int kThreads = 256;

// Means of the blocks of fp32 frames, beside their append.  grid: x = n_frames * blocks of a frame, y = head, z = stream
template <int D>
__global__ void __launch_bounds__(kThreads) block_means_kernel(DevGeom g, const float* __restrict__ k, float* __restrict__ means, int key_block,
                                                               int frame_blocks, int n_frames, StreamInts next_n) {
  constexpr int kRows = kThreads / D;
  __shared__ double scratch[kThreads];
  const int fi = blockIdx.x / frame_blocks, j = blockIdx.x - fi * frame_blocks, h = blockIdx.y, b = blockIdx.z, d = threadIdx.x % D;
  const int first = j * key_block, n = g.T - first < key_block ? g.T - first : key_block;
  const int slot = slot_of_frame_number((int64_t)next_n.v[b] + fi, g.C, g.S);
  const float* rows = k + ((((int64_t)b * n_frames + fi) * g.T + first) * g.H + h) * D + d;
  double sum = 0.;
  for (int r = threadIdx.x / D; r < n; r += kRows) sum += (double)rows[(int64_t)r * g.H * D];
  scratch[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x >= D) return;
#pragma unroll
  for (int r = 1; r < kRows; ++r) sum += scratch[r * D + d];
  means[(((int64_t)b * g.H + h) * g.C * frame_blocks + (int64_t)slot * frame_blocks + j) * D + d] = (float)(sum / n);
}

// An append of bf16 frames that keeps means: keys rotated into their slots, values copied, as rope_scatter.hip does (the same
// bits), and the means from the keys that pass through.  A workgroup takes one block of one head.  Bound by its bytes, K and V in
// and out; a launch of its own for the means read K again (12 heads of 128, 3 frames of 1560, 4 streams: 51 + 16 us).
// grid: x = n_frames * blocks of a frame, y = head, z = stream
template <int D>
__global__ void __launch_bounds__(kThreads) append_means_kernel(DevGeom g, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                                                                __bf16* __restrict__ k_cache, __bf16* __restrict__ v_cache,
                                                                float* __restrict__ means, int key_block, int frame_blocks, int n_frames,
                                                                StreamInts first_frame, StreamInts next_n) {
  constexpr int CPR = D / 8, kRows = kThreads / CPR, kUnroll = 4;
  __shared__ double scratch[kThreads * 8];
  __shared__ double2 tab_t[D / 2];
  const int fi = blockIdx.x / frame_blocks, j = blockIdx.x - fi * frame_blocks, h = blockIdx.y, b = blockIdx.z, t = threadIdx.x;
  const int first = j * key_block, n = g.T - first < key_block ? g.T - first : key_block;
  const int slot = slot_of_frame_number((int64_t)next_n.v[b] + fi, g.C, g.S);
  const int c = t % CPR, r0 = t / CPR;
  const bool rope = g.n_t + g.n_h + g.n_w != 0;
  const int64_t in0 = ((((int64_t)b * n_frames + fi) * g.T + first) * g.H + h) * D + c * 8, stride = (int64_t)g.H * D;
  const int64_t out0 = (((int64_t)b * g.H + h) * g.C * g.T + (int64_t)slot * g.T + first) * D + c * 8;
  double sum[8] = {};
  for (int base = 0; base < n; base += kUnroll * kRows) {
    bf16x8 x[kUnroll], y[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = base + u * kRows + r0;
      if (r < n) {
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(k + in0 + r * stride));
        y[u] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(v + in0 + r * stride));
      }
    }
    if (rope && base == 0) {  // under the loads
      exact_temporal(g, tab_t, first_frame.v[b] + fi);
      __syncthreads();
    }
    ExactAngles at;
    auto angles = [&](int r) __attribute__((always_inline)) {
      const int tok = first + (r < n ? r : n - 1), row = tok / g.gw;
      at.load_spatial(g, row, tok - row * g.gw, c * 4);
    };
    if (rope) {
      at.load_temporal(g, tab_t, c * 4);
      angles(base + r0);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int r = base + u * kRows + r0;
      if (r >= n) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += (double)(float)x[u][i];
      if (rope) {
        x[u] = cached_key8(x[u], at);
        if (u + 1 < kUnroll) angles(r + kRows);  // before the stores: a wait for them would be a wait for the stores as well
      }
      __builtin_nontemporal_store(x[u], reinterpret_cast<bf16x8*>(k_cache + out0 + r * D));
      __builtin_nontemporal_store(y[u], reinterpret_cast<bf16x8*>(v_cache + out0 + r * D));
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) scratch[r0 * D + c * 8 + i] = sum[i];
  __syncthreads();
  float* to = means + (((int64_t)b * g.H + h) * g.C * frame_blocks + (int64_t)slot * frame_blocks + j) * D;
  for (int d = t; d < D; d += kThreads) {
    double total = 0.;
#pragma unroll
    for (int r = 0; r < kRows; ++r) total += scratch[r * D + d];
    to[d] = (float)(total / n);
  }
}

// scores in the order of unsigned integers
__device__ __forceinline__ uint32_t ordered(float x) {
  x = x != x ? -INFINITY : x == 0.f ? 0.f : x;  // (both zeros are one)
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The n_select largest of a wave's n keys, in the order of their numbers, -1 behind them.  hist: 256 words of this wave.
__device__ __forceinline__ void take_largest(const uint32_t* keys, int n, int n_select, uint32_t* hist, int32_t* list) {
  const int lane = threadIdx.x & 63;
  // The last one taken, a byte at a time from the top: prefix = its bytes so far, want = how many of the keys that begin
  // with them are taken.
  uint32_t prefix = 0, want = n_select;
  const bool all = n <= n_select;
  for (int shift = 24; shift >= 0 && !all; shift -= 8) {
    *reinterpret_cast<u32x4*>(hist + 4 * lane) = u32x4{0, 0, 0, 0};
    wave_lds_sync();
    for (int j = lane; j < n; j += 64) {
      const uint32_t k = keys[j];
      if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[(k >> shift) & 255], 1u);
    }
    wave_lds_sync();
    const u32x4 x = *reinterpret_cast<const u32x4*>(hist + 252 - 4 * lane);  // lane 0: the four largest bytes
    const uint32_t sum = x[0] + x[1] + x[2] + x[3];
    uint32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    uint32_t before = upto - sum, byte = 0, left = 0;
    const bool here = before < want && upto >= want;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      if (left == 0 && before + x[i] >= want) {
        byte = 252 - 4 * lane + i;
        left = want - before;
      }
      before += x[i];
    }
    const int at = __ffsll((unsigned long long)__ballot(here)) - 1;
    prefix |= __shfl(byte, at) << shift;
    want = __shfl(left, at);
    wave_lds_sync();
  }
  int taken = 0, equal = 0;
  const uint64_t below = (1ull << lane) - 1;
  for (int j0 = 0; j0 < n; j0 += 64) {
    const int j = j0 + lane;
    const uint32_t k = j < n ? keys[j] : 0;
    const uint64_t same = __ballot(j < n && !all && k == prefix);
    const bool take = j < n && (all || k > prefix || (k == prefix && equal + __popcll(same & below) < (int)want));
    const uint64_t chosen = __ballot(take);
    if (take) list[taken + __popcll(chosen & below)] = j;
    equal += __popcll(same);
    taken += __popcll(chosen);
  }
  for (int e = taken + lane; e < n_select; e += 64) list[e] = -1;
}

// A workgroup takes up to eight groups of queries of one head: their means, then the products with the means of all resident
// blocks as 64-bit matrix instructions (A = 16 blocks x 4 columns straight from memory, B = 4 columns x the groups, held in
// registers), so that a mean is read once per workgroup, then a wave selects for a group.  grid: (tiles of groups * H) x candidates.
// Bound by the products for long windows, 2 G NB D in 64 bits, 16 columns however few groups there are: 37 groups of 128 columns over 1500
// blocks, 48 heads 64 us (products 28, selection 17, the queries' means); with a workgroup per group and vector
// products each read all means again, 235 us.
constexpr int kSelectThreads = 512;
constexpr int kSelectKeys = 12288;  // scores that a workgroup holds, 48 KB; a row's 8192 always fit
static_assert((ASTRO_MAX_SELECT_BLOCKS | 1) <= kSelectKeys, "one group's scores");
template <typename Elem, int D>
__global__ void __launch_bounds__(kSelectThreads) select_blocks_kernel(DevGeom g, const Elem* __restrict__ q, const float* __restrict__ means,
                                                                       int frame_blocks, int Nq, int group, int query_block, int n_select,
                                                                       int n_groups, int log_groups, int stride, StreamInts resident,
                                                                       int32_t* __restrict__ blocks) {
  constexpr int kWaves = kSelectThreads / 64, EPC = 16 / sizeof(Elem), CPR = D / EPC, kRows = 64 / CPR;
  typedef Elem Chunk __attribute__((ext_vector_type(EPC)));
  typedef double f64x4 __attribute__((ext_vector_type(4)));
  extern __shared__ uint32_t keys[];  // [groups of the workgroup][stride]
  __shared__ double part[kWaves][D];
  __shared__ float qbar[kWaves][D];
  __shared__ __attribute__((aligned(16))) uint32_t hist[kWaves][256];
  const int per_wg = 1 << log_groups, ways = kWaves >> log_groups;  // groups here, waves to a group's mean
  const int h = blockIdx.x % g.H, g0 = (int)(blockIdx.x / g.H) << log_groups, c = blockIdx.y, b = c / group;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = resident.v[b] * frame_blocks;
  const float* kbar = means + ((int64_t)b * g.H + h) * g.C * frame_blocks * D;
  {
    const int gi = g0 + wave / ways, q0 = gi * query_block, rows = gi < n_groups ? (Nq - q0 < query_block ? Nq - q0 : query_block) : 0;
    const Elem* from = q + (((int64_t)c * Nq + q0) * g.H + h) * D + lane % CPR * EPC;
    double sum[EPC] = {};
#pragma unroll 4
    for (int r = wave % ways * kRows + lane / CPR; r < rows; r += ways * kRows) {
      const Chunk x = *reinterpret_cast<const Chunk*>(from + (int64_t)r * g.H * D);
#pragma unroll
      for (int i = 0; i < EPC; ++i) sum[i] += (double)(float)x[i];
    }
#pragma unroll
    for (int d = CPR; d < 64; d <<= 1)
#pragma unroll
      for (int i = 0; i < EPC; ++i) sum[i] += __shfl_xor(sum[i], d);
    if (lane < CPR)
#pragma unroll
      for (int i = 0; i < EPC; ++i) part[wave][lane * EPC + i] = sum[i];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < per_wg * D; e += kSelectThreads) {
    const int i = e / D, d = e - i * D, q0 = (g0 + i) * query_block;
    double t = 0.;
    for (int w = 0; w < ways; ++w) t += part[i * ways + w][d];
    qbar[i][d] = (float)(t / (Nq - q0 < query_block ? Nq - q0 : query_block));
  }
  __syncthreads();
  const int i16 = lane & 15, k4 = lane >> 4;
  f32x4 qb[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) qb[s] = i16 < per_wg ? *reinterpret_cast<const f32x4*>(&qbar[i16][16 * s + 4 * k4]) : f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 x[D / 16], next[D / 16];  // the next tile's means are on their way under this one's products
  auto fetch = [&](int j0) __attribute__((always_inline)) {
    if (j0 >= n) return;
    const float* row = kbar + (int64_t)(j0 + i16 < n ? j0 + i16 : n - 1) * D + 4 * k4;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) next[s] = *reinterpret_cast<const f32x4*>(row + 16 * s);
  };
  fetch(wave * 16);
  for (int j0 = wave * 16; j0 < n; j0 += kWaves * 16) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) x[s] = next[s];
    fetch(j0 + kWaves * 16);
    f64x4 acc[2] = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e & 1] = __builtin_amdgcn_mfma_f64_16x16x4f64((double)x[s][e], (double)qb[s][e], acc[e & 1], 0, 0, 0);
    if (i16 < per_wg)
#pragma unroll
      for (int v = 0; v < 4; ++v)  // row 4 v + lane / 16 of the product
        if (j0 + 4 * v + k4 < n) keys[i16 * stride + j0 + 4 * v + k4] = ordered((float)(acc[0][v] + acc[1][v]));
  }
  __syncthreads();
  if (wave < per_wg && g0 + wave < n_groups)
    take_largest(keys + wave * stride, n, n_select, hist[wave], blocks + (((int64_t)c * g.H + h) * n_groups + g0 + wave) * n_select);
}

}  // namespace

hipError_t launch_block_means_f32(const DevGeom& g, const void* k, float* means, int key_block, int n_frames, const StreamInts& next_n,
                                  hipStream_t stream) {
  const int frame_blocks = blocks_of(g.T, key_block);
  const dim3 grid(n_frames * frame_blocks, g.H, g.B);
  ProfileScope prof("kv_block_means", stream);
  if (g.D == 128)
    block_means_kernel<128><<<grid, kThreads, 0, stream>>>(g, (const float*)k, means, key_block, frame_blocks, n_frames, next_n);
  else
    block_means_kernel<64><<<grid, kThreads, 0, stream>>>(g, (const float*)k, means, key_block, frame_blocks, n_frames, next_n);
  return hipGetLastError();
}

hipError_t launch_append_means_bf16(const DevGeom& g, const void* k, const void* v, void* k_cache, void* v_cache, float* means, int key_block,
                                    int n_frames, const StreamInts& first_frame, const StreamInts& next_n, hipStream_t stream) {
  const int frame_blocks = blocks_of(g.T, key_block);
  const dim3 grid(n_frames * frame_blocks, g.H, g.B);
  ProfileScope prof("kv_append_rope_means", stream);
  auto run = [&](auto d) {
    append_means_kernel<decltype(d)::value><<<grid, kThreads, 0, stream>>>(g, (const __bf16*)k, (const __bf16*)v, (__bf16*)k_cache,
                                                                          (__bf16*)v_cache, means, key_block, frame_blocks, n_frames,
                                                                          first_frame, next_n);
  };
  if (g.D == 128)
    run(std::integral_constant<int, 128>{});
  else
    run(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

hipError_t launch_select_blocks(const DevGeom& g, int dtype, const void* q, const float* means, int frame_blocks, int Nq, int group,
                                int query_block, int n_select, const StreamInts& resident, int32_t* blocks, hipStream_t stream) {
  int most = 1;
  for (int b = 0; b < g.B / group; ++b) most = resident.v[b] * frame_blocks > most ? resident.v[b] * frame_blocks : most;
  const int n_groups = blocks_of(Nq, query_block), stride = most | 1;  // (odd: the columns of a product go to different banks)
  // As many groups to a workgroup as there are waves to select for them, but no more than fill the chip, and their scores
  // have to fit the LDS.
  int log_groups = 3;
  while (log_groups > 0 && ((int64_t)blocks_of(n_groups, 1 << log_groups) * g.H * g.B < (g.n_cus * 3) / 4 || stride << log_groups > kSelectKeys)) --log_groups;
  const dim3 grid(blocks_of(n_groups, 1 << log_groups) * g.H, g.B);
  const size_t lds = ((size_t)stride << log_groups) * sizeof(uint32_t);
  ProfileScope prof("select_blocks", stream);
  auto run = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (dtype == ASTRO_BF16)
      select_blocks_kernel<__bf16, D><<<grid, kSelectThreads, lds, stream>>>(g, (const __bf16*)q, means, frame_blocks, Nq, group, query_block,
                                                                            n_select, n_groups, log_groups, stride, resident, blocks);
    else
      select_blocks_kernel<float, D><<<grid, kSelectThreads, lds, stream>>>(g, (const float*)q, means, frame_blocks, Nq, group, query_block,
                                                                           n_select, n_groups, log_groups, stride, resident, blocks);
  };
  if (g.D == 128)
    run(std::integral_constant<int, 128>{});
  else
    run(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace astro

// Queries and chunk keys of a call over selected blocks, rotated in fp32 and laid out head-major, as two bf16 halves each:
//   q~ = R(phi) q * log2(e) / sqrt(D) = q_hi + q_lo,  k~ = R(phi) k = k_hi + k_lo  (each pair keeps 16 bits)
// and, for few rows, what they leave of all 24.  Bound by its bytes, two tensors in and four out.
#include "kernels.hpp"
#include "select_walk.hpp"

namespace astro {
namespace {

constexpr int kThreads = 256;

// grid: x = n_frames * gh (frame in chunk, row), y = head, z = candidate
template <int D, bool kFine>
__global__ void __launch_bounds__(kThreads) select_stage_kernel(DevGeom g, const __bf16* __restrict__ q, const __bf16* __restrict__ k,
                                                                SelectStaged to, int n_frames, StreamInts first_frame, float q_scale) {
  constexpr int CPR = D / 8;
  __shared__ float2 tab[D / 2];  // of the frame's and the row's pairs
  const int fi = blockIdx.x / g.gh, row = blockIdx.x - fi * g.gh, h = blockIdx.y, b = blockIdx.z, t = threadIdx.x;
  const bool rope = g.n_t + g.n_h + g.n_w != 0;
  const int nb = g.n_t + g.n_h;
  if (rope) {
    if (t < g.n_t) {
      double s, c;
      sincos((double)(first_frame.v[b] + fi) * g.inv_freq_t[t], &s, &c);
      tab[t] = make_float2((float)c, (float)s);
      if (row == 0 && h == 0) to.tab_t[((int64_t)b * n_frames + fi) * g.n_t + t] = tab[t];
    } else if (t < nb) {
      tab[t] = g.tab_h[row * g.n_h + (t - g.n_t)];
    }
    __syncthreads();
  }
  const int64_t n_q = (int64_t)n_frames * g.T, tok0 = (int64_t)fi * g.T + (int64_t)row * g.gw;
  for (int i = t; i < g.gw * CPR; i += kThreads) {
    const int w = i / CPR, c = i % CPR;
    const int64_t in = (((int64_t)b * n_q + tok0 + w) * g.H + h) * D + c * 8, out = (((int64_t)b * g.H + h) * n_q + tok0 + w) * D + c * 8;
    const bf16x8 x[2] = {*reinterpret_cast<const bf16x8*>(q + in), *reinterpret_cast<const bf16x8*>(k + in)};
    bf16x8 hi[2], lo[2], rest[2];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int pair = c * 4 + v;
      const float2 cs = !rope ? make_float2(1.f, 0.f) : pair < nb ? tab[pair] : g.tab_w[w * g.n_w + (pair - nb)];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float a = (float)x[m][2 * v], e = (float)x[m][2 * v + 1], scale = m == 0 ? q_scale : 1.f;
        const f32x2 turned = rope ? f32x2{a * cs.x - e * cs.y, a * cs.y + e * cs.x} : f32x2{a, e};  // (without: not through a product with 0)
        const f32x2 y = turned * scale;
        const HalfPairs r = halves_of_any(y);
        if constexpr (kFine) {
#pragma unroll
          for (int j = 0; j < 2; ++j) rest[m][2 * v + j] = (__bf16)(__builtin_isfinite((float)r.hi[j]) ? y[j] - (float)r.hi[j] - (float)r.lo[j] : 0.f);
        }
        hi[m][2 * v] = r.hi[0], hi[m][2 * v + 1] = r.hi[1];
        lo[m][2 * v] = r.lo[0], lo[m][2 * v + 1] = r.lo[1];
      }
    }
    *reinterpret_cast<bf16x8*>((__bf16*)to.q_hi + out) = hi[0];
    *reinterpret_cast<bf16x8*>((__bf16*)to.q_lo + out) = lo[0];
    *reinterpret_cast<bf16x8*>((__bf16*)to.k_hi + out) = hi[1];
    *reinterpret_cast<bf16x8*>((__bf16*)to.k_lo + out) = lo[1];
    if constexpr (kFine) {
      *reinterpret_cast<bf16x8*>((__bf16*)to.q_rest + out) = rest[0];
      *reinterpret_cast<bf16x8*>((__bf16*)to.k_rest + out) = rest[1];
    }
  }
}

}  // namespace

hipError_t launch_select_stage(const DevGeom& g, const void* q, const void* k, const SelectStaged& to, int n_frames,
                               const StreamInts& first_frame, float q_scale, hipStream_t stream) {
  const dim3 grid(n_frames * g.gh, g.H, g.B);
  ProfileScope prof("select_stage", stream);
  auto run = [&](auto d, auto fine) {
    select_stage_kernel<decltype(d)::value, decltype(fine)::value>
        <<<grid, kThreads, 0, stream>>>(g, (const __bf16*)q, (const __bf16*)k, to, n_frames, first_frame, q_scale);
  };
  auto of_width = [&](auto d) { to.q_rest ? run(d, std::true_type{}) : run(d, std::false_type{}); };
  if (g.D == 128)
    of_width(std::integral_constant<int, 128>{});
  else
    of_width(std::integral_constant<int, 64>{});
  return hipGetLastError();
}

}  // namespace astro

// Buffers of the calls over selected blocks that share bytes with one another or with what the cache keeps: every pair of them that would be
// written and read, or written twice, is refused and launches nothing.
#include <cstdio>
#include <string>
#include <vector>

#include "hip_stubs.hpp"

namespace {

constexpr size_t kPart = 1 << 20;
char* memory() {
  static std::vector<char> m(40 * kPart + 256);
  return (char*)(((uintptr_t)m.data() + 255) & ~(uintptr_t)255);
}
int wrong = 0;
void expect(const std::string& what, int got, int want, bool launches_want) {
  if (got == want && (launches > 0) == launches_want) return;
  std::printf("%s: %d instead of %d, %d launches\n", what.c_str(), got, want, launches);
  ++wrong;
}

void run(int dtype, bool moving) {
  enum { K, V, SINK, MEANS, Q, KC, VC, OUT, LSE, DOUT, LISTS, DQ, DK, DV, SPACE, N };
  const char* names[] = {"k_storage", "v_storage", "k_sink_storage", "means", "q", "k_chunk", "v_chunk", "out", "lse", "dout", "blocks", "dq", "dk_chunk",
                         "dv_chunk", "workspace"};
  char* at[N];
  for (int i = 0; i < N; ++i) at[i] = memory() + 2 * i * kPart;
  astro_kvcache_desc_t d{};
  d.batch = 2, d.heads = 2, d.head_dim = 64, d.grid_h = d.grid_w = 4, d.capacity_frames = 4, d.sink_frames = 1, d.max_chunk_frames = 2;
  d.rope_pairs_t = 12, d.rope_pairs_h = d.rope_pairs_w = 10, d.rope_base = 10000., d.dtype = dtype;
  d.flags = moving ? ASTRO_FLAG_WINDOW_RELATIVE : 0;
  d.k_storage = at[K], d.v_storage = at[V], d.k_sink_storage = moving ? at[SINK] : nullptr;
  astro_kvcache_t* c = nullptr;
  if (astro_kvcache_create(&d, &c) != ASTRO_OK) ++wrong;
  for (int i : {K, V, SINK})
    if (i != SINK || moving) {
      launches = 0;
      expect(std::string("means over ") + names[i], astro_kvcache_keep_means(c, 32, (float*)(at[i] + 64)), ASTRO_ERR_INVALID_ARG, false);
    }
  expect("means", astro_kvcache_keep_means(c, 64, (float*)at[MEANS]), ASTRO_OK, false);
  expect("means where they were", astro_kvcache_keep_means(c, 32, (float*)at[MEANS]), ASTRO_OK, false);

  size_t fwd_bytes = 0, bwd_bytes = 0;
  if (astro_select_attn_workspace_bytes(c, 1, 1, &fwd_bytes, &bwd_bytes) != ASTRO_OK || bwd_bytes > kPart) ++wrong;
  auto select = [&](char** a) { return astro_select_blocks(c, a[Q], 1, 1, 64, 3, (int32_t*)a[LISTS], nullptr); };
  auto fwd = [&](char** a) {
    return astro_select_attn_fwd(c, a[Q], a[KC], a[VC], 1, 1, (const int32_t*)a[LISTS], 64, 3, a[OUT], (float*)a[LSE], a[SPACE], fwd_bytes, nullptr);
  };
  auto bwd = [&](char** a) {
    return astro_select_attn_bwd(c, a[Q], a[KC], a[VC], a[OUT], (const float*)a[LSE], a[DOUT], 1, 1, (const int32_t*)a[LISTS], 64, 3, (float*)a[DQ],
                                 (float*)a[DK], (float*)a[DV], a[SPACE], bwd_bytes, nullptr);
  };
  auto every = [&](const char* call, auto f, std::vector<int> in, std::vector<int> out) {
    launches = 0;
    expect(call, f(at), ASTRO_OK, true);
    std::vector<int> all = in;
    all.insert(all.end(), out.begin(), out.end());
    for (int i : {K, V, MEANS}) all.push_back(i);
    if (moving) all.push_back(SINK);
    for (int o : out)
      for (int i : all) {
        if (i == o) continue;
        char* a[N];
        std::copy(at, at + N, a);
        a[o] = at[i];
        launches = 0;
        expect(std::string(call) + ": " + names[o] + " over " + names[i], f(a), ASTRO_ERR_INVALID_ARG, false);
      }
  };
  every("select", select, {Q}, {LISTS});
  every("forward", fwd, {Q, KC, VC, LISTS}, {OUT, LSE, SPACE});
  every("backward", bwd, {Q, KC, VC, OUT, LSE, DOUT, LISTS}, {DQ, DK, DV, SPACE});
  if (astro_kvcache_destroy(c) != ASTRO_OK) ++wrong;
}

}  // namespace

int main() {
  for (int dtype : {ASTRO_BF16, ASTRO_F32})
    for (bool moving : {false, true}) run(dtype, moving);
  if (!wrong) std::puts("ok");
  return wrong != 0;
}

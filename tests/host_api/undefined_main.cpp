// A handle whose ring rows no longer match its tables, after an append or a fork whose launch failed: every call but the tables', the reset of all
// streams and destroy answers ASTRO_ERR_BAD_STATE and launches nothing.
#include <cstdio>
#include <vector>

#include "hip_stubs.hpp"

namespace {

int wrong = 0;
void expect(const char* what, int got, int want) {
  if (got == want) return;
  std::printf("%s: %d instead of %d\n", what, got, want);
  ++wrong;
}

astro_kvcache_t* make(std::vector<char>& memory, int dtype) {
  memory.assign(1 << 20, 0);
  char* at = (char*)(((uintptr_t)memory.data() + 255) & ~(uintptr_t)255);
  astro_kvcache_desc_t d{};
  d.batch = 2, d.heads = 2, d.head_dim = 64, d.grid_h = d.grid_w = 4, d.capacity_frames = 4, d.sink_frames = 1, d.max_chunk_frames = 2;
  d.rope_pairs_t = 12, d.rope_pairs_h = d.rope_pairs_w = 10, d.rope_base = 10000., d.dtype = dtype;
  d.k_storage = at, d.v_storage = at + (1 << 18);
  astro_kvcache_t* c = nullptr;
  expect("create", astro_kvcache_create(&d, &c), ASTRO_OK);
  expect("means", astro_kvcache_keep_means(c, 32, (float*)(at + (1 << 19))), ASTRO_OK);
  return c;
}

void run(int dtype, bool by_fork) {
  std::vector<char> m1, m2;
  astro_kvcache_t *c = make(m1, dtype), *other = make(m2, dtype);
  alignas(256) static char x[1 << 16];
  const int32_t source[2] = {1, 0};
  expect("append", astro_kvcache_append(other, x, x, 1, nullptr), ASTRO_OK);
  launches_fail = true;
  expect("failing", by_fork ? astro_kvcache_fork(c, other, source, nullptr) : astro_kvcache_append(c, x, x, 1, nullptr), ASTRO_ERR_HIP);
  launches_fail = false;
  launches = 0;
  int32_t next[2];
  expect("tables", astro_kvcache_tables(c, nullptr, nullptr, next), ASTRO_OK);
  expect("tables", next[0] + next[1], 0);
  const int bad = ASTRO_ERR_BAD_STATE;
  float* f = (float*)x;
  int32_t* i = (int32_t*)x;
  expect("append", astro_kvcache_append(c, x, x, 1, nullptr), bad);
  expect("fork to", astro_kvcache_fork(c, other, source, nullptr), bad);
  expect("fork from", astro_kvcache_fork(other, c, source, nullptr), bad);
  expect("reset of one", astro_kvcache_reset(c, 0, 0), bad);
  expect("means", astro_kvcache_keep_means(c, 64, (float*)(m1.data() + (1 << 20) - (1 << 18) + 256)), bad);
  expect("select", astro_select_blocks(c, x, 1, 1, 64, 1, i, nullptr), bad);
  expect("forward", astro_select_attn_fwd(c, x, x, x, 1, 1, i, 64, 1, x, f, x, sizeof x, nullptr), bad);
  expect("backward", astro_select_attn_bwd(c, x, x, x, x, f, x, 1, 1, i, 64, 1, f, f, f, x, sizeof x, nullptr), bad);
  expect("launches", launches, 0);
  expect("reset", astro_kvcache_reset(c, -1, 5), ASTRO_OK);
  expect("means again", astro_kvcache_keep_means(c, 32, (float*)(((uintptr_t)m1.data() + 255 & ~(uintptr_t)255) + (1 << 19))), ASTRO_OK);
  expect("append again", astro_kvcache_append(c, x, x, 1, nullptr), ASTRO_OK);
  expect("destroy", astro_kvcache_destroy(c), ASTRO_OK);
  expect("destroy", astro_kvcache_destroy(other), ASTRO_OK);
}

}  // namespace

int main() {
  for (int dtype : {ASTRO_BF16, ASTRO_F32})
    for (bool by_fork : {false, true}) run(dtype, by_fork);
  if (!wrong) std::puts("ok");
  return wrong != 0;
}

"""Caches that are dropped, at once or by the garbage collector, while a graph is captured: the capture goes on."""
import gc

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_a_cycle", [False, True])
def test_a_cache_dropped_during_a_capture(in_a_cycle):
    import torch
    import paper_2603_17051_amd as A
    make = lambda: A.astro_kvcache_create(1, 2, 64, 8, 8, 4, 0, 1, (12, 10, 10), key_block=32)
    kept, dropped = make(), make()
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    q, k, v = (torch.randn((1, 64, 2, 64), generator=gen, device="cuda:0").to(torch.bfloat16) for _ in range(3))
    A.astro_kvcache_append(kept, k, v, 1)
    blocks = A.astro_select_blocks(kept, q, 1, 2, 64)
    want = A.astro_select_attn_fwd(kept, q, k, v, blocks, 1, 64)
    torch.cuda.synchronize()
    if in_a_cycle:
        dropped.itself = dropped
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        del dropped
        gc.collect()
        got = A.astro_select_attn_fwd(kept, q, k, v, blocks, 1, 64)
    for _ in range(3):
        got[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    make()  # what was dropped is given back by now
    assert not A.binding._dropped

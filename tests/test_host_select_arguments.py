"""Arguments of the calls over selected blocks that 32 bits do not hold: refused, not taken for others."""
import pytest

import paper_2603_17051_amd as A
from paper_2603_17051_amd import binding

SIZES = (2, 2, 64, 4, 4, 5, 1, 2, (12, 10, 10))


@pytest.mark.parametrize("off", [1 << 32, -(1 << 32), 1 << 64])
def test_sizes_beyond_32_bits_are_refused(off):
    cache = A.astro_kvcache_create(*SIZES, host_only=True, key_block=32)
    for call in (lambda: A.astro_kvcache_create(*SIZES, host_only=True, key_block=32 + off), lambda: A.astro_kvcache_mean_bytes(A.make_desc(*SIZES), 32 + off),
                 lambda: A.astro_select_attn_workspace_bytes(cache, 1 + off), lambda: A.astro_select_attn_workspace_bytes(cache, 1, 1 + off)):
        with pytest.raises(A.AstroError) as e:
            call()
        assert e.value.code == binding.ASTRO_ERR_INVALID_ARG


@pytest.mark.parametrize("frames,group", [(3, 1), (1 << 40, 1), (1, 33), (2, 1 << 40), (0, 1), (1, 0), (-1, 1), (1, -1)])
def test_nothing_is_allocated_for_a_call_that_is_refused(frames, group, monkeypatch):
    import torch
    cache = A.astro_kvcache_create(*SIZES, host_only=True, key_block=32)
    q = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("allocated"))
    with pytest.raises((ValueError, A.AstroError)):
        A.astro_select_blocks(cache, q, frames, 2, 64, group)

"""Entries of a fork's source that 32 bits do not hold: refused, not taken for others."""
import pytest

import paper_2603_17051_amd as A
from paper_2603_17051_amd import binding


def make(batch):
    return A.astro_kvcache_create(batch, 2, 64, 4, 4, 5, 1, 2, (12, 10, 10), host_only=True)


@pytest.mark.parametrize("bad", [1 << 32, (1 << 32) - 1, (1 << 32) + 1, -(1 << 32), -(1 << 32) + 1, 1 << 31, 1 << 63, 1 << 64, 1 << 100, -(1 << 100), 3, -2])
@pytest.mark.parametrize("as_tuple", [False, True])
def test_entries_out_of_range_are_refused(bad, as_tuple):
    src, dst = make(3), make(2)
    A.astro_kvcache_reset(src, -1, 7)
    A.astro_kvcache_append(src, n_frames=2)
    before = A.astro_kvcache_tables(dst)
    source = (0, bad) if as_tuple else [0, bad]
    with pytest.raises(A.AstroError) as e:
        A.astro_kvcache_fork(dst, src, source)
    assert e.value.code == binding.ASTRO_ERR_INVALID_ARG and A.astro_kvcache_tables(dst) == before
    A.astro_kvcache_fork(dst, src, (2, -1))
    assert A.astro_kvcache_tables(dst)[2] == [2, 0]

"""Attention over selected blocks where keys that are attended to are not finite: what the definition gives, with one key range and with several."""
import numpy as np
import pytest

from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu


def pair(head_dim, dtype, listed, **kw):
    """128 queries of two frames of 64 in two groups; lists of `listed` blocks of 32 rows, of which block 3 is the first group's alone.
    100 blocks are walked in eight ranges, 3 in one or two."""
    p = Pair(heads=2, head_dim=head_dim, grid=(8, 8), capacity=60, appended=(60,), frames=2, dtype=dtype, rope=False, seed=head_dim + listed, **kw)
    lists = np.empty((1, 2, 2, listed), dtype=np.int32)
    lists[:, :, 0] = np.arange(1, listed + 1)
    lists[:, :, 1] = np.arange(4, listed + 4)
    return p, lists


def rows(p, which):
    return (p.cache.k_storage if which == "k" else p.cache.v_storage).view(p.cache.torch_dtype).view(p.heads, -1, p.head_dim)


def results(p, lists, chunk):
    out, lse = p.A.astro_select_attn_fwd(p.cache, *chunk[:3], dev_lists(lists), 2, 64)
    return [out, lse, *p.A.astro_select_attn_bwd(p.cache, *chunk[:3], out, lse, chunk[3], dev_lists(lists), 2, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("listed", [3, 100])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_a_key_that_is_not_a_number(head_dim, listed, dtype):
    """A softmax over it is none: output, log-sum-exp and gradients say so, for the queries that list it alone."""
    import torch
    p, lists = pair(head_dim, dtype, listed)
    chunk = [p.dev(x) for x in p.chunk()]
    want = results(p, lists, chunk)
    rows(p, "k")[:, 3 * 32 + 7, 5] = float("nan")
    got = results(p, lists, chunk)
    for i, tokens in ((0, 1), (1, 2), (2, 1)):  # out, lse, dq
        first, second = got[i].narrow(tokens, 0, 64), got[i].narrow(tokens, 64, 64)
        assert first.isnan().all(), i
        assert torch.equal(second, want[i].narrow(tokens, 64, 64)) and second.isfinite().all(), i
    assert got[3].isnan().all() and got[4].isnan().all()  # every chunk key is a key of those queries

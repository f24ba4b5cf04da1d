"""Outputs over selected blocks where all values are the same: a mean of them is that value, whatever the weights, to the last bit."""
import pytest

from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim,query_block", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("size,listed", [(dict(grid=(1, 1), appended=(0,), heads=3), 1),  # a single key
                                         (dict(grid=(1, 1), appended=(0,), heads=8, batch=16), 1), (dict(grid=(9, 7), appended=(4,), frames=2, block_frames=1), 7),
                                         (dict(grid=(8, 8), capacity=40, appended=(40,)), 70)])  # several ranges
def test_the_mean_of_equal_values(size, listed, head_dim, query_block, dtype):
    """Weights are probabilities rounded to bf16 over the sum of the rounded ones, so they sum to 1 within fp32: sums tile after tile, of at most 80 tiles
    of 32 keys, lose (80 + 32) 2^-24 twice, far from the half step of 2^-8 that a bf16 output is rounded by.  (Over the sum of those before, one
    key's value came out a step off.)  The fp32 path adds key after key: N keys lose up to N 2^-24 in the sum of weights and, with
    the product's rounding, twice that in that of values, N < 2400: below 2^-11."""
    import torch
    p = Pair(head_dim=head_dim, dtype=dtype, key_block=32, seed=listed, **size)
    q, k, v, _ = (p.dev(x) for x in p.chunk())
    value = v[:, :1].clone()  # of each stream and head
    v[:] = value
    p.cache.v_storage.view(p.cache.torch_dtype).view(p.batch, p.heads, -1, head_dim)[:] = value.permute(0, 2, 1, 3)
    out, _ = p.A.astro_select_attn_fwd(p.cache, q, k, v, dev_lists(p.lists(listed, query_block)), p.frames, query_block)
    if dtype == "bf16":
        assert torch.equal(out, value.expand_as(out))
    else:
        assert ((out - value).abs() <= 2.0**-11 * value.abs()).all()

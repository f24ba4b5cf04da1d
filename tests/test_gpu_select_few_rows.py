"""Gradients and log-sum-exps over selected blocks where there are few rows: one probability may make most of a gradient, so they are formed from
more than 16 bits, as far as the rule of launches goes."""
import numpy as np
import pytest

from helpers import host_f64
from oracle import selected_blocks as sb
from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu

# (rows of all heads: 2, 4, 48, 48, 500)
SIZES = [dict(grid=(2, 1), heads=1), dict(grid=(1, 1), heads=2, batch=2), dict(grid=(3, 4), frames=2, heads=1, batch=2), dict(grid=(3, 4), frames=2, heads=2, block_frames=1),
         dict(grid=(10, 25), frames=1, heads=2)]


@pytest.mark.parametrize("head_dim,query_block", [(64, 64), (64, 128), (128, 64), (128, 128)])
@pytest.mark.parametrize("size", SIZES)
def test_gradients_of_few_rows(size, head_dim, query_block):
    """Probabilities from 24-bit scores; P and dS enter their products as two halves, which lose 2^-17 of them at most, and a half-lost vector
    operand (a rotated query or key) another 2^-17 of its own at most, in other directions: below sqrt(2) 2^-17 = 1.08e-5 however the
    gradient is made up; fp32 sums are 2^-22 of it."""
    worst = np.zeros(3)
    for seed in range(25):
        p = Pair(head_dim=head_dim, capacity=6, appended=(6,), key_block=32, seed=seed, **size)
        lists = p.lists(4, query_block)
        p.oracle.cache_rounding = True
        q, k, v, do = p.chunk()
        dev = [p.dev(x) for x in (q, k, v, do)]
        out, lse = p.A.astro_select_attn_fwd(p.cache, *dev[:3], dev_lists(lists), p.frames, query_block)
        grads = p.A.astro_select_attn_bwd(p.cache, *dev[:3], out, lse, dev[3], dev_lists(lists), p.frames, query_block)
        ref = sb.attend(p.oracle, *(p.wide(x) for x in (q, k, v)), lists, p.frames, 32, query_block, dout=p.wide(do), given=(host_f64(out), host_f64(lse)))
        worst = np.maximum(worst, [np.linalg.norm(host_f64(a) - b) / np.linalg.norm(b) for a, b in zip(grads, ref[2:])])
    assert (worst < np.sqrt(2) * 2.0**-17).all(), worst


@pytest.mark.parametrize("head_dim,query_block", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_log_sum_exps_of_single_keys(head_dim, query_block):
    """No key but the query's own: a score, near 0 now and then.  Operands of 24 bits lose 2^-24 of each product, fp32 sums of 128 of them and of
    256 MFMA terms 2^-20 of the sum of their sizes at most."""
    for seed in range(10):
        p = Pair(grid=(1, 1), heads=8, head_dim=head_dim, capacity=4, appended=(0,), key_block=32, seed=seed)
        lists = p.lists(2, query_block)
        q, k, v, _ = p.chunk()
        _, lse = p.A.astro_select_attn_fwd(p.cache, *(p.dev(x) for x in (q, k, v)), dev_lists(lists), 1, query_block)
        q, k = p.wide(q)[0, 0], p.wide(k)[0, 0]
        score, size = (q * k).sum(1) / np.sqrt(head_dim), (np.abs(q) @ np.abs(k).T).diagonal() / np.sqrt(head_dim)
        assert (np.abs(host_f64(lse)[0, :, 0] - score) < 2.0**-20 * size).all()

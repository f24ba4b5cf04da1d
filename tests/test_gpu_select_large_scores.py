"""The forward over selected blocks at scores of several hundred, against the definition at unrounded queries and chunk keys."""
import numpy as np
import pytest

from helpers import host_f64
from oracle import rope_rotate
from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu

FACTORS = (3.0, 60.0, 0.0, 40.0, 1.0, 80.0)  # of the keys of block after block: references move up, and stay


@pytest.mark.parametrize("listed", [2, 36])  # walked in one range, and in several
@pytest.mark.parametrize("query_block", [64, 128])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_large_scores(head_dim, query_block, listed):
    """A half loses 2^-8 of its operand, two lose 2^-16; with both operands' losses, the product of small halves left out (2^-16) and fp32 sums of
    128 products (2^-17 at worst) a score is off by at most 2^-14 A, A = sum |q k| / sqrt(D).  So is the log-sum-exp, which is a mean of the scores plus
    what does not depend on them, with A of its row's largest.  In the mean the errors of D products add up as roots do: below 2^-17 A.  (Operands rounded
    once: 2^-8 A / sqrt(D), ten times that.)  Outputs: probabilities off by twice the score's and by half a step of 2^-8, the output by
    another."""
    import torch
    p = Pair(heads=2, head_dim=head_dim, grid=(8, 8), capacity=40, appended=(40,), frames=2, key_block=64, seed=head_dim + listed)
    keys = p.cache.k_storage.view(torch.bfloat16).view(2, 40, 64, head_dim)
    for s in range(40):
        keys[:, s] *= FACTORS[s % len(FACTORS)]
    q, k, v, _ = (p.dev(x) for x in p.chunk())
    lists = np.broadcast_to(np.arange(listed, dtype=np.int32), (1, 2, p.groups(query_block), listed))
    out, lse = p.A.astro_select_attn_fwd(p.cache, q, k, v, dev_lists(lists), 2, query_block)
    phi, squares = p.oracle._chunk_phi(0, 2), []
    for h in range(2):
        turned = lambda x: rope_rotate(host_f64(x)[0, :, h:h + 1], phi)[:, 0]
        ring = lambda x: host_f64(x.view(torch.bfloat16).view(2, 40 * 64, head_dim)[h, :listed * 64])
        kt, vt = np.concatenate([ring(p.cache.k_storage), turned(k)]), np.concatenate([ring(p.cache.v_storage), host_f64(v)[0, :, h]])
        s, most = turned(q) @ kt.T / np.sqrt(head_dim), np.abs(turned(q)) @ np.abs(kt).T / np.sqrt(head_dim)
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
        z = e.sum(1, keepdims=True)
        ref, ref_lse, bound = e @ vt / z, (m + np.log(z))[:, 0], most.max(1)
        err = np.abs(host_f64(lse)[0, h] - ref_lse)
        assert s.max() > 150 and (err < 2.0**-14 * bound).all(), (err / bound).max()
        squares.append([(err**2).mean(), (bound**2).mean()])
        off, mass = np.abs(host_f64(out)[0, :, h] - ref), e @ np.abs(vt) / z
        assert (off <= (2.0**-8 + 2.0**-13 * bound[:, None]) * mass + 2.0**-8 * np.abs(ref)).all()
    err, bound = np.sum(squares, axis=0)
    assert np.sqrt(err) < 2.0**-17 * np.sqrt(bound), np.sqrt(err / bound) * 2**17

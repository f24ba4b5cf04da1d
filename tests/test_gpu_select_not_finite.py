"""Attention over selected blocks where keys that are attended to are not finite: what the definition gives, with one key range and with several."""
import numpy as np
import pytest

from helpers import assert_bf16_close, assert_f32_close, host_f64
from oracle import selected_blocks as sb
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


def close(p, got, ref, what):
    (assert_bf16_close if p.dtype == "bf16" else assert_f32_close)(host_f64(got), ref, what)


def oracle(p, lists, chunk, given=None):
    with np.errstate(invalid="ignore"):
        q, k, v, do = (host_f64(x) for x in chunk)
        return sb.attend(p.oracle, q, k, v, lists, 2, p.key_block, 64, dout=do, given=given)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("where", ["chunk", "ring"])
@pytest.mark.parametrize("block_frames", [0, 1])
@pytest.mark.parametrize("listed", [3, 100])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_an_infinite_key_of_weight_zero(head_dim, listed, block_frames, where, dtype):
    """All scores of it are -inf: everything is as without it, but for the column of dQ that is 0 * inf, of queries that attend to it."""
    import torch
    p, lists = pair(head_dim, dtype, listed, block_frames=block_frames)
    chunk = [p.dev(x) for x in p.chunk()]
    chunk[0][..., 7] = chunk[0][..., 7].abs() + 0.5
    want = results(p, lists, chunk)
    if where == "ring":  # the first group's
        rows(p, "k")[:, 3 * 32 + 7, 7] = -float("inf")
        p.oracle.history[0][1][0][39, :, 7] = -np.inf
        sees = slice(0, 64)
    else:
        chunk[1][:, 70, :, 7] = -float("inf")
        sees = slice(64 if block_frames else 0, 128)
    got, ref = results(p, lists, chunk), oracle(p, lists, chunk)
    for what, a, b in zip(("out", "lse"), got, ref):
        close(p, a, b, what)
    close(p, got[3], ref[3], "dk")
    close(p, got[4], ref[4], "dv")
    assert got[2][:, sees, :, 7].isnan().all()
    for a in (got[2], want[2]):
        a[:, sees, :, 7] = 0
    others = [i for i in range(128) if not sees.start <= i < sees.stop]
    assert torch.equal(got[2][:, others], want[2][:, others]) and got[2].isfinite().all()
    if where == "chunk":  # without a key that had a weight, the others' grow: only those queries that do not see it keep theirs
        assert (got[4][:, 70] == 0).all()
    ref[2][..., 7] = 0
    got[2][..., 7] = 0
    close(p, got[2], ref[2], "dq")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("listed", [3, 100])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_an_infinite_key_of_either_sign(head_dim, listed, dtype):
    """Scores of +inf make a softmax that is no number, those of -inf of other queries leave theirs."""
    p, lists = pair(head_dim, dtype, listed)
    chunk = [p.dev(x) for x in p.chunk()]
    chunk[0][..., 7] = chunk[0][..., 7].sign() * (chunk[0][..., 7].abs() + 0.25)
    chunk[1][:, 70, :, 7] = float("inf")
    out, lse = p.A.astro_select_attn_fwd(p.cache, *chunk[:3], dev_lists(lists), 2, 64)
    ref = oracle(p, lists, chunk)
    up = chunk[0][0, :, :, 7] > 0  # [tokens, heads]
    assert 64 < int(up.sum()) < 192
    assert out[0][up].isnan().all() and out[0][~up].isfinite().all() and lse[0].T[up].isnan().all() and lse[0].T[~up].isfinite().all()
    down = ~up.cpu().numpy()
    close(p, out[0][~up], ref[0][0][down], "out")
    close(p, lse[0].T[~up], ref[1][0].T[down], "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_an_infinite_output_gradient(head_dim, dtype):
    """dV = P^T dO: infinite in its column, the others and the other queries' dQ as they were."""
    import torch
    p, lists = pair(head_dim, dtype, 3)
    chunk = [p.dev(x) for x in p.chunk()]
    want = results(p, lists, chunk)
    chunk[3][:, 9, :, 3] = -float("inf")
    got = results(p, lists, chunk)
    assert (got[4][..., 3] == -float("inf")).all()
    others = [i for i in range(128) if i != 9]
    assert torch.equal(got[2][:, others], want[2][:, others]) and not got[2][:, 9].isfinite().any()
    got[4][..., 3], want[4][..., 3] = 0, 0
    close(p, got[4], host_f64(want[4]), "dv")

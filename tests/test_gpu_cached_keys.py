"""The keys that a bf16 cache keeps, bit for bit: the definition's rotation, rounded to 32 bits and then to bf16, whether an append
stores them, one that also keeps block means, or sinks that move on; and the fp32 results over selected blocks of such keys."""
import numpy as np
import pytest

from helpers import host_f64
from oracle import rope_angles, rope_rotate
from oracle import selected_blocks as sb
from oracle.rolling_attention import round_to_bf16
from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu


def rounded_keys(p, b, slot):
    """[T, H, D]: what slot `slot` of stream b has to hold, None where there is no frame"""
    n = p.oracle.tables[b].slot_number[slot]
    if n is None:
        return None
    o, frame = p.oracle, p.oracle.start[b] + n
    if o.window_relative and n < o.S:
        frame += max(0, len(o.history[b]) - o.C)
    phi = rope_angles(frame, o.gh, o.gw, o.pairs, o.base)
    return round_to_bf16(rope_rotate(np.asarray(o.history[b][n][0], dtype=np.float64), phi))


@pytest.mark.parametrize("key_block", [0, 32, 128])
@pytest.mark.parametrize("window_relative", [False, True])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_cached_keys_are_the_rounded_rotation(head_dim, window_relative, key_block):
    """1.2 million keys' elements and more each; in 32 bits, with tables rounded to 32, 10 to 30 of them are off by a step."""
    import torch
    p = Pair(batch=2, heads=4, head_dim=head_dim, grid=(23, 17), capacity=6, sinks=2, frames=2, key_block=key_block, appended=(9, 4), starts=[3, 4999],
             seed=head_dim + key_block, window_relative=window_relative)
    p.append(2)
    keys = host_f64(p.cache.k_storage.view(torch.bfloat16).view(2, 4, 6, p.tokens, head_dim))
    seen = 0
    for b in range(2):
        for slot in range(6):
            want = rounded_keys(p, b, slot)
            if want is not None:
                assert (keys[b, :, slot].transpose(1, 0, 2) == want).all(), (b, slot, (keys[b, :, slot].transpose(1, 0, 2) != want).sum())
                seen += want.size
    assert seen > 1.1e6 * head_dim / 64


@pytest.mark.parametrize("head_dim,query_block,key_block", [(64, 64, 32), (64, 128, 64), (128, 64, 128), (128, 128, 32)])
def test_fp32_results_over_appended_keys_keep_16_bits(head_dim, query_block, key_block):
    """Log-sum-exps and gradients over listed blocks of keys that the appends rotated, at the definition's keys rounded to bf16.  The
    bound is that of the operands: halves lose 2^-18 of one and the product of the small halves is left out, 2^-18 again, so that up to three such
    make a score's error and one a gradient's operand; 2^-16 leaves room for fp32 sums.  No element is further off than 32 times that bound:
    the largest of a million normal errors is 5 times their root mean square."""
    p = Pair(batch=2, heads=2, head_dim=head_dim, grid=(23, 17), capacity=9, sinks=1, frames=2, key_block=key_block, appended=(12, 6), starts=[5, 700], block_frames=1)
    lists = p.lists(9 * (-(-p.tokens // key_block)) // 2, query_block)
    p.oracle.cache_rounding = True
    q, k, v, do = p.chunk()
    dev = [p.dev(x) for x in (q, k, v, do)]
    out, lse = p.A.astro_select_attn_fwd(p.cache, *dev[:3], dev_lists(lists), 2, query_block)
    got = (lse, *p.A.astro_select_attn_bwd(p.cache, *dev[:3], out, lse, dev[3], dev_lists(lists), 2, query_block))
    ref = sb.attend(p.oracle, *(p.wide(x) for x in (q, k, v)), lists, 2, key_block, query_block, dout=p.wide(do), given=(host_f64(out), host_f64(lse)))
    for what, a, b in zip(("lse", "dq", "dk", "dv"), got, ref[1:]):
        e, rms = host_f64(a) - b, np.sqrt((b**2).mean())
        assert np.sqrt((e**2).mean()) < 2.0**-16 * rms, (what, np.sqrt((e**2).mean()) / rms)
        far = (np.abs(e) / np.maximum(rms, np.abs(b))).max()
        assert far < 2.0**-11, (what, far)

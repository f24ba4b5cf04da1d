"""Calls over selected blocks that are given no workspace: at the same time on several streams, and in several graphs."""
import pytest

from select_helpers import Pair, dev_lists

pytestmark = pytest.mark.gpu


def make(**kw):
    p = Pair(batch=2, grid=(12, 10), heads=4, appended=(4,), head_dim=64, frames=2, key_block=32, seed=4, **kw)
    return p, [[p.dev(x) for x in p.chunk()] for _ in range(2)], [dev_lists(p.lists(6, 64)) for _ in range(2)]


def both(p, chunk, lists, stream=None):
    out, lse = p.A.astro_select_attn_fwd(p.cache, *chunk[:3], lists, 2, 64, stream=stream)
    return [out, lse, *p.A.astro_select_attn_bwd(p.cache, *chunk[:3], out, lse, chunk[3], lists, 2, 64, stream=stream)]


@pytest.mark.parametrize("named", [False, True])
def test_two_streams(named):
    import torch
    p, chunks, lists = make()
    want = [both(p, c, l) for c, l in zip(chunks, lists)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            # (outputs belong to the stream too)
            with torch.cuda.stream(s):
                got[i].append(both(p, chunks[i], lists[i], s if named else None))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for run in g:
            assert all(torch.equal(a, b) for a, b in zip(run, w))
    spaces = p.cache._select_spaces
    assert len({t.data_ptr() for t in spaces.values()}) == len(spaces) == 3


def test_a_larger_call_leaves_the_space_of_one_in_flight():
    """The tensor that a larger one replaces goes back to the stream that used it."""
    import torch
    p, chunks, lists = make(max_chunk=2)
    side = torch.cuda.Stream()
    half = [x[:, :120].contiguous() for x in chunks[0]]
    one = dev_lists(p.lists(6, 64)[:, :, :2])
    call = lambda: p.A.astro_select_attn_fwd(p.cache, *half[:3], one, 1, 64)
    want = call()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = call()
        both(p, chunks[0], lists[0])
        torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0").fill_(255)
    other = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0").fill_(255)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and int(other[0]) == 255


def test_two_graphs_at_the_same_time():
    import torch
    p, chunks, lists = make()
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)], []
    want = [both(p, c, l) for c, l in zip(chunks, lists)]
    torch.cuda.synchronize()
    for g, c, l in zip(graphs, chunks, lists):
        with torch.cuda.graph(g):
            outs.append(both(p, c, l))
    for _ in range(4):
        for o in outs:
            for x in o:
                x.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = both(p, chunks[0], lists[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want[0]))
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))

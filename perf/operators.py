"""Measured cases of the rolling cache's fork, its block means, the block selection and the attention over selected blocks.

Five operators, each in a plain form (`own = False`: elementary torch operations) and as the library's calls
(`own = True`):

  fork    dst stream i becomes a copy of src stream source[i]
  append  a cache is rebuilt by appends that also keep the mean of every block of keys
  select  the n blocks of the cache whose mean key has the largest product with the mean query of a group of queries
  fwd     attention of a chunk over the selected blocks of the cache and the chunk itself
  bwd     its gradients with the cache detached

A frame has T = grid_h * grid_w tokens in ceil(T / key_block) key blocks, the last of which may be shorter; block
j of the frame in ring slot s has number s * ceil(T / key_block) + j.  Queries are grouped by query_block consecutive
rows of the chunk.  Keys are cached after rotation, rounded to the cache's type; means are taken of the keys and
queries as they are handed in.  The lists of selected blocks ascend, filled up with -1.
"""
import math

import torch

own = False

DEV = "cuda:0"
LOG_BASE = math.log(10000.0)


def _case(name, op, **sizes):
    case = dict(name=name, op=op, batch=1, heads=2, head_dim=64, grid_h=8, grid_w=8, capacity=4, sinks=0, frames=1, group=1,
                key_block=64, query_block=64, n_select=2, block_frames=0, start=0, appended="4", streams=1, source="")
    case.update(sizes)
    return case


def listed():
    return [
        # candidates of the smallest cache: latency
        _case("fork_small", "fork", streams=4, source="0,0,0,0"),
        # one prompt's full window becomes the windows of eight candidates that go on by themselves
        _case("fork_candidates", "fork", heads=12, head_dim=128, grid_h=30, grid_w=52, capacity=18, frames=3, appended="18",
              streams=8, source="0,0,0,0,0,0,0,0"),
        # the streams that go on are moved together; windows of different lengths, an odd frame, an empty stream
        _case("compact_ragged", "fork", batch=8, heads=6, grid_h=23, grid_w=17, capacity=9, sinks=1, frames=2,
              appended="9,0,3,40,9,5,1,17", streams=5, source="7,1,2,3,5"),
        # three frames of the smallest cache rebuilt, one frame an append: latency
        _case("append_small", "append", appended="3", key_block=32),
        # a full window of four streams rebuilt, with sinks and evictions, three frames an append
        _case("append_window", "append", batch=4, heads=12, head_dim=128, grid_h=30, grid_w=52, capacity=18, sinks=3, frames=3,
              appended="24"),
        # one 64-token frame over four: latency
        _case("select_small", "select", key_block=32),
        # three frames over a window of sixty, four streams
        _case("select_window", "select", batch=4, heads=12, head_dim=128, grid_h=30, grid_w=52, capacity=60, frames=3,
              appended="60", query_block=128, n_select=64),
        # one 64-token frame over half of four: latency
        _case("fwd_small", "fwd", key_block=32, n_select=4),
        # odd frames, causal frame by frame, candidates over one cache, windows of different lengths
        _case("fwd_ragged", "fwd", batch=2, heads=6, grid_h=23, grid_w=17, capacity=21, sinks=3, frames=2, group=2, key_block=32,
              n_select=24, block_frames=1, appended="21,7"),
        # a rollout's chunk over a long window, an eighth of it selected
        _case("fwd_window", "fwd", heads=12, head_dim=128, grid_h=30, grid_w=52, capacity=36, frames=3, appended="36",
              query_block=128, n_select=112),
        # the update's backward at odd frames and 64 columns
        _case("bwd_ragged", "bwd", batch=2, heads=6, grid_h=23, grid_w=17, capacity=21, sinks=3, frames=2, key_block=32,
              n_select=24, block_frames=1, appended="21,7"),
        # the update of two clips, a tenth of the window selected
        _case("bwd_window", "bwd", batch=2, heads=12, head_dim=128, grid_h=30, grid_w=52, capacity=18, frames=3, appended="18",
              query_block=128, n_select=44),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _draw(rng):
    op = rng.choice(["fork", "append", "select", "fwd", "fwd", "bwd", "bwd"])
    case = _case("", op, head_dim=rng.choice([64, 128]), heads=rng.randint(1, 12))
    tokens = _log_int(rng, 1, 1560)
    case["grid_w"] = max(1, int(math.sqrt(tokens) * rng.uniform(0.7, 1.6)))
    case["grid_h"] = max(1, tokens // case["grid_w"])
    case["batch"] = _log_int(rng, 1, 8)
    case["group"] = rng.choice([1, 1, 2]) if op in ("select", "fwd", "bwd") else 1
    case["frames"] = rng.randint(1, 3)
    case["capacity"] = _log_int(rng, 4, 57) + case["frames"]
    case["sinks"] = rng.randint(0, min(5, case["capacity"] - case["frames"]))
    case["key_block"] = rng.choice([32, 64, 128, 256])
    case["query_block"] = rng.choice([64, 128])
    case["block_frames"] = rng.choice([0, 0, 1])
    case["start"] = _log_int(rng, 1, 5000)
    least = 1 if op == "append" else 0
    case["appended"] = ",".join(str(rng.choice([case["capacity"], rng.randint(least, case["capacity"] + 9)])) for _ in range(case["batch"]))
    blocks = case["capacity"] * _frame_blocks(case)
    case["n_select"] = min(_log_int(rng, 1, 112), blocks, 1024 * 32 // case["key_block"])
    if op == "fork":
        case["streams"] = rng.randint(1, 8)
        case["source"] = ",".join(str(rng.randrange(case["batch"])) for _ in range(case["streams"]))
    del case["name"]
    return case


def draw(rng):
    most = [work(case) for case in listed()]
    while True:
        case = _draw(rng)
        cost = work(case)
        if all(cost[x] <= max(m[x] for m in most) for x in ("bytes", "flops")):
            return case


def _ints(text):
    return [int(x) for x in text.split(",") if x]


def _appended(case):
    n = _ints(case["appended"])
    return n if len(n) == case["batch"] else n * case["batch"]


def _pairs(case):
    """rotary pairs by frame, row and column"""
    third = case["head_dim"] // 6
    return case["head_dim"] // 2 - 2 * third, third, third


def _tokens(case):
    return case["grid_h"] * case["grid_w"]


def _frame_blocks(case):
    return -(-_tokens(case) // case["key_block"])


def _groups(case):
    return -(-case["frames"] * _tokens(case) // case["query_block"])


def _slots(case, appended):
    """the frame number in every slot of a stream's ring, oldest writes replaced; -1 = empty"""
    slots = [-1] * case["capacity"]
    for n in range(appended):
        window = case["capacity"] - case["sinks"]
        slots[n if n < case["capacity"] else case["sinks"] + (n - case["sinks"]) % window] = n
    return slots


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _angles(case, first_frames, n_frames):
    """[len(first_frames), n_frames * T, head_dim / 2], in 64 bits"""
    n_t, n_h, n_w = _pairs(case)
    freq = lambda n: torch.exp(torch.arange(n, device=DEV, dtype=torch.float64) * (-LOG_BASE / n))
    at = torch.arange(n_frames * _tokens(case), device=DEV)
    frame, rest = at // _tokens(case), at % _tokens(case)
    row = (rest // case["grid_w"]).double()[:, None] * freq(n_h)
    col = (rest % case["grid_w"]).double()[:, None] * freq(n_w)
    first = torch.tensor(first_frames, device=DEV, dtype=torch.float64)
    time = (first[:, None] + frame)[:, :, None] * freq(n_t)
    spread = lambda x: x.expand(len(first_frames), *x.shape)
    return torch.cat([time, spread(row), spread(col)], dim=2)


def _rotate(x, angles, back=False):
    """x [B, N, H, D]: adjacent pairs turned by angles [B, N, D / 2]"""
    cos, sin = angles.cos().to(x.dtype)[:, :, None], angles.sin().to(x.dtype)[:, :, None]
    if back:
        sin = -sin
    even, odd = x[..., 0::2], x[..., 1::2]
    return torch.stack([even * cos - odd * sin, even * sin + odd * cos], dim=-1).flatten(-2)


def _block_means(case, k):
    """raw keys [B, n_frames * T, H, D] -> fp32 [B, H, n_frames, blocks of a frame, D], sums in 64 bits"""
    b, n, h, d = k.shape
    frames, blocks, size = n // _tokens(case), _frame_blocks(case), case["key_block"]
    x = torch.zeros(b, frames, blocks * size, h, d, device=DEV, dtype=torch.float64)
    x[:, :, : _tokens(case)] = k.view(b, frames, _tokens(case), h, d)
    counts = torch.full((blocks,), size, device=DEV, dtype=torch.float64)
    counts[-1] = _tokens(case) - (blocks - 1) * size
    sums = x.view(b, frames, blocks, size, h, d).sum(3)
    return (sums / counts[:, None, None]).float().permute(0, 3, 1, 2, 4)


def _rope(case):
    return case["op"] != "fork"  # a fork moves rows whatever they mean


def _new_cache(case, batch):
    import paper_2603_17051_amd as astro
    return astro.astro_kvcache_create(batch, case["heads"], case["head_dim"], case["grid_h"], case["grid_w"], case["capacity"],
                                      case["sinks"], case["frames"], _pairs(case) if _rope(case) else (0, 0, 0), device=DEV,
                                      block_frames=case["block_frames"], key_block=case["key_block"])


class _Ring:
    """what a program without the library keeps: rotated keys, values [B, H, C * T, D], means, frames appended"""

    def __init__(self, case, batch):
        shape = (batch, case["heads"], case["capacity"] * _tokens(case), case["head_dim"])
        self.k = torch.zeros(shape, device=DEV, dtype=torch.bfloat16)
        self.v = torch.zeros(shape, device=DEV, dtype=torch.bfloat16)
        self.means = torch.zeros(batch, case["heads"], case["capacity"] * _frame_blocks(case), case["head_dim"], device=DEV)
        self.appended = [0] * batch

    def reset(self):
        self.appended = [0] * len(self.appended)

    def put(self, case, b, slots, k, v, means):
        """frames with rotated keys k, v [n * T, H, D], means [H, n, blocks, D] into the slots of stream b"""
        t, nb = _tokens(case), _frame_blocks(case)
        for i, s in enumerate(slots):
            self.k[b, :, s * t:(s + 1) * t] = k[i * t:(i + 1) * t].transpose(0, 1)
            self.v[b, :, s * t:(s + 1) * t] = v[i * t:(i + 1) * t].transpose(0, 1)
            self.means[b, :, s * nb:(s + 1) * nb] = means[:, i]

    def append(self, case, k, v, first_frame, precise):
        """k, v [B, n * T, H, D] as handed in; rotated in 64 bits if `precise`"""
        n = k.shape[1] // _tokens(case)
        turned = k.double() if precise else k.float()
        if _rope(case):
            turned = _rotate(turned, _angles(case, [first_frame + a for a in self.appended], n))
        turned = turned.to(torch.bfloat16)
        means = _block_means(case, k)
        for b, a in enumerate(self.appended):
            after = _slots(case, a + n)
            self.put(case, b, [after.index(a + i) for i in range(n)], turned[b], v[b], means[b])
            self.appended[b] = a + n


def _window(case, seed, steps):
    """the frames of `steps` appends, newest last"""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    shape = (case["batch"], case["frames"] * _tokens(case), case["heads"], case["head_dim"])
    drift = torch.randn(case["batch"], 1, case["heads"], case["head_dim"], generator=gen, device=DEV) * 0.3
    for _ in range(steps):
        # keys of a video drift: what a block of them has in common is what a selection goes by
        drift = 0.9 * drift + 0.3 * torch.randn(drift.shape, generator=gen, device=DEV)
        k = (torch.randn(shape, generator=gen, device=DEV) + drift).to(torch.bfloat16)
        yield k, _normal(shape, gen)


def _filled(case, seed, library):
    """a cache whose stream b has got appended[b] frames, by the library or as a _Ring"""
    t, n_b = _tokens(case), _appended(case)
    steps = -(-max(n_b) // case["frames"]) if max(n_b) else 0
    total = steps * case["frames"]
    data = list(_window(case, seed, steps))
    if not library:
        ring = _Ring(case, case["batch"])
        frames_k = torch.cat([k for k, _ in data], 1) if data else None
        frames_v = torch.cat([v for _, v in data], 1) if data else None
        for b, n in enumerate(n_b):
            slots = _slots(case, n)
            for s, f in enumerate(slots):
                if f < 0:
                    continue
                at = (total - n + f) * t
                k, v = frames_k[b:b + 1, at:at + t], frames_v[b:b + 1, at:at + t]
                turned = _rotate(k.double(), _angles(case, [case["start"] + f], 1)) if _rope(case) else k
                ring.put(case, b, [s], turned[0].to(torch.bfloat16), v[0], _block_means(case, k)[0])
            ring.appended[b] = n
        return ring
    import paper_2603_17051_amd as astro
    cache = _new_cache(case, case["batch"])
    # streams with fewer frames are emptied where their first one comes
    astro.astro_kvcache_reset(cache, -1, case["start"])
    done = 0
    for k, v in data:
        cuts = sorted({0, case["frames"]} | {total - n - done for n in n_b if 0 <= total - n - done < case["frames"]})
        for lo, hi in zip(cuts, cuts[1:]):
            for b, n in enumerate(n_b):
                if total - n == done + lo:
                    astro.astro_kvcache_reset(cache, b, case["start"])
            astro.astro_kvcache_append(cache, k[:, lo * t:hi * t].contiguous(), v[:, lo * t:hi * t].contiguous(), hi - lo)
        done += case["frames"]
    for b, n in enumerate(n_b):
        if n == 0:
            astro.astro_kvcache_reset(cache, b, case["start"])
    return cache


def _lists(case, seed):
    """selections as an earlier call left them: ascending, for each head and group, blocks of the newest frame among them"""
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)
    out = torch.full((case["batch"] * case["group"], case["heads"], _groups(case), case["n_select"]), -1, dtype=torch.int32, device=DEV)
    for c in range(out.shape[0]):
        blocks = min(_appended(case)[c // case["group"]], case["capacity"]) * _frame_blocks(case)
        n = min(blocks, case["n_select"])
        if n:
            order = torch.rand(case["heads"], _groups(case), blocks, generator=gen, device=DEV)
            out[c, :, :, :n] = order.topk(n, dim=-1).indices.sort(dim=-1).values
    return out


class _Chunk:
    """q, k, v (and dout) of the chunk and its place"""

    def __init__(self, case, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed + 2)
        shape = (case["batch"] * case["group"], case["frames"] * _tokens(case), case["heads"], case["head_dim"])
        self.q, self.k, self.v, self.dout = (_normal(shape, gen) for _ in range(4))
        self.first = [case["start"] + _appended(case)[c // case["group"]] for c in range(shape[0])]


def prepare(case, seed):
    state = {"case": case}
    if case["op"] == "append":
        steps = -(-max(_appended(case)) // case["frames"])
        state["chunks"] = list(_window(case, seed, steps))
        state["cache"] = _new_cache(case, case["batch"]) if own else _Ring(case, case["batch"])
        return state
    state["cache"] = _filled(case, seed, own)
    if case["op"] == "fork":
        state["to"] = _new_cache(case, case["streams"]) if own else _Ring(case, case["streams"])
        state["source"] = _ints(case["source"])
        return state
    chunk = state["chunk"] = _Chunk(case, seed)
    if case["op"] == "select":
        return state
    state["blocks"] = _lists(case, seed)
    if case["op"] == "bwd":  # of the forward before it
        ring = _filled(case, seed, False) if own else state["cache"]
        state["out"], state["lse"] = _forward(case, ring, chunk, state["blocks"])
    return state


def _rows(case, blocks):
    """lists [..., n] -> ring rows [..., n * key_block] and whether each counts"""
    size, t, nb = case["key_block"], _tokens(case), _frame_blocks(case)
    within = (blocks.clamp(min=0) % nb)[..., None] * size + torch.arange(size, device=DEV)
    rows = (blocks.clamp(min=0) // nb)[..., None] * t + within
    counts = (blocks >= 0)[..., None] & (within < t)
    return (rows * counts).flatten(-2).long(), counts.flatten(-2)


def _chunk_mask(case):
    """[Nq, Nq]: which chunk keys a chunk query sees"""
    frame = torch.arange(case["frames"] * _tokens(case), device=DEV) // _tokens(case)
    if not case["block_frames"]:
        return torch.ones(len(frame), len(frame), device=DEV, dtype=torch.bool)
    return (frame // case["block_frames"])[:, None] >= (frame // case["block_frames"])[None]


def _grouped(case, x):
    """[Nq, D] -> [groups, query_block, D], zeros behind the last row"""
    g, size = _groups(case), case["query_block"]
    return torch.nn.functional.pad(x, (0, 0, 0, g * size - x.shape[0])).view(g, size, -1)


def _scores(case, ring, blocks, c, h, q, k, mask, scale):
    """of candidate c's head h: the selected rows' keys and values, scores over them and over the chunk"""
    b, n = c // case["group"], q.shape[0]
    rows, counts = _rows(case, blocks[c, h])
    kept = ring.k[b, h].float()[rows]
    over_ring = (_grouped(case, q) @ kept.transpose(1, 2) * scale).masked_fill(~counts[:, None], -math.inf)
    over_ring = over_ring.flatten(0, 1)[:n]
    over_chunk = (q @ k.T * scale).masked_fill(~mask, -math.inf)
    return rows, kept, over_ring, over_chunk


def _forward(case, ring, chunk, blocks):
    angles, mask = _angles(case, chunk.first, case["frames"]), _chunk_mask(case)
    q, k, v = _rotate(chunk.q.float(), angles), _rotate(chunk.k.float(), angles), chunk.v.float()
    out = torch.empty(q.shape, device=DEV, dtype=torch.bfloat16)
    lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], device=DEV)
    for c in range(q.shape[0]):
        for h in range(q.shape[2]):
            rows, _, s_ring, s_chunk = _scores(case, ring, blocks, c, h, q[c, :, h], k[c, :, h], mask, case["head_dim"] ** -0.5)
            top = torch.maximum(s_ring.amax(1), s_chunk.amax(1))[:, None]
            p_ring, p_chunk = (s_ring - top).exp(), (s_chunk - top).exp()
            total = p_ring.sum(1, True) + p_chunk.sum(1, True)
            o = _grouped(case, p_ring) @ ring.v[c // case["group"], h].float()[rows]
            o = o.flatten(0, 1)[: q.shape[1]] + p_chunk @ v[c, :, h]
            out[c, :, h] = (o / total).to(torch.bfloat16)
            lse[c, h] = (top + total.log())[:, 0]
    return out, lse


def _backward(case, ring, chunk, blocks, out, lse):
    angles, mask, scale = _angles(case, chunk.first, case["frames"]), _chunk_mask(case), case["head_dim"] ** -0.5
    q, k, v, dout = _rotate(chunk.q.float(), angles), _rotate(chunk.k.float(), angles), chunk.v.float(), chunk.dout.float()
    dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    delta = (dout * out.float()).sum(-1)
    for c in range(q.shape[0]):
        for h in range(q.shape[2]):
            rows, kept, s_ring, s_chunk = _scores(case, ring, blocks, c, h, q[c, :, h], k[c, :, h], mask, scale)
            p_ring, p_chunk = (s_ring - lse[c, h][:, None]).exp(), (s_chunk - lse[c, h][:, None]).exp()
            do, less = dout[c, :, h], delta[c, :, h][:, None]
            dp = _grouped(case, do) @ ring.v[c // case["group"], h].float()[rows].transpose(1, 2)
            ds_ring = p_ring * (dp.flatten(0, 1)[: q.shape[1]] - less) * scale
            ds_chunk = p_chunk * (do @ v[c, :, h].T - less) * scale
            dq[c, :, h] = (_grouped(case, ds_ring) @ kept).flatten(0, 1)[: q.shape[1]] + ds_chunk @ k[c, :, h]
            dk[c, :, h] = ds_chunk.T @ q[c, :, h]
            dv[c, :, h] = p_chunk.T @ do
    return _rotate(dq, angles, back=True), _rotate(dk, angles, back=True), dv


def _select(case, means, appended, q):
    """the lists of a selection by scores in 64 bits, rounded once; q [Nq, H, D]"""
    n, g, size = min(appended, case["capacity"]) * _frame_blocks(case), _groups(case), case["query_block"]
    lists = torch.full((q.shape[1], g, case["n_select"]), -1, device=DEV, dtype=torch.int32)
    if n == 0:
        return lists
    sums = torch.nn.functional.pad(q.double(), (0, 0, 0, 0, 0, g * size - q.shape[0])).view(g, size, *q.shape[1:]).sum(1)
    counts = torch.full((g, 1, 1), size, device=DEV, dtype=torch.float64)
    counts[-1] = q.shape[0] - (g - 1) * size
    mean = (sums / counts).float().double()
    score = (mean.transpose(0, 1) @ means[:, :n].double().transpose(1, 2)).float()
    score = score.masked_fill(score.isnan(), -math.inf)
    best = score.sort(dim=2, descending=True, stable=True).indices[..., : case["n_select"]]
    lists[..., : best.shape[2]] = best.sort(dim=2).values.int()
    return lists


def run(state):
    case, cache = state["case"], state["cache"]
    if own:
        import paper_2603_17051_amd as astro
        shape = lambda c: (-1, case["heads"], case["capacity"] * _tokens(case), case["head_dim"])
        rows = lambda c, x: x.view(torch.bfloat16).view(shape(c))
        if case["op"] == "fork":
            to = state["to"]
            astro.astro_kvcache_fork(to, cache, state["source"])
            return rows(to, to.k_storage), rows(to, to.v_storage), to.k_means
        if case["op"] == "append":
            astro.astro_kvcache_reset(cache, -1, case["start"])
            for k, v in state["chunks"]:
                astro.astro_kvcache_append(cache, k, v, case["frames"])
            return rows(cache, cache.k_storage), rows(cache, cache.v_storage), cache.k_means
        chunk = state["chunk"]
        if case["op"] == "select":
            return astro.astro_select_blocks(cache, chunk.q, case["frames"], case["n_select"], query_block=case["query_block"],
                                             group=case["group"])
        if case["op"] == "fwd":
            return astro.astro_select_attn_fwd(cache, chunk.q, chunk.k, chunk.v, state["blocks"], case["frames"],
                                               query_block=case["query_block"], group=case["group"])
        return astro.astro_select_attn_bwd(cache, chunk.q, chunk.k, chunk.v, state["out"], state["lse"], chunk.dout, state["blocks"],
                                           case["frames"], query_block=case["query_block"], group=case["group"])
    if case["op"] == "fork":
        to, t, nb = state["to"], _tokens(case), _frame_blocks(case)
        for i, b in enumerate(state["source"]):
            frames = min(cache.appended[b], case["capacity"])
            to.k[i, :, : frames * t] = cache.k[b, :, : frames * t]
            to.v[i, :, : frames * t] = cache.v[b, :, : frames * t]
            to.means[i, :, : frames * nb] = cache.means[b, :, : frames * nb]
            to.appended[i] = cache.appended[b]
        return to.k, to.v, to.means
    if case["op"] == "append":
        cache.reset()
        for k, v in state["chunks"]:
            cache.append(case, k, v, case["start"], False)
        return cache.k, cache.v, cache.means
    chunk = state["chunk"]
    if case["op"] == "select":
        return torch.stack([_select(case, cache.means[c // case["group"]], cache.appended[c // case["group"]], chunk.q[c])
                            for c in range(chunk.q.shape[0])])
    if case["op"] == "fwd":
        return _forward(case, cache, chunk, state["blocks"])
    return _backward(case, cache, chunk, state["blocks"], state["out"], state["lse"])


def work(case):
    t, h, d, b = _tokens(case), case["heads"], case["head_dim"], case["batch"]
    row = 2 * d * h
    resident = [min(n, case["capacity"]) for n in _appended(case)]
    mean_frame = 4 * d * h * _frame_blocks(case)
    if case["op"] == "fork":
        source = _ints(case["source"])
        frames = sum(resident[s] for s in set(source)) + sum(resident[s] for s in source)
        return {"bytes": frames * (2 * t * row + mean_frame), "flops": 0}
    if case["op"] == "append":
        frames = b * -(-max(_appended(case)) // case["frames"]) * case["frames"]
        return {"bytes": frames * (4 * t * row + mean_frame), "flops": frames * t * h * d * 4}
    n_q, c = case["frames"] * t, b * case["group"]
    blocks = [r * _frame_blocks(case) for r in resident]
    if case["op"] == "select":
        return {"bytes": c * n_q * row + sum(blocks) * 4 * d * h + 4 * c * h * _groups(case) * case["n_select"],
                "flops": case["group"] * sum(blocks) * _groups(case) * h * 2 * d + c * n_q * h * d}
    listed_rows = [min(case["n_select"] * min(case["key_block"], t), r * t) for r in resident]
    touched = [min(r * t, _groups(case) * case["group"] * n) for r, n in zip(resident, listed_rows)]
    ring_pairs = case["group"] * n_q * h * sum(listed_rows)
    seen = case["frames"] * t * n_q
    if case["block_frames"]:
        f, step = case["frames"], case["block_frames"]
        seen = t * t * sum(min((i // step + 1) * step, f) for i in range(f))
    chunk_pairs = c * h * seen
    lists = 4 * c * h * _groups(case) * case["n_select"]
    if case["op"] == "fwd":
        return {"bytes": c * n_q * (4 * row + 4 * h) + 2 * sum(touched) * row + lists, "flops": 4 * d * (ring_pairs + chunk_pairs)}
    return {"bytes": c * n_q * (5 * row + 4 * h + 6 * row) + 2 * sum(touched) * row + lists,
            "flops": d * (6 * ring_pairs + 10 * chunk_pairs)}


def exact(case, seed):
    """the definition, token by token, in 64 bits"""
    t, heads, d, cap = _tokens(case), case["heads"], case["head_dim"], case["capacity"]
    if case["op"] in ("fork", "append"):
        return _exact_state(case, seed)
    ring = _filled(case, seed, False)
    chunk = _Chunk(case, seed)
    n_q, size = case["frames"] * t, case["query_block"]
    token = torch.arange(cap * t, device=DEV)
    block_of = token // t * _frame_blocks(case) + token % t // case["key_block"]
    group_of = torch.arange(n_q, device=DEV) // size
    if case["op"] == "select":
        return _exact_lists(case, ring, chunk)
    lists = _lists(case, seed).long()
    angles = _angles(case, chunk.first, case["frames"])
    turn = torch.polar(torch.ones_like(angles), angles)[:, :, None]
    turned = lambda x: torch.view_as_real(torch.view_as_complex(x.double().unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
    turned_back = lambda x: torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * turn.conj()).flatten(-2)
    q, k = turned(chunk.q), turned(chunk.k)
    frame = torch.arange(n_q, device=DEV) // t
    step = case["block_frames"] or case["frames"]
    sees = (frame[None] // step) <= (frame[:, None] // step)
    out, lse = torch.empty_like(q), torch.empty(q.shape[0], heads, n_q, device=DEV, dtype=torch.float64)
    backward = case["op"] == "bwd"
    if backward:
        given_out, given_lse = _forward(case, ring, chunk, lists)
        grads = [torch.empty_like(q) for _ in range(3)]
    for c in range(q.shape[0]):
        b = c // case["group"]
        for h in range(heads):
            chosen = torch.zeros(_groups(case), cap * _frame_blocks(case) + 1, device=DEV, dtype=torch.bool)
            chosen.scatter_(1, torch.where(lists[c, h] < 0, chosen.shape[1] - 1, lists[c, h]), True)
            visible = torch.cat([chosen[:, block_of][group_of], sees], dim=1)
            keys = torch.cat([ring.k[b, h].double(), k[c, :, h]])
            values = torch.cat([ring.v[b, h].double(), chunk.v[c, :, h].double()])
            s = (q[c, :, h] @ keys.T) / math.sqrt(d)
            s[~visible] = -math.inf
            if not backward:
                lse[c, h] = s.logsumexp(1)
                out[c, :, h] = s.softmax(1) @ values
                continue
            p = (s - given_lse[c, h].double()[:, None]).exp()
            do = chunk.dout[c, :, h].double()
            ds = p * (do @ values.T - (do * given_out[c, :, h].double()).sum(1, True)) / math.sqrt(d)
            grads[0][c, :, h] = ds @ keys
            grads[1][c, :, h] = ds[:, cap * t:].T @ q[c, :, h]
            grads[2][c, :, h] = p[:, cap * t:].T @ do
    if backward:
        return turned_back(grads[0]), turned_back(grads[1]), grads[2]
    return out, lse


def _exact_lists(case, ring, chunk):
    """by counting, for each block, the blocks that come before it"""
    result = []
    for c in range(chunk.q.shape[0]):
        b = c // case["group"]
        n = min(ring.appended[b], case["capacity"]) * _frame_blocks(case)
        for h in range(case["heads"]):
            for rows in chunk.q[c, :, h].double().split(case["query_block"]):
                score = (ring.means[b, h, :n].double() * rows.mean(0).float().double()).sum(1).float()
                index = torch.arange(n, device=DEV)
                ahead = (score[None] > score[:, None]) | ((score[None] == score[:, None]) & (index[None] < index[:, None]))
                chosen = index[ahead.sum(1) < case["n_select"]].int()
                result.append(torch.nn.functional.pad(chosen, (0, case["n_select"] - len(chosen)), value=-1))
    return torch.stack(result).view(chunk.q.shape[0], case["heads"], _groups(case), case["n_select"])


def _exact_state(case, seed):
    t, nb = _tokens(case), _frame_blocks(case)
    steps = -(-max(_appended(case)) // case["frames"])
    if case["op"] == "append":
        numbers = [steps * case["frames"]] * case["batch"]
    else:
        numbers = _appended(case)
    data = list(_window(case, seed, steps))
    source = _ints(case["source"]) if case["op"] == "fork" else range(case["batch"])
    k_out = torch.zeros(len(source), case["heads"], case["capacity"] * t, case["head_dim"], device=DEV, dtype=torch.float64)
    v_out, means = torch.zeros_like(k_out), torch.zeros(*k_out.shape[:2], case["capacity"] * nb, case["head_dim"], device=DEV, dtype=torch.float64)
    for i, b in enumerate(source):
        for slot, n in enumerate(_slots(case, numbers[b])):
            if n < 0:
                continue
            step, frame = divmod(steps * case["frames"] - numbers[b] + n, case["frames"])
            k, v = (x[b, frame * t:(frame + 1) * t].double() for x in data[step])  # [T, H, D]
            for j, part in enumerate(k.split(case["key_block"])):
                means[i, :, slot * nb + j] = part.mean(0)
            if _rope(case):
                a = _angles(case, [case["start"] + n], 1)[0][:, None]
                k = torch.view_as_real(torch.view_as_complex(k.unflatten(-1, (-1, 2)).contiguous()) * torch.polar(torch.ones_like(a), a)).flatten(-2)
            k_out[i, :, slot * t:(slot + 1) * t] = k.transpose(0, 1)
            v_out[i, :, slot * t:(slot + 1) * t] = v.transpose(0, 1)
    return k_out, v_out, means

"""Performance cases of attention that weighs the cache, and of rotary
positions with several axes.

A decoder may evict by what its attention looked at: each attention call then
also sums, per cached slot, the weights that the queries gave it, and the
eviction step keeps the slots with the largest sums.  And a prompt with images
or video gives every token a position on several axes (time, height, width),
each of which turns some of the head's pairs.  Each case is one such call.

Kinds of case:
  axes    rotation of a [batch][chunk][heads][head_dim] tensor by positions of
          several axes, or its gradient (`backward`)
  append  `chunk` new tokens per sequence into the pages, keys and queries
          rotated by positions of several axes; a 4-bit cache's new rows are
          read back as the values they stand for
  weigh   `chunk` queries per sequence (causal among themselves) over the
          paged cache, with the log of the softmax's sum, and the weights of
          the last `watch` tokens' queries (0: all) added to the slots' sums
"""
import math
import random

import torch

own = False

THETA = 500000.0
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TABLE = 32768  # positions of the rotary table

# A 4096-wide decoder layer of 32 query heads and 8 KV heads of 128, 16-token
# pages, bf16: the repository's default configuration.
_BASE = dict(batch=1, chunk=1, heads=32, kv_heads=8, head_dim=128)
_ROPE = dict(pairs="16 24 24", turns=False, apart=False, interleaved=False)
_PAGED = dict(page=16, n_min=4224, n_max=4224, fmt="bf16")


def _case(name, kind, **kw):
    c = dict(_BASE, kind=kind)
    if kind in ("axes", "append"):
        c.update(_ROPE)
    if kind == "axes":
        c.update(dtype="bf16", backward=False)
        del c["kv_heads"]
    else:
        c.update(_PAGED)
    if kind == "weigh":
        c.update(watch=0, decay=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The queries of a decode batch of 32, one token each, after prompts
        # with images: latency.
        _case("axes_decode_32seq", "axes", batch=32),
        # A prompt of 16,384 tokens, most of them video: the axes take turns
        # along the pairs.
        _case("axes_video_prompt", "axes", chunk=16384, pairs="24 20 20", turns=True),
        # Training an image encoder: the gradient through interleaved pairs,
        # half of them turned by height and half by width, in 32 bits.
        _case("axes_image_gradient", "axes", batch=4, chunk=4097, heads=16, head_dim=64, pairs="16 16", apart=True,
              interleaved=True, dtype="fp32", backward=True),
        # Every decoded token of a batch of 32 at its budget.
        _case("append_axes_decode_32seq", "append", batch=32, n_min=4097, n_max=4224),
        # A prompt of odd length with images into a cache in 4 bits.
        _case("append4_axes_prompt", "append", chunk=8191, n_min=8191, n_max=8191, pairs="24 20 20", turns=True,
              fmt="mxfp4"),
        # One interactive session at its budget of 4096: the smallest read.
        _case("weigh_1seq", "weigh"),
        # One session with a long past.
        _case("weigh_long_1seq", "weigh", n_min=131071, n_max=131071),
        # The benchmark's ragged batch, one token each, before its eviction.
        _case("weigh_ragged_32seq", "weigh", batch=32, n_min=8192, n_max=32768),
        # The same over a cache in 4 bits, older weights fading.
        _case("weigh4_ragged_32seq", "weigh", batch=32, n_min=8192, n_max=32768, fmt="mxfp4", decay=0.96875),
        # Chunks of the eviction cadence (128 new tokens) for eight sequences
        # at 32,768 tokens in 4 bits, all of them counted.
        _case("weigh4_chunk_8seq", "weigh", batch=8, chunk=128, n_min=32768, n_max=32768, fmt="mxfp4"),
        # A prefill chunk of 4096 tokens over a 16k cache, all of it counted.
        _case("weigh_prefill", "weigh", chunk=4096, n_min=16384, n_max=16384),
        # A prompt of odd length whose last 64 tokens choose what is kept.
        _case("weigh_prompt_window", "weigh", chunk=8191, n_min=8191, n_max=8191, watch=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _split(rng, pairs, axes):
    """`pairs` in `axes` parts of one at least, even or not."""
    if rng.random() < 0.4:
        parts = [pairs // axes + (a < pairs % axes) for a in range(axes)]
    else:
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        parts = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
    return " ".join(str(n) for n in parts)


def draw(rng):
    """One more call of the ranges above: batches, odd lengths, head shapes
    and groups, page sizes, axes, layouts, windows and both formats of the
    cache."""
    kind = rng.choice(["axes", "append", "weigh", "weigh", "prefill", "prefill"])
    heads, kv_heads, d = rng.choice([(32, 8, 128), (32, 8, 128), (16, 2, 128), (8, 8, 128), (24, 8, 64),
                                     (64, 8, 128), (40, 8, 128), (8, 1, 128), (16, 8, 256),
                                     (32, 4, 64), (7, 1, 64)])
    rotary = rng.choice([d, d, d // 2])
    rot = dict(pairs=_split(rng, rotary // 2, rng.choice([2, 3, 3, 3, 4])), turns=rng.random() < 0.5,
               apart=rng.random() < 0.3, interleaved=rng.random() < 0.4)
    shape = dict(heads=heads, kv_heads=kv_heads, head_dim=d)
    paged = dict(page=rng.choice([16, 16, 16, 32, 64, 12, 128]), fmt=rng.choice(["bf16", "mxfp4"]))
    if kind == "axes":
        tokens = _log_int(rng, 1, 16384 * 4096 // (heads * d))
        batch = min(tokens, _log_int(rng, 1, 64))
        return _case(None, "axes", batch=batch, chunk=min(16384, tokens // batch), heads=heads, head_dim=d,
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), backward=rng.random() < 0.4, **rot)
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        chunk = 1 if rng.random() < 0.4 else _log_int(rng, 2, 8191 // batch)
        n = chunk + _log_int(rng, 1, 4096)
        return _case(None, "append", batch=batch, chunk=chunk, n_min=n, n_max=n + rng.choice([0, 0, 37, 301]),
                     **shape, **rot, **paged)
    decay = rng.choice([1.0, 1.0, 0.96875, 0.0])
    if kind == "weigh":
        batch = _log_int(rng, 1, 64)
        chunk = rng.choice([1, 1, 1, 1, 2, 3, 5, 8])
        room = min(131072, 640 * 1024 * 1024 // (batch * kv_heads * d))
        n_max = _log_int(rng, 64, room)
        n_min = n_max if rng.random() < 0.4 else _log_int(rng, max(chunk, n_max // 8), n_max)
        return _case(None, "weigh", batch=batch, chunk=chunk, n_min=n_min, n_max=n_max,
                     watch=rng.choice([0, 0, 0, 1]), decay=decay, **shape, **paged)
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    chunk = _log_int(rng, 17, 4096 // batch)
    room = min(32768, 16384 * 4096 * 4096 // (batch * chunk * heads * d))
    n = max(chunk, _log_int(rng, chunk, max(chunk + 1, room)))
    watch = rng.choice([0, 0, min(chunk, _log_int(rng, 1, 128))])
    return _case(None, "weigh", batch=batch, chunk=chunk, n_min=n, n_max=n, watch=watch, decay=decay, **shape, **paged)


# ---------------------------------------------------------------------------
# Inputs (plain torch, from the seed alone)
# ---------------------------------------------------------------------------
def _lengths(c):
    """Tokens cached per sequence, the new ones included: ragged between
    n_min and n_max, both reached, in an order of no meaning."""
    B, lo, hi = c["batch"], c["n_min"], c["n_max"]
    n = [hi - (hi - lo) * i // max(1, B - 1) for i in range(B)]
    random.Random(B * 1000003 + hi).shuffle(n)
    return n


def _row_bytes(c):
    hd = c["kv_heads"] * c["head_dim"]
    return 2 * hd if c["fmt"] == "bf16" else max(128, (hd // 2 + hd // 32 + 15) // 16 * 16)


def _pairs(c):
    """How many pairs each axis turns."""
    return [int(n) for n in c["pairs"].split()]


def _axis_of(c):
    """The axis that turns each pair, and the pair's number on its axis."""
    left, axis, place = _pairs(c), [], []
    while any(left):
        for a, n in enumerate(_pairs(c)):
            take = left[a] if not c["turns"] else min(1, left[a])
            axis += [a] * take
            place += range(n - left[a], n - left[a] + take)
            left[a] -= take
    return axis, place


def _rotation_table(c, device):
    """float32 [TABLE][pairs][2]: the cosine and sine of each pair at every
    position of its axis; frequencies over the whole head, or over each axis'
    own pairs (`apart`)."""
    axis, place = (torch.tensor(x, device=device) for x in _axis_of(c))
    count = torch.tensor(_pairs(c), device=device, dtype=torch.float64)[axis]
    at = place if c["apart"] else torch.arange(len(axis), device=device)
    part = at / (count if c["apart"] else float(len(axis)))
    angle = torch.arange(TABLE, device=device, dtype=torch.float64)[:, None] * THETA ** -part
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def _positions(c, g, dev):
    """int32 [batch][axes][chunk]: text, whose axes go together, around
    frames of a grid; or a grid alone for two axes.  Single tokens: [batch][axes]."""
    B, C, A = c["batch"], c["chunk"], len(_pairs(c))
    first = torch.randint(0, 8192, (B, 1, 1), generator=g, device=dev)
    if C == 1:
        return (first[..., 0] + torch.randint(0, 4, (B, A), generator=g, device=dev)).int()
    before = 0 if A == 2 else C // 8
    n = C - 2 * before
    side = max(1, math.isqrt(n if A == 2 else n // 4))
    i = torch.arange(C, device=dev)
    j = (i - before).clamp(0, n - 1)
    grid = torch.stack([j // (side * side), j // side % side, j % side, i % 7])
    grid = torch.stack([j // side, j % side]) if A == 2 else grid[:A]
    after = int(grid.max()) + 1
    p = torch.where((i >= before) & (i < before + n), grid + before,
                    torch.where(i < before, i, before + after + i - before - n))
    return (first + p).int().contiguous()


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=dev).to(dtype)

    B, C, Hq, d = c["batch"], c["chunk"], c["heads"], c["head_dim"]
    s = {"case": c}
    if c["kind"] != "weigh":
        s["positions"] = _positions(c, g, dev)
        s["axis"] = torch.tensor(_axis_of(c)[0], device=dev)
        s["table"] = _rotation_table(c, dev)
    if c["kind"] == "axes":
        s["x"] = normal(B, C, Hq, d, dtype=torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        s["y"] = torch.empty_like(s["x"])
        return s
    H, page = c["kv_heads"], c["page"]
    n = torch.tensor(_lengths(c), device=dev, dtype=torch.int32)
    width = -(-c["n_max"] // page)
    s["n_cached"] = n
    s["page_table"] = torch.randperm(B * width, generator=g, device=dev).view(B, width).int()
    s["q"] = normal(B, C, Hq, d)
    # keys with a few loud channels, as rotated keys have
    profile = torch.exp(0.5 * torch.randn((H, d), generator=g, device=dev))
    rows = (1, 2, B * width, page)
    if c["kind"] == "append":
        s["k"] = (torch.randn((B, C, H, d), generator=g, device=dev) * profile).bfloat16()
        s["v"] = normal(B, C, H, d)
        # the tokens' ids: the cache has been evicted from, ids run ahead of slots
        s["ids"] = n - C + torch.randint(0, 8192, (B,), generator=g, device=dev, dtype=torch.int32)
        s["q_out"] = torch.empty_like(s["q"])
        s["pos"] = torch.full((B, c["n_max"]), -1, device=dev, dtype=torch.int32)
        if c["fmt"] == "bf16":
            s["pool"] = normal(*rows, H, d)
        else:
            s["pool"] = torch.zeros(*rows, _row_bytes(c), device=dev, dtype=torch.uint8)
            s["k_held"], s["v_held"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        return s
    pool = normal(*rows, H, d)
    pool[:, 0] *= profile.bfloat16()
    if c["fmt"] != "bf16":
        packed = torch.zeros(*rows, _row_bytes(c), device=dev, dtype=torch.uint8)
        flat, out = pool.view(-1, H * d), packed.view(-1, packed.shape[-1])
        for a in range(0, flat.shape[0], 1 << 18):
            out[a:a + (1 << 18)] = _pack(flat[a:a + (1 << 18)].float(), packed.shape[-1])
        pool = packed
    s["pool"] = pool
    # what a few earlier tokens' queries left, heavy-tailed; new tokens have none yet
    s["before"] = torch.randn((B, c["n_max"]), generator=g, device=dev).exp_().mul_(2 * Hq / c["n_max"])
    s["weights"] = torch.zeros_like(s["before"])
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(B, Hq, C, device=dev)
    return s


# ---------------------------------------------------------------------------
# The plain form, in 32 bits
# ---------------------------------------------------------------------------
def _pack(x, row_bytes):
    """float32 [rows][channels] as 4-bit rows: two codes a byte (the lower
    channel in the low bits), then a scale byte per 32 channels."""
    rows, n = x.shape
    blk = x.view(rows, n // 32, 32)
    top = blk.abs().amax(-1)
    exponent = torch.frexp(top)[1] - 3                       # floor(log2(top)) - 2
    exponent = exponent + (top > torch.ldexp(torch.full_like(top, 7.0), exponent)).int()
    exponent = torch.where(top > 0, exponent.clamp(min=-126), torch.full_like(exponent, -126))
    scaled = torch.ldexp(blk, -exponent[..., None])
    a = scaled.abs()
    code = sum((a > t).to(torch.uint8) if up else (a >= t).to(torch.uint8)
               for t, up in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True),
                             (3.5, False), (5.0, True)))     # ties to the even code
    code = code | ((scaled < 0).to(torch.uint8) << 3)
    code = code.view(rows, n)
    out = torch.zeros(rows, row_bytes, device=x.device, dtype=torch.uint8)
    out[:, :n // 2] = code[:, 0::2] | (code[:, 1::2] << 4)
    out[:, n // 2:n // 2 + n // 32] = (exponent + 127).to(torch.uint8)
    return out


def _unpack(rows, n):
    """The float32 values of 4-bit rows [...][row_bytes]."""
    byte = rows[..., :n // 2]
    code = torch.stack([byte & 15, byte >> 4], -1).flatten(-2).int()
    value = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=rows.device)[code]
    exponent = rows[..., n // 2:n // 2 + n // 32].int() - 127
    return torch.ldexp(value.unflatten(-1, (n // 32, 32)), exponent[..., None]).flatten(-2)


def _turns(s):
    """[batch][chunk][pairs][2]: each token's cosines and sines, pair by pair
    from the row of its axis' position."""
    B, C = s["case"]["batch"], s["case"]["chunk"]
    p = s["positions"].view(B, -1, C)[:, s["axis"]].transpose(1, 2).long()
    return s["table"][p, torch.arange(s["axis"].numel(), device=p.device)]


def _rotate(x, cs, c, backward=False):
    """float32 x [B][C][heads][d] by cs [B][C][pairs][2]."""
    r = 2 * sum(_pairs(c))
    cos, sin = cs[..., 0].unsqueeze(2), cs[..., 1].unsqueeze(2)
    if backward:
        sin = -sin
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _run_plain(s):
    c = s["case"]
    B, C, Hq, d = c["batch"], c["chunk"], c["heads"], c["head_dim"]
    if c["kind"] == "axes":
        return _rotate(s["x"].float(), _turns(s), c, c["backward"]).to(s["x"].dtype)
    dev = s["pool"].device
    step = torch.arange(C, device=dev)
    H, page = c["kv_heads"], c["page"]
    n = s["n_cached"].long()
    if c["kind"] == "append":
        slot = n[:, None] - C + step
        where = s["page_table"].gather(1, slot // page).long(), slot % page
        cs = _turns(s)
        k = _rotate(s["k"].float(), cs, c)
        q = _rotate(s["q"].float(), cs, c).bfloat16()
        s["pos"].scatter_(1, slot, s["ids"][:, None] + step.int())
        kp, vp = s["pool"][0]
        if c["fmt"] == "bf16":
            kp[where] = k.bfloat16()
            vp[where] = s["v"]
            return {"pool": s["pool"], "q": q, "pos": s["pos"]}
        kp[where] = _pack(k.reshape(B * C, H * d), kp.shape[-1]).view(B, C, -1)
        vp[where] = _pack(s["v"].float().reshape(B * C, H * d), vp.shape[-1]).view(B, C, -1)
        return {"k": _unpack(kp[where], H * d).view(B, C, H, d).bfloat16(),
                "v": _unpack(vp[where], H * d).view(B, C, H, d).bfloat16(), "q": q, "pos": s["pos"]}
    N, G = c["n_max"], Hq // H
    slot = torch.arange(N, device=dev)
    rows = (s["page_table"][:, slot // page].long(), (slot % page).expand(B, N))
    kp, vp = s["pool"][0]
    k, v = kp[rows], vp[rows]
    if c["fmt"] == "bf16":
        k, v = k.float(), v.float()
    else:
        k, v = _unpack(k, H * d).view(B, N, H, d), _unpack(v, H * d).view(B, N, H, d)
    q = s["q"].float().view(B, C, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * C, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).view(B, H, G, C, N)
    score.mul_(1.0 / math.sqrt(d))
    hidden = slot >= (n[:, None] - C + 1 + step)[..., None]           # [B][C][N]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(B, H, G * C, N), v.permute(0, 2, 1, 3).contiguous())
    out = out.view(B, H, G, C, d) / total
    lse = (top + total.log()).view(B, Hq, C)
    counted = weight[:, :, :, C - (c["watch"] or C):].div_(total[:, :, :, C - (c["watch"] or C):]).sum((1, 2, 3))
    # (a new token's sum starts here)
    before = torch.where(slot < n[:, None] - C, c["decay"] * s["before"], 0.0)
    weights = torch.where(slot < n[:, None], before + counted, s["weights"])
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(B, C, Hq, d).bfloat16(), "lse": lse, "weights": weights}


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _plan(s):
    """What a program builds once for its buffers: configuration, argument
    structs and workspace."""
    from paper_2606_26472_amd import epikv as E
    c = s["case"]
    B, C, Hq, d = c["batch"], c["chunk"], c["heads"], c["head_dim"]
    p = {"E": E}
    if "table" in s:
        p["rope"] = E.default_rope(rotary_dim=2 * sum(_pairs(c)), n_pos=TABLE, theta=THETA,
                                   layout=E.ROPE_INTERLEAVED if c["interleaved"] else E.ROPE_HALF)
        p["axes"] = E.axes_of(_pairs(c), order=E.AXES_TURNS if c["turns"] else E.AXES_SECTIONS,
                              frequencies=E.AXES_APART if c["apart"] else E.AXES_SHARED)
        p["ld_pos"] = C if C > 1 else 0
    if c["kind"] == "axes":
        p["x"], p["y"] = E.rows_of(s["x"]), E.rows_of(s["y"])
        p["dtype"] = E.DTYPE_BF16 if c["dtype"] == "bf16" else E.DTYPE_FP32
        return p
    fmt = E.KV_BF16 if c["fmt"] == "bf16" else E.KV_MXFP4
    cfg = p["cfg"] = E.default_cfg(batch=B, n_layers=1, n_kv_heads=c["kv_heads"], head_dim=d,
                                   page_size=c["page"], kv_format=fmt)
    pool = E.pool_of(s["pool"])
    width = s["page_table"].shape[1]
    if c["kind"] == "append":
        p["io"] = E.make_append_io(C, pool, 0, s["page_table"], width, s["n_cached"], s["k"], s["v"],
                                   rope=p["rope"], table=s["table"], positions=s["positions"], ld_pos=p["ld_pos"],
                                   axes=p["axes"], ids=s["ids"], q=s["q"], q_out=s["q_out"], pos=s["pos"],
                                   ld_s=s["pos"].shape[1])
        if fmt == E.KV_MXFP4:
            p["read"] = E.make_read_io(C, pool, 0, s["page_table"], width, s["n_cached"] - C,
                                       s["k_held"], s["v_held"])
        return p
    nbytes = E.attend_weigh_workspace_bytes(cfg, C, Hq, width, watch=c["watch"])
    ws = torch.empty(max(nbytes, 16), device=s["q"].device, dtype=torch.uint8)
    p["io"] = E.make_attend_io(C, pool, 0, s["page_table"], width, s["n_cached"], s["q"], s["out"],
                               lse=s["lse"], workspace=ws, workspace_bytes_=nbytes)
    p["weigh"] = E.make_weigh_io(s["weights"], s["weights"].shape[1], old=s["before"], keep_old=c["decay"],
                                 keep_new=0.0, watch=c["watch"])
    return p


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    p, c = s["plan"], s["case"]
    E = p["E"]
    if c["kind"] == "axes":
        E.epikv_rope_axes(p["rope"], p["axes"], s["table"], p["dtype"], c["batch"], c["chunk"], c["heads"],
                          c["head_dim"], p["x"], p["y"], s["positions"], p["ld_pos"], transpose=c["backward"])
        return s["y"]
    if c["kind"] == "append":
        E.epikv_append_axes(p["cfg"], p["io"])
        if c["fmt"] == "bf16":
            return {"pool": s["pool"], "q": s["q_out"], "pos": s["pos"]}
        E.epikv_read(p["cfg"], p["read"])
        return {"k": s["k_held"], "v": s["v_held"], "q": s["q_out"], "pos": s["pos"]}
    E.epikv_attend_weigh(p["cfg"], p["io"], p["weigh"])
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    B, C, Hq, d = c["batch"], c["chunk"], c["heads"], c["head_dim"]
    if c["kind"] != "weigh":
        r = 2 * sum(_pairs(c))
        where = 4 * r + 4 * len(_pairs(c))      # a token's cosines and sines, and positions
    if c["kind"] == "axes":
        size = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": B * C * (2 * Hq * d * size + where), "flops": 3 * B * C * Hq * r}
    H = c["kv_heads"]
    hd = H * d
    row = 2 * hd if c["fmt"] == "bf16" else hd // 2 + hd // 32
    if c["kind"] == "append":
        per = 2 * 2 * hd + 2 * row + 2 * 2 * Hq * d + where + 4
        if c["fmt"] != "bf16":
            per += 2 * row + 2 * 2 * hd  # read back
        return {"bytes": B * C * per, "flops": 3 * B * C * (Hq + H) * r}
    n = _lengths(c)
    seen = sum(C * (m - C) + C * (C + 1) // 2 for m in n)
    old = 4 * sum(m - C for m in n) if c["decay"] else 0
    return {"bytes": 2 * row * sum(n) + B * C * Hq * (2 * 2 * d + 4) + 4 * sum(n) + old, "flops": 4 * d * Hq * seen}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _rotated64(x, s, c, sign=1.0):
    """Each pair as a complex number times exp(i angle), axis by axis."""
    B, C, r = c["batch"], c["chunk"], 2 * sum(_pairs(c))
    axis = _axis_of(c)[0]
    position = s["positions"].view(B, -1, C).long()
    y = x.double().clone()
    even, odd = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous())
    for i, a in enumerate(axis):
        t = s["table"][:, i].double()[position[:, a]]
        z[..., i] *= torch.complex(t[..., 0], sign * t[..., 1])[..., None]
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _held64(x):
    """What 4-bit blocks of 32 along the last axis hold: the nearest level
    (ties to the even code) times the block's power of two."""
    shape = x.shape
    blk = x.reshape(-1, 32)
    top = blk.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2
    e = torch.where(top / 2.0 ** e > 7, e + 1, e).clamp(min=-126)
    a = (blk / 2.0 ** e).abs()
    levels = torch.tensor(LEVELS, device=x.device, dtype=torch.float64)
    best, at = torch.full_like(a, math.inf), torch.zeros_like(a)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):                      # even codes win ties
        off = (a - levels[i]).abs()
        nearer = off < best
        best, at = torch.where(nearer, off, best), torch.where(nearer, levels[i].expand_as(at), at)
    return (at * blk.sign() * 2.0 ** e).reshape(shape)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    B, C, Hq, d = c["batch"], c["chunk"], c["heads"], c["head_dim"]
    if c["kind"] == "axes":
        return _rotated64(s["x"], s, c, -1.0 if c["backward"] else 1.0)
    H, page = c["kv_heads"], c["page"]
    if c["kind"] == "append":
        k, q = _rotated64(s["k"], s, c), _rotated64(s["q"], s, c)
        if c["fmt"] != "bf16":
            return {"k": _held64(k), "v": _held64(s["v"].double()), "q": q, "pos": None}
        pool = s["pool"].double()
        for b, m in enumerate(_lengths(c)):
            slot = torch.arange(m - C, m, device=pool.device)
            pages = s["page_table"][b].long()[slot // page]
            pool[0, 0, pages, slot % page] = k[b]
            pool[0, 1, pages, slot % page] = s["v"][b].double()
        return {"pool": pool, "q": q, "pos": None}
    G = Hq // H
    dev = s["q"].device
    out = torch.empty(B, C, Hq, d, device=dev, dtype=torch.float64)
    lse = torch.empty(B, Hq, C, device=dev, dtype=torch.float64)
    sums = s["weights"].double()
    levels = torch.tensor(LEVELS, device=dev, dtype=torch.float64)
    for b, m in enumerate(_lengths(c)):
        slot = torch.arange(m, device=dev)
        rows = s["pool"][0][:, s["page_table"][b].long()[slot // page], slot % page]
        if c["fmt"] == "bf16":
            k, v = rows.double()
        else:
            n = H * d
            code = torch.empty(2, m, n, device=dev, dtype=torch.long)
            code[..., 0::2], code[..., 1::2] = rows[..., :n // 2] % 16, rows[..., :n // 2] // 16
            scale = 2.0 ** (rows[..., n // 2:n // 2 + n // 32].double() - 127)
            held = levels[code % 8] * (1 - 2 * (code // 8)) * scale.repeat_interleave(32, -1)
            k, v = held.view(2, m, H, d)
        seen = slot[None] <= (m - C + torch.arange(C, device=dev))[:, None]
        sums[b, :m] = 0.0
        sums[b, :m - C] = c["decay"] * s["before"][b, :m - C].double()
        for h in range(Hq):
            x = (s["q"][b, :, h].double() @ k[:, h // G].T) / math.sqrt(d)
            x = x.masked_fill(~seen, -math.inf)
            lse[b, h] = torch.logsumexp(x, -1)
            w = torch.exp(x - lse[b, h][:, None])
            out[b, :, h] = w @ v[:, h // G]
            sums[b, :m] += w[C - (c["watch"] or C):].sum(0)
    return {"out": out, "lse": lse, "weights": sums}

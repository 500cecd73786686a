"""Rotary positions on several axes: the table, the rotation and its gradient,
and appending, against the 64-bit oracle and against the calls of one axis."""
import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import DEV, Cache, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


MODES = {"plain": 0, "linear": 1, "ntk": 2, "bands": 3, "yarn": 4}
DEALS = [(16, 24, 24), (24, 20, 20), (1, 62, 1), (40, 24), (64,), (7, 19, 31, 7)]


def table_of(E, rope, axes):
    t = torch.full((rope.n_pos, rope.rotary_dim // 2, 2), float("nan"), device=DEV)
    E.epikv_rope_axes_table(rope, axes, t)
    return t


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("mode", sorted(MODES))
@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("pairs", [(16, 24, 24), (40, 24), (7, 19, 31, 7)])
def test_table(E, mode, apart, turns, pairs):
    """Rounded once from 64 bits: half a unit in the last place, and the 64-bit
    angle's own error."""
    high = 32.0 if mode == "yarn" else 4.0
    rope = E.default_rope(rotary_dim=128, n_pos=3001, theta=500000.0, scaling=MODES[mode], factor=8.0, original=8192,
                          turns_low=1.0, turns_high=high, amplitude=1.25)
    got = f64(table_of(E, rope, E.axes_of(pairs, order=int(turns), frequencies=int(apart))))
    f = R.rope_axes_frequencies(pairs, turns, apart, 500000.0, mode, factor=8.0, original=8192, low=1.0, high=high)
    ang = np.arange(3001)[:, None] * f
    ref = 1.25 * np.stack([np.cos(ang), np.sin(ang)], -1)
    assert np.abs(got - ref).max() <= 2.0 ** -23 * 1.25 / 2 + 1e-10


def rows_for(table, pairs, turns, pos):
    """[B][C][pairs][2] of positions [B][axes][C]: each pair's own row."""
    axis = np.array(R.axes_of_pairs(pairs, turns)[0])
    return table[np.moveaxis(pos[:, axis], 1, 2), np.arange(len(axis))]


def steps(x, cs, r, il, transpose):
    """The float32 steps: two products and a sum, each rounded."""
    c, s = cs[..., 0].unsqueeze(2), cs[..., 1].unsqueeze(2)
    s = -s if transpose else s
    xf, want = x.float(), x.float().clone()
    lo, hi = (slice(0, r, 2), slice(1, r, 2)) if il else (slice(0, r // 2), slice(r // 2, r))
    a, b = xf[..., lo], xf[..., hi]
    want[..., lo], want[..., hi] = a * c - b * s, b * c + a * s
    return want.to(x.dtype)


SHAPES = [(1, 1, 1, 16, 16, (3, 5)), (32, 1, 32, 128, 128, (16, 24, 24)), (2, 37, 5, 64, 32, (5, 7, 4)),
          (3, 11, 7, 256, 64, (8, 8, 8, 8)), (1, 300, 8, 128, 128, (24, 20, 20)), (2, 3, 3, 80, 48, (11, 13)),
          (5, 2, 40, 96, 96, (48,)), (1, 7, 1, 1024, 1024, (100, 200, 12, 200)), (2, 9, 16, 64, 64, (16, 16))]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotation(E, shape, il, turns, transpose, dtype):
    """Bit for bit the float32 steps, which are 3 2^-24 of the magnitudes off
    the 64-bit rotation and, in bf16, 2^-8 of the result."""
    B, C, heads, d, r, pairs = shape
    g = torch.Generator().manual_seed(B * 100 + d)
    x = torch.randn(B, C, heads, d, generator=g) * torch.exp(torch.randn(d, generator=g))
    x = x.bfloat16() if dtype == "bf16" else x
    rope = E.default_rope(rotary_dim=r, n_pos=500, layout=int(il))
    axes = E.axes_of(pairs, order=int(turns), frequencies=(B + d) % 2)
    table = table_of(E, rope, axes)
    th, dt = table.cpu(), E.DTYPE_BF16 if dtype == "bf16" else E.DTYPE_FP32
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    for per_token in (False, True):
        if per_token:
            given = torch.randint(0, 500, (B, len(pairs), C + 3), generator=g, dtype=torch.int32)
            pos, ld = given[..., :C].numpy(), C + 3
        else:
            given = torch.randint(0, 500 - C + 1, (B, len(pairs)), generator=g, dtype=torch.int32)
            pos, ld = given.numpy()[..., None] + np.arange(C), 0
        xd, y = x.to(DEV), torch.full_like(x, float("nan")).to(DEV)
        E.epikv_rope_axes(rope, axes, table, dt, B, C, heads, d, xd, y, given.to(DEV), ld, transpose=transpose,
                          seq_status=status)
        cs = torch.from_numpy(rows_for(th.numpy(), pairs, turns, pos))
        assert same(steps(x, cs, r, il, transpose), y.cpu())
        t = cs.double().numpy()
        ref = R.rotate(f64(x), t[..., 0], t[..., 1], il, transpose)
        a = np.abs(t)
        big = np.maximum(np.abs(R.rotate(np.abs(f64(x)), a[..., 0], a[..., 1], il, True)),
                         np.abs(R.rotate(np.abs(f64(x)), a[..., 0], a[..., 1], il)))
        tol = 3 * 2.0 ** -24 * (big + np.abs(ref)) + (2.0 ** -8 * np.abs(ref) * 1.01 if dtype == "bf16" else 0)
        assert np.all(np.abs(f64(y) - ref) <= tol + 1e-38)
        E.epikv_rope_axes(rope, axes, table, dt, B, C, heads, d, xd, xd, given.to(DEV), ld, transpose=transpose)
        assert same(xd, y)
    assert not status.any().item()


@pytest.mark.parametrize("pairs", DEALS)
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("il", [False, True])
def test_equal_positions_are_one_axis(E, pairs, turns, il):
    B, C, heads, d = 3, 5, 6, 128
    rope, axes = E.default_rope(n_pos=300, layout=int(il)), E.axes_of(pairs, order=int(turns))
    table, plain = table_of(E, rope, axes), torch.empty(300, 64, 2, device=DEV)
    E.epikv_rope_table(rope, plain)
    assert same(table, plain)
    x = torch.randn(B, C, heads, d, device=DEV).bfloat16()
    first = torch.tensor([0, 295, 77], dtype=torch.int32, device=DEV)
    a, b = torch.empty_like(x), torch.empty_like(x)
    E.epikv_rope(rope, plain, E.DTYPE_BF16, B, C, heads, d, x, a, first)
    E.epikv_rope_axes(rope, axes, table, E.DTYPE_BF16, B, C, heads, d, x, b,
                      first[:, None].expand(-1, len(pairs)).contiguous())
    assert same(a, b)


@pytest.mark.parametrize("il", [0, 1])
@pytest.mark.parametrize("turns", [0, 1])
def test_gradient_is_the_derivative(E, il, turns):
    B, C, heads, d, pairs = 2, 5, 3, 64, (5, 9, 10)
    g = torch.Generator().manual_seed(3)
    rope, axes = E.default_rope(rotary_dim=48, n_pos=64, layout=il, amplitude=1.125), E.axes_of(pairs, order=turns)
    table = table_of(E, rope, axes)
    pos = torch.randint(0, 64, (B, 3, C), generator=g, dtype=torch.int32).to(DEV)

    def run(v, tr=False):
        out = torch.empty_like(v)
        E.epikv_rope_axes(rope, axes, table, E.DTYPE_FP32, B, C, heads, d, v, out, pos, C, transpose=tr)
        return out
    x, e, w = (torch.randn(B, C, heads, d, generator=g).to(DEV) for _ in range(3))
    h = 1.0 / 64
    diff = (run(x + h * e).double() - run(x - h * e).double()) / (2 * h)
    num = (w.double() * diff).sum().item()
    ana = (run(w, True).double() * e.double()).sum().item()
    # 1920 terms of size ~1, each off by a few 2^-24 / h
    assert abs(num - ana) <= 1920 * 8 * 2.0 ** -24 * 64
    cs = rows_for(f64(table), pairs, bool(turns), pos.cpu().numpy())
    assert np.abs(f64(run(w, True)) - R.rotate(f64(w), cs[..., 0], cs[..., 1], bool(il), True)).max() <= 2.0 ** -20


def test_strides(E):
    """A view into a fused projection into a transposed output."""
    B, C, heads, d, pairs = 2, 9, 4, 64, (9, 11, 12)
    fused = torch.randn(B, C, heads + 3, d, device=DEV).bfloat16()
    x = fused[:, :, 2:2 + heads]
    y = torch.zeros(B, heads, C, d, device=DEV, dtype=torch.bfloat16)
    rope, axes = E.default_rope(rotary_dim=64, n_pos=100), E.axes_of(pairs, order=E.AXES_TURNS)
    table = table_of(E, rope, axes)
    pos = torch.randint(0, 100, (B, 3, C), dtype=torch.int32, device=DEV)
    E.epikv_rope_axes(rope, axes, table, E.DTYPE_BF16, B, C, heads, d, x, y.transpose(1, 2), pos, C)
    z = torch.empty(B, C, heads, d, device=DEV, dtype=torch.bfloat16)
    E.epikv_rope_axes(rope, axes, table, E.DTYPE_BF16, B, C, heads, d, x.contiguous(), z, pos, C)
    assert same(z, y.transpose(1, 2))


def test_positions_out_of_range_leave_the_token(E):
    """On any axis."""
    B, C, heads, d = 4, 4, 2, 32
    x = torch.randn(B, C, heads, d, device=DEV)
    y = torch.full_like(x, 7.0)
    rope, axes = E.default_rope(rotary_dim=32, n_pos=10), E.axes_of((4, 5, 7))
    table = table_of(E, rope, axes)
    first = torch.tensor([[0, 8, 0], [3, 2, -2], [6, 6, 6], [2 ** 31 - 1, 0, 0]], dtype=torch.int32, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    E.epikv_rope_axes(rope, axes, table, E.DTYPE_FP32, B, C, heads, d, x, y, first, seq_status=status)
    assert status.tolist() == [2, 2, 0, 2]
    left = (y == 7.0).flatten(2).all(-1).cpu().numpy()
    assert left.tolist() == [[False, False, True, True], [True, True, False, False], [False] * 4, [True] * 4]


def test_large_tables(E):
    """Entries past 2^32 bytes: the largest n_pos."""
    rope, axes = E.default_rope(rotary_dim=64, n_pos=1 << 24, theta=1e6), E.axes_of((10, 11, 11), order=E.AXES_TURNS)
    table = table_of(E, rope, axes)
    x = torch.randn(1, 1, 2, 64, device=DEV)
    y = torch.empty_like(x)
    at = [(1 << 24) - 1, 5, (1 << 24) - 9]
    E.epikv_rope_axes(rope, axes, table, E.DTYPE_FP32, 1, 1, 2, 64, x, y, torch.tensor([at], dtype=torch.int32, device=DEV))
    axis = R.axes_of_pairs((10, 11, 11), True)[0]
    cs = torch.stack([table[at[a], i] for i, a in enumerate(axis)]).cpu()[None, None]
    assert same(steps(x.cpu(), cs, 64, False, False), y.cpu())


# ---------------------------------------------------------------------------
# Appending
# ---------------------------------------------------------------------------
def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Appended:
    """One append of B sequences' chunk, with positions on several axes, or by
    a table made of each token's own turns, position = its number (`plain`)."""

    def __init__(self, E, fmt, heads, pairs, turns, il, per_token, plain, B=3, C=5, page=4, queries=True, in_place=False,
                 side=None):
        Hq, H, d = heads
        g = torch.Generator().manual_seed(d + C)
        rng = np.random.default_rng(d)
        r = 2 * sum(pairs)
        self.n, self.nn = [C, C + 20, 3], [C, C, 2]
        c = self.c = Cache(E, rng, fmt, B, H, d, page, 40)
        rope = E.default_rope(rotary_dim=r, n_pos=200, layout=int(il))
        axes = E.axes_of(pairs, order=int(turns))
        table = table_of(E, rope, axes)
        if per_token:
            given = torch.randint(0, 200, (B, len(pairs), C + 1), generator=g, dtype=torch.int32)
            pos, ld = given[..., :C].numpy(), C + 1
        else:
            given = torch.randint(0, 200 - C, (B, len(pairs)), generator=g, dtype=torch.int32)
            pos, ld = given.numpy()[..., None] + np.arange(C), 0

        def rand(h):
            return torch.randn(B, C, h, d, generator=g).bfloat16().to(DEV)
        self.q, self.k, self.v = rand(Hq), rand(H), rand(H)
        self.q_out = self.q if in_place else torch.full_like(self.q, 5.0)
        self.pos = torch.full((B, 40), -1, dtype=torch.int32, device=DEV)
        self.status = ints([0] * B)
        ids = torch.randint(0, 10 ** 6, (B, C), generator=g, dtype=torch.int32)
        self.ids = ids.numpy()
        kw = dict(n_new=ints(self.nn), seq_status=self.status)
        if queries:
            kw.update(q=self.q, q_out=self.q_out)
        call = E.epikv_append_axes
        if plain:
            rows = torch.from_numpy(rows_for(table.cpu().numpy(), pairs, turns, pos)).reshape(B * C, r // 2, 2)
            rope = E.default_rope(rotary_dim=r, n_pos=B * C, layout=int(il))
            kw.update(rope=rope, table=rows.contiguous().to(DEV), positions=ints([b * C for b in range(B)]))
            call = E.epikv_append
        else:
            kw.update(rope=rope, table=table, positions=given.to(DEV), ld_pos=ld, axes=axes, ids=ids.to(DEV), ld_ids=C,
                      pos=self.pos, ld_s=40)
        io = E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(self.n), self.k, self.v, **kw)
        call(c.cfg, io, stream=side)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("heads,pairs", [((8, 2, 128), (16, 24, 24)), ((7, 1, 64), (3, 29)), ((6, 3, 64), (5, 5, 6)),
                                         ((4, 4, 256), (60, 30, 20, 18)), ((5, 5, 128), (1, 63))])
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("per_token", [False, True])
def test_append(E, fmt, heads, pairs, turns, il, per_token):
    """Byte for byte the append of one axis by a table of each token's own
    turns: rows, queries; and the ids beside them."""
    a = Appended(E, fmt, heads, pairs, turns, il, per_token, False)
    b = Appended(E, fmt, heads, pairs, turns, il, per_token, True)
    assert same(a.c.bytes, b.c.bytes) and same(a.q_out, b.q_out)
    assert not a.status.any().item()
    ids = a.pos.cpu().numpy()
    for s in range(3):
        first = a.n[s] - a.nn[s]
        assert np.array_equal(ids[s, first:a.n[s]], a.ids[s, :a.nn[s]])
        assert np.all(ids[s, :first] == -1) and np.all(ids[s, a.n[s]:] == -1)


def test_append_other_forms(E):
    """Without queries, in place, on another stream."""
    args = (0, (8, 2, 128), (16, 24, 24), True, False, True)
    a = Appended(E, *args, False)
    b = Appended(E, *args, False, queries=False)
    c = Appended(E, *args, False, in_place=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    d = Appended(E, *args, False, side=side)
    torch.cuda.synchronize()
    for x in (b, c, d):
        assert same(a.c.bytes, x.c.bytes) and same(a.pos, x.pos)
    for s in range(3):
        assert same(a.q_out[s, :a.nn[s]], c.q_out[s, :a.nn[s]]) and same(a.q_out[s], d.q_out[s])


def test_append_out_of_range(E):
    """A position out of range on one axis leaves the token out; ids may be
    left away; a slot without a place for its id flags."""
    B, C, H, d = 3, 2, 2, 64
    rng = np.random.default_rng(1)
    rope, axes = E.default_rope(rotary_dim=64, n_pos=50), E.axes_of((10, 11, 11))
    table = table_of(E, rope, axes)
    c = Cache(E, rng, E.KV_BF16, B, H, d, 4, 16)
    k, v = (torch.randn(B, C, H, d, device=DEV).bfloat16() for _ in range(2))
    n, pos = ints([2, 9, 16]), ints([[0, 49, 0], [0, 0, 0], [1, 2, 3]])
    status, before = ints([0] * B), c.bytes.clone()
    E.epikv_append_axes(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, n, k, v, rope=rope, table=table,
                                                positions=pos, axes=axes, seq_status=status))
    assert status.tolist() == [2, 0, 0]
    assert (c.rows(0, 0, 2)[1] == 255).all() and not (c.rows(0, 0, 1) == 255).all() and not same(before, c.bytes)
    status.zero_()
    ids = torch.full((B, 15), -1, dtype=torch.int32, device=DEV)
    E.epikv_append_axes(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, n, k, v, rope=rope, table=table,
                                                positions=pos, axes=axes, ids=ints([100, 200, 300]), pos=ids, ld_s=15,
                                                seq_status=status))
    assert status.tolist() == [2, 0, 2]
    assert ids[0].tolist() == [100] + [-1] * 14 and ids[1, 7:9].tolist() == [200, 201] and ids[2, 14].item() == 300


def test_graph(E):
    """Captured once, replayed with other positions: the eager call's bytes."""
    B, C, H, Hq, d = 2, 3, 2, 4, 64
    rope, axes = E.default_rope(rotary_dim=64, n_pos=90), E.axes_of((10, 11, 11), order=E.AXES_TURNS)
    table = table_of(E, rope, axes)

    def buffers():
        c = Cache(E, np.random.default_rng(2), E.KV_MXFP4, B, H, d, 4, 16)
        q, k, v = (torch.zeros(B, C, h, d, device=DEV, dtype=torch.bfloat16) for h in (Hq, H, H))
        s = dict(c=c, q=q, k=k, v=v, n=ints([3, 8]), positions=ints([[0] * 3] * B), ids=ints([0, 0]),
                 q_out=torch.zeros_like(q), pos=torch.zeros(B, 16, dtype=torch.int32, device=DEV), y=torch.zeros_like(q))
        s["io"] = E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, s["n"], k, v, rope=rope, table=table,
                                   positions=s["positions"], axes=axes, ids=s["ids"], q=q, q_out=s["q_out"], pos=s["pos"],
                                   ld_s=16)
        return s

    def run(s):
        E.epikv_append_axes(s["c"].cfg, s["io"])
        E.epikv_rope_axes(rope, axes, table, E.DTYPE_BF16, B, C, Hq, d, s["q"], s["y"], s["positions"], transpose=True)
    a, b = buffers(), buffers()
    run(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(b)
    b["c"].bytes.copy_(a["c"].bytes)
    b["pos"].zero_()
    for step in range(4):
        new = {k: torch.randn(a[k].shape, device=DEV).bfloat16() for k in ("q", "k", "v")}
        new.update(positions=torch.randint(0, 87, (B, 3), device=DEV).int(), ids=ints([7 * step, 3]),
                   n=ints([3 + step, 8 + 2 * step]))
        for s in (a, b):
            for key, t in new.items():
                s[key].copy_(t)
        run(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(a["c"].bytes, b["c"].bytes) and all(same(a[k], b[k]) for k in ("q_out", "pos", "y")), step

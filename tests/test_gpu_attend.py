"""Attention over the paged cache against the 64-bit oracle."""
import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import DEV, Cache, bf16, f64

pytestmark = pytest.mark.gpu
FMTS = ["bf16", "mxfp4"]


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def run(E, c, C, n, q, nn=None, table=None, out=None, scale=0.0, stream=None, noise=0xA5):
    B, _, Hq, d = q.shape
    need = E.attend_workspace_bytes(c.cfg, C, Hq)
    ws = torch.full((max(need, 16),), noise, dtype=torch.uint8, device=DEV)
    out = torch.full((B, C, Hq, d), 9.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    lse = torch.full((B, Hq, C), 9.0, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    io = E.make_attend_io(C, c.pool, c.layer, c.table if table is None else table, c.ld_pt, ints(n), q, out,
                          n_new=None if nn is None else ints(nn), lse=lse, scale=scale,
                          seq_status=status, workspace=ws, workspace_bytes_=need)
    E.epikv_attend(c.cfg, io, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    return out, lse, status


def bounds(out, lse, mag, size, d):
    """Scores: products of bf16 are exact in float32, their sum of d terms and
    the scaling cost (d + 4) 2^-24 of the largest sum of magnitudes; exp2 and
    the sums a few 2^-22.  The weights' rounding to bf16 (8 significant bits)
    costs 2^-8 of the weighted mean of |v|, the result's 2^-8 of itself."""
    eps = (d + 4) * 2.0 ** -24 * size + 2.0 ** -20
    per = np.moveaxis(eps, -1, 0)[..., None]                       # [C][Hq][1]
    tol_out = 1.01 * 2.0 ** -8 * (mag + np.abs(out)) + 3 * per * mag + 1e-37
    tol_lse = eps + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))
    return tol_out, tol_lse


def check(E, fmt, B, C, Hq, H, d, page, n, nn=None, seed=0, ok=None, spread=1.0, scale=0.0, layers=1,
          edit=None, **cache):
    fmt = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(seed + 17 * C + d)
    c = Cache(E, rng, fmt, B, H, d, page, max(max(n), 1), layers=layers, layer=layers - 1, **cache)
    q, q64 = bf16(rng.standard_normal((B, C, Hq, d)) * spread)
    held = []
    for b in range(B):
        kv = [rng.standard_normal((n[b], H, d)) * np.exp(0.5 * rng.standard_normal((H, d)))
              for _ in range(2)]
        if edit:
            edit(b, *kv)
        got = []
        for i in range(2):
            raw, val = c.encode(kv[i])
            c.fill_rows(b, i, raw)
            got.append(val)
        held.append(got)
    out, lse, status = run(E, c, C, n, q, nn, scale=scale)
    again = run(E, c, C, n, q, nn, scale=scale, noise=0x5A)
    assert torch.equal(out.view(torch.int16), again[0].view(torch.int16))
    assert torch.equal(lse.view(torch.int32), again[1].view(torch.int32))
    assert not status.any().item()
    out, lse = f64(out), f64(lse)
    for b in range(B):
        m = C if nn is None else nn[b]
        with np.errstate(invalid="ignore", over="ignore"):
            ro, rl, mag, size = R.attend(q64[b, :m], *held[b], m, scale or d ** -0.5)
            to, tl = bounds(ro, rl, mag, size, d)
        bad = np.isnan(ro)
        assert np.array_equal(np.isnan(out[b, :m]), bad)
        assert np.all((np.abs(out[b, :m] - ro) <= to) | bad), (b, np.nanmax(np.abs(out[b, :m] - ro) / to))
        fin = np.isfinite(rl)
        assert np.array_equal(np.isfinite(lse[b, :, :m]), fin)
        assert np.all((np.abs(lse[b, :, :m] - rl) <= tl) | ~fin)
        assert np.all(out[b, m:] == 0) and np.all(lse[b, :, m:] == -np.inf)
    return c


LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 8, 64), (16, 2, 256), (7, 1, 64), (40, 8, 128),
                                   (6, 3, 128), (17, 1, 128), (36, 12, 128), (64, 32, 64)])
def test_single_tokens(E, fmt, heads):
    """Every length around a tile's and a page's end, with an empty sequence."""
    n = [0] + LENGTHS
    check(E, fmt, len(n), 1, *heads, 16, n, nn=[0] + [1] * len(LENGTHS))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [1, 3, 12, 48, 64, 1024])
def test_pages(E, fmt, page):
    check(E, fmt, 3, 2, 8, 2, 128, page, [2, 130, 777], seed=page, gap=48, layers=2)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [2, 3, 5, 8])
@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 4, 64), (24, 2, 128), (8, 2, 256)])
def test_short_chunks(E, fmt, C, heads):
    n = [C, C + 1, 33, 64, 200, 129]
    nn = [C, C, 1, C - 1, C, 0]
    check(E, fmt, 6, C, *heads, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,n,nn", [
    (17, [17, 400, 100], [17, 17, 3]), (33, [33, 65], None), (64, [64, 1000], [64, 63]),
    (100, [100, 163], None), (129, [129, 500], [129, 1]), (300, [300], None), (300, [812], None),
    (257, [300, 257, 1], [257, 130, 0])])
@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 1, 64), (2, 2, 256), (5, 1, 128)])
def test_chunks(E, fmt, C, n, nn, heads):
    check(E, fmt, len(n), C, *heads, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
def test_long_sequence_alone(E, fmt):
    """One sequence over many workgroups, joined; and ragged neighbours."""
    check(E, fmt, 1, 1, 4, 1, 128, 16, [20011])
    check(E, fmt, 5, 1, 8, 2, 64, 16, [9001, 1, 0, 64, 12345], [1, 1, 0, 1, 1])


@pytest.mark.parametrize("fmt", FMTS)
def test_large_batches(E, fmt):
    """More sequences than are cut into shares."""
    rng = np.random.default_rng(4)
    n = rng.integers(0, 90, 300).tolist()
    check(E, fmt, 300, 1, 4, 2, 64, 16, n, [min(x, 1) for x in n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 4, 70])
def test_peaked_and_flat_scores(E, fmt, C):
    """Scores from 1e3 to none: a late token that takes all, growing maxima,
    equal scores."""
    def late(b, k, v):
        if b == 0:
            k[-C - 1:] *= 30
        elif b == 1:
            k *= np.linspace(0, 10, k.shape[0])[:, None, None]
        else:
            k[:] = 0.5
    check(E, fmt, 3, C, 8, 2, 128, 16, [300, 517, 201], spread=4.0, edit=late)
    check(E, fmt, 2, C, 8, 2, 128, 16, [300, 97], scale=1e-6)
    check(E, fmt, 2, C, 8, 2, 64, 16, [300, 97], scale=2.5)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,Hq,H,d", [(1, 8, 2, 128), (5, 8, 2, 128), (3, 4, 4, 64), (2, 8, 2, 256),
                                      (40, 8, 2, 128), (200, 4, 1, 64), (70, 2, 1, 256)])
def test_hidden_slots_hold_anything(E, fmt, C, Hq, H, d):
    """NaN and infinities in a later token's key and value do not reach the
    tokens before it; they do reach those that see them.  (Unused bytes of
    every page are NaN throughout these tests.)"""
    n = [C + 50, C + 3]

    def edit(b, k, v):
        at = n[b] - C + C // 2 + (1 if C > 1 else 0)
        if at < n[b]:
            k[at, 0, 3] = np.nan
            v[at, H - 1, 5], v[at, 0, 9] = np.nan, np.inf
    check(E, fmt, 2, C, Hq, H, d, 16, n, edit=edit)


@pytest.mark.parametrize("C,n", [(1, 40), (1, 5000), (4, 3000), (40, 3000), (200, 300)])
def test_nan_and_infinity_that_are_seen(E, C, n):
    """A NaN query, a NaN key, an infinite value and an infinite score reach
    exactly the rows that the definition lets them reach."""
    B, Hq, H, d = 4, 4, 2, 128
    rng = np.random.default_rng(n)
    c = Cache(E, rng, E.KV_BF16, B, H, d, 16, n)
    q = rng.standard_normal((B, C, Hq, d))
    q[0, C - 1, 1, 7] = np.nan
    kv = rng.standard_normal((B, 2, n, H, d))
    kv[1, 0, n // 2, 0, 3] = np.nan
    kv[2, 1, n // 3, 1, 5] = np.inf
    kv[3, 0, n // 4, 1, 6] = np.inf
    qd, q64 = bf16(q)
    held = []
    for b in range(B):
        got = []
        for i in range(2):
            raw, val = c.encode(kv[b, i])
            c.fill_rows(b, i, raw)
            got.append(val)
        held.append(got)
    out, lse, _ = run(E, c, C, [n] * B, qd)
    out = f64(out)
    for b in range(B):
        with np.errstate(invalid="ignore", over="ignore"):
            ro, rl, mag, size = R.attend(q64[b], *held[b], C, d ** -0.5)
            to, _ = bounds(ro, rl, mag, size, d)
        assert np.array_equal(np.isnan(out[b]), np.isnan(ro))
        assert np.array_equal(np.isinf(out[b]), np.isinf(ro))
        fine = np.isfinite(ro)
        assert np.all(np.abs(out[b] - ro)[fine] <= to[fine])


@pytest.mark.parametrize("C,n", [(1, 1), (1, 33), (1, 700), (1, 5000), (1, 40000), (3, 9000),
                                 (40, 3000)])
def test_infinite_value_in_the_last_slot(E, C, n):
    """An infinity stays one however the sequence is cut and joined."""
    Hq, H, d = 4, 2, 128
    rng = np.random.default_rng(n)
    c = Cache(E, rng, E.KV_BF16, 1, H, d, 16, n)
    q, q64 = bf16(rng.standard_normal((1, C, Hq, d)))
    kv = rng.standard_normal((2, n, H, d))
    kv[1, n - 1, 0, 5], kv[1, n - 1, 1, 6] = np.inf, -np.inf
    held = []
    for i in range(2):
        raw, val = c.encode(kv[i])
        c.fill_rows(0, i, raw)
        held.append(val)
    out = f64(run(E, c, C, [n], q)[0])[0]
    ro, rl, mag, size = R.attend(q64[0], *held, C, d ** -0.5)
    to, _ = bounds(ro, rl, mag, size, d)
    fine = np.isfinite(ro)
    assert np.array_equal(out[~fine], ro[~fine])
    assert np.all(np.abs(out - ro)[fine] <= to[fine])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,heads", [(1, (4, 2, 64)), (3, (8, 2, 128)), (1, (2, 1, 256))])
def test_batches_past_a_thousand(E, fmt, C, heads):
    """More sequences than are cut into shares, whose outputs are written
    without a join."""
    rng = np.random.default_rng(11)
    n = rng.integers(0, 60, 1100).tolist()
    n[5], n[1099] = 0, 400
    check(E, fmt, 1100, C, *heads, 16, n, [min(x, C) for x in n])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 6, 90])
def test_pages_out_of_range_are_left_out(E, fmt, C):
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(C)
    B, Hq, H, d, page = 4, 8, 2, 128, 16
    n = [C + 170, C + 40, 5000, C - 1]
    nn = [C, C, C, C]
    c = Cache(E, rng, fm, B, H, d, page, max(n[:2]))
    q, q64 = bf16(rng.standard_normal((B, C, Hq, d)))
    held = []
    for b in range(2):
        got = []
        for i in range(2):
            raw, val = c.encode(rng.standard_normal((n[b], H, d)))
            c.fill_rows(b, i, raw)
            got.append(val)
        held.append(got)
    table = c.table.clone()
    table[0, 3], table[0, 7] = -1, 2 ** 30
    table[1, :] = 10 ** 9
    out, lse, status = run(E, c, C, n, q, nn, table=table)
    assert status.tolist() == [2, 2, 2, 2]
    ok = np.ones(n[0], bool)
    ok[48:64] = ok[112:128] = False
    ro, rl, mag, size = R.attend(q64[0], *held[0], C, d ** -0.5, ok)
    to, tl = bounds(ro, rl, mag, size, d)
    assert np.all(np.abs(f64(out)[0] - ro) <= to) and np.all(np.abs(f64(lse)[0] - rl) <= tl)
    for b in (1, 2, 3):  # nothing to see, a length past the table, more new than cached
        assert not out[b].any().item() and torch.all(lse[b] == -float("inf"))


def test_strides(E):
    """Queries of a fused projection, outputs [B][heads][chunk][d]."""
    rng = np.random.default_rng(9)
    for C in (1, 3, 50):
        B, Hq, H, d = 2, 8, 2, 64
        n = [C + 20, C + 90]
        c = Cache(E, rng, E.KV_BF16, B, H, d, 16, max(n), fill=0)
        for b in range(B):
            for i in range(2):
                c.fill_rows(b, i, c.encode(rng.standard_normal((n[b], H, d)))[0])
        fused = torch.randn(B, C, Hq + 4, d, device=DEV).bfloat16()
        q = fused[:, :, 1:1 + Hq]
        a, la, _ = run(E, c, C, n, q.contiguous())
        room = torch.full((B, Hq, C, d), 9.0, dtype=torch.bfloat16, device=DEV)
        o, lo, _ = run(E, c, C, n, q, out=room.transpose(1, 2))
        assert torch.equal(a, o) and torch.equal(la, lo)
        one = torch.randn(1, C, Hq, d, device=DEV).bfloat16()
        x = run(E, c, C, n, one.expand(B, C, Hq, d))[0]
        y = run(E, c, C, n, one.expand(B, C, Hq, d).contiguous())[0]
        assert torch.equal(x, y)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 48])
def test_other_streams_and_graphs(E, fmt, C):
    """On a stream of its own, and captured: replays with eager work between
    them give the eager call's bits."""
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(3)
    B, Hq, H, d = 3, 8, 2, 128
    n = [C + 500, C + 2, C + 3000]
    c = Cache(E, rng, fm, B, H, d, 16, max(n))
    for b in range(B):
        for i in range(2):
            c.fill_rows(b, i, c.encode(rng.standard_normal((n[b], H, d)))[0])
    q = torch.randn(B, C, Hq, d, device=DEV).bfloat16()
    want, wl, _ = run(E, c, C, n, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, gl, _ = run(E, c, C, n, q, stream=side)
    assert torch.equal(want, got) and torch.equal(wl, gl)
    need = E.attend_workspace_bytes(c.cfg, C, Hq)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device=DEV)
    out, lse, nd = torch.zeros_like(want), torch.zeros_like(wl), ints(n)
    io = E.make_attend_io(C, c.pool, 0, c.table, c.ld_pt, nd, q, out, lse=lse, workspace=ws,
                          workspace_bytes_=need)
    E.epikv_attend(c.cfg, io)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.epikv_attend(c.cfg, io)
    for i in range(4):
        out.zero_()
        lse.zero_()
        ws.fill_(i * 37)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl)


def test_rows_past_four_gigabytes(E):
    """Offsets past 32 bits inside a plane, both formats."""
    for fmt in (E.KV_BF16, E.KV_MXFP4):
        rng = np.random.default_rng(8)
        H, d, page, n_pages, Hq = 1, 64, 1024, 40000, 4
        cfg = E.default_cfg(batch=1, n_layers=1, n_kv_heads=H, head_dim=d, page_size=page, kv_format=fmt)
        stride = page * E.kv_row_bytes(cfg)
        big = torch.zeros(2 * n_pages * stride, dtype=torch.uint8, device=DEV)
        c = Cache(E, rng, fmt, 1, H, d, page, 1200)
        n = 1100
        for i in range(2):
            c.fill_rows(0, i, c.encode(rng.standard_normal((n, H, d)))[0])
        for C in (1, 40):
            q = torch.randn(1, C, Hq, d, device=DEV).bfloat16()
            want, wl, _ = run(E, c, C, [n], q)
            view = big.view(2, n_pages, stride)
            pages = ints([[39999, 35000]])
            for m in range(2):
                view[:, int(pages[0, m])] = c.bytes[0, :, int(c.table_host[0, m])]
            c2 = type("C2", (), dict(cfg=cfg, pool=E.Pool(big.data_ptr(), 0, n_pages * stride, stride, n_pages),
                                     layer=0, table=pages, ld_pt=2))
            got, gl, _ = run(E, c2, C, [n], q)
            assert torch.equal(want, got) and torch.equal(wl, gl)
        del big


@pytest.mark.parametrize("seed", range(16))
def test_random_mixes(E, seed):
    rng = np.random.default_rng(1000 + seed)
    d = int(rng.choice([64, 128, 256]))
    H = int(rng.choice([1, 2, 3, 4]))
    G = int(rng.choice([1, 2, 3, 4, 6, 8, 11]))
    C = int(rng.choice([1, 1, 2, 3, 7, 16, 31, 64, 130]))
    B = int(rng.integers(1, 6))
    nn = [int(rng.integers(0, C + 1)) for _ in range(B)]
    n = [x + int(rng.integers(0, 700)) for x in nn]
    check(E, FMTS[seed % 2], B, C, G * H, H, d, int(rng.choice([1, 7, 16, 32, 100])), n, nn, seed=seed)

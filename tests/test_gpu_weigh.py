"""Attention that sums its weights per slot, against the 64-bit oracle."""
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


def attend_only(E, c, C, n, q, nn=None, table=None, scale=0.0):
    B, _, Hq, d = q.shape
    need = E.attend_workspace_bytes(c.cfg, C, Hq)
    ws = torch.full((max(need, 16),), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty(q.shape, dtype=q.dtype, device=DEV), torch.empty(B, Hq, C, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    E.epikv_attend(c.cfg, E.make_attend_io(C, c.pool, c.layer, c.table if table is None else table, c.ld_pt, ints(n), q,
                                           out, n_new=None if nn is None else ints(nn), lse=lse, scale=scale,
                                           seq_status=status, workspace=ws, workspace_bytes_=need))
    return out, lse, status


def run(E, c, C, n, q, nn=None, table=None, scale=0.0, stream=None, noise=0xA5, weights=None, old=None, ld_s=None,
        with_lse=True, out=None, watch=0, **kw):
    """(The workspace is exactly as large as asked for, between two bands that
    no call may write.)"""
    B, _, Hq, d = q.shape
    need = E.attend_weigh_workspace_bytes(c.cfg, C, Hq, c.ld_pt, watch)
    room = torch.full((256 + need + 256,), noise, dtype=torch.uint8, device=DEV)
    ws = room[256:256 + need]
    out = torch.full((B, C, Hq, d), 9.0, dtype=torch.bfloat16, device=DEV) if out is None else out
    lse = torch.full((B, Hq, C), 9.0, device=DEV) if with_lse else None
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    io = E.make_attend_io(C, c.pool, c.layer, c.table if table is None else table, c.ld_pt, ints(n), q, out,
                          n_new=None if nn is None else ints(nn), lse=lse, scale=scale,
                          seq_status=status, workspace=ws, workspace_bytes_=need)
    E.epikv_attend_weigh(c.cfg, io, E.make_weigh_io(weights, ld_s or weights.shape[1], old=old, watch=watch, **kw),
                         stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    assert torch.all(room[:256] == noise) and torch.all(room[256 + need:] == noise)
    return out, lse, status


def expected(q64, k, v, m, scale, old, keep_old, keep_new, gain, watch, ok=None):
    """The sums and how far they may be off: a row's score by eps = (d + 4)
    2^-24 of its largest sum of magnitudes and 2^-20 for exp2 (as the
    attention's own bound counts), its log-sum by that and 2^-20 (1 + |lse|) for
    the logarithm and the change of base; the weight by both, of itself; the
    sum by 2^-24 of itself for each term."""
    d = k.shape[2]
    w = R.attend_weights(q64, k, m, scale, ok)
    _, lse, _, _ = R.attend(q64, k, v, m, scale, ok)
    # (an infinite key's score is -infinity where its row counts, and its weight
    # exactly 0: the rounding is that of the finite ones)
    heads = np.arange(q64.shape[1]) * k.shape[1] // q64.shape[1]
    size = scale * np.einsum("nhd,chd->hcn", np.abs(k)[:, heads], np.abs(q64))
    size = np.where(np.isfinite(size), size, 0.0).max(-1)
    want = R.weigh(w, old, m, keep_old, keep_new, gain, watch)
    first = max(0, m - watch) if watch else 0
    size = np.where(np.isfinite(lse), size, 0.0)                                    # (those count)
    eps = (d + 4) * 2.0 ** -24 * size + 2.0 ** -20                                  # [Hq][m]
    row = 2 * eps + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))
    tol = gain * (w * np.moveaxis(row, -1, 0)[..., None])[first:].sum((0, 1))
    terms = (m - first) * q64.shape[1] + 4
    return want, tol + terms * 2.0 ** -24 * np.abs(want) + 1e-37


def fill(c, rng, n, H, d, edit=None):
    held = []
    for b in range(len(n)):
        kv = [rng.standard_normal((n[b], H, d)) * np.exp(0.5 * rng.standard_normal((H, d))) for _ in range(2)]
        if edit:
            edit(b, *kv)
        got = []
        for i in range(2):
            raw, val = c.encode(kv[i])
            c.fill_rows(b, i, raw)
            got.append(val)
        held.append(got)
    return held


def same(a, b):
    """Bit for bit."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check(E, fmt, B, C, Hq, H, d, page, n, nn=None, seed=0, spread=1.0, scale=0.0, layers=1, edit=None, watch=0,
          keep_old=1.0, keep_new=0.0, gain=1.0, old="apart", slack=5, **cache):
    fmt = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(seed + 17 * C + d)
    room = max(max(n), 1)
    c = Cache(E, rng, fmt, B, H, d, page, room, layers=layers, layer=layers - 1, **cache)
    q, q64 = bf16(rng.standard_normal((B, C, Hq, d)) * spread)
    held = fill(c, rng, n, H, d, edit)
    before = torch.from_numpy(rng.exponential(2.0, (B, room + slack)).astype(np.float32)).to(DEV)
    kw = dict(nn=nn, scale=scale)
    acc = dict(watch=watch, keep_old=keep_old, keep_new=keep_new, gain=gain)
    got = []
    for noise in (0xA5, 0x5A):
        w = torch.full_like(before, 7.0) if old != "in place" else before.clone()
        src = {"apart": before, "in place": w, "none": None}[old]
        out, lse, status = run(E, c, C, n, q, weights=w, old=src, noise=noise, with_lse=noise == 0xA5, **kw, **acc)
        got.append((w, out, lse, status))
    assert same(got[0][0], got[1][0]) and same(got[0][1], got[1][1])
    out0, lse0, status0 = attend_only(E, c, C, n, q, **kw)
    assert same(out0, got[0][1]) and same(lse0, got[0][2])
    assert not got[0][3].any().item() and not status0.any().item()
    w = f64(got[0][0])
    b64 = f64(before)
    for b in range(B):
        m = C if nn is None else nn[b]
        live = n[b] if m > 0 else 0
        rest = b64[b, live:] if old == "in place" else 7.0
        assert np.all(w[b, live:] == rest), b
        if not live:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            want, tol = expected(q64[b, :m], *held[b], m, scale or d ** -0.5, None if old == "none" else b64[b, :live],
                                 keep_old, keep_new, gain, watch)
        assert np.isfinite(want).all() and np.isfinite(w[b, :live]).all(), b
        off = np.abs(w[b, :live] - want)
        assert np.all(off <= tol), (b, np.nanmax(off / tol), int(np.nanargmax(off / tol)))
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
    check(E, fmt, 3, 30, 8, 2, 128, page, [30, 131, 777], seed=page, gap=48, layers=2)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [2, 3, 5, 8])
@pytest.mark.parametrize("heads", [(32, 8, 128), (4, 4, 64), (24, 2, 128), (8, 2, 256)])
def test_short_chunks(E, fmt, C, heads):
    n = [C, C + 1, 33, 64, 200, 129]
    nn = [C, C, 1, C - 1, C, 0]
    for watch in (0, 1, 2):
        check(E, fmt, 6, C, *heads, 16, n, nn, watch=watch)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,n,nn", [
    (17, [17, 400, 100], [17, 17, 3]), (33, [33, 65], None), (64, [64, 1000], [64, 63]),
    (100, [100, 163], None), (129, [129, 500], [129, 1]), (300, [300], None), (300, [812], None),
    (257, [300, 257, 1], [257, 130, 0])])
@pytest.mark.parametrize("heads", [(8, 2, 128), (3, 1, 64), (2, 2, 256), (5, 1, 128)])
def test_chunks(E, fmt, C, n, nn, heads):
    check(E, fmt, len(n), C, *heads, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("watch", [1, 7, 32, 64, 65, 1000])
@pytest.mark.parametrize("heads", [(8, 2, 128), (7, 1, 64), (24, 2, 64)])
def test_windows(E, fmt, watch, heads):
    """The last tokens alone are counted, of each sequence its own last."""
    check(E, fmt, 4, 150, *heads, 16, [150, 700, 400, 130], [150, 150, 40, 0], watch=watch)


@pytest.mark.parametrize("old", ["apart", "in place", "none"])
@pytest.mark.parametrize("C", [1, 3, 40])
@pytest.mark.parametrize("keep", [(1.0, 1.0, 1.0), (0.75, 0.0, 0.03125), (0.0, 0.0, 1.0), (0.0, 1.0, 3.0)])
def test_what_is_kept(E, old, C, keep):
    check(E, "bf16", 3, C, 8, 2, 64, 16, [C + 300, C, 77 + C], old=old, keep_old=keep[0], keep_new=keep[1], gain=keep[2])


def test_sums_kept_by_zero_are_not_read(E):
    """A new token's slot, and with keep_old 0 every slot, may hold anything
    before: NaN does not come through."""
    rng = np.random.default_rng(2)
    for C in (1, 4, 30):
        n, H, d = [C + 90, C], 2, 64
        c = Cache(E, rng, E.KV_BF16, 2, H, d, 16, max(n))
        fill(c, rng, n, H, d)
        q = torch.randn(2, C, 8, d, device=DEV).bfloat16()
        w = torch.full((2, C + 90), float("nan"), device=DEV)
        run(E, c, C, n, q, weights=w, old=w, keep_old=0.0)
        assert torch.isfinite(w[0]).all() and torch.isfinite(w[1, :C]).all() and torch.isnan(w[1, C:]).all()
        before = torch.rand(2, C + 90, device=DEV)
        before[0, 90:] = float("nan")
        run(E, c, C, n, q, weights=w, old=before, keep_old=0.5)
        assert torch.isfinite(w[0]).all()


@pytest.mark.parametrize("fmt", FMTS)
def test_layers_add_up(E, fmt):
    """In place over three layers: every query's weights add up to 1, so the
    sums to layers x heads x tokens, and slots fade by the factor once."""
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(4)
    for C in (1, 5, 60):
        n, Hq, H, d = [C + 200, C + 3], 8, 2, 128
        w = torch.rand(2, C + 200, device=DEV)
        before = f64(w)
        for layer in range(3):
            c = Cache(E, rng, fm, 2, H, d, 16, max(n))
            fill(c, rng, n, H, d)
            q = torch.randn(2, C, Hq, d, device=DEV).bfloat16()
            run(E, c, C, n, q, weights=w, old=w, keep_old=0.5 if layer == 0 else 1.0, keep_new=float(layer > 0))
        for b in range(2):
            kept = 0.5 * before[b, :n[b] - C].sum()
            assert abs(f64(w)[b, :n[b]].sum() - kept - 3 * Hq * C) <= 1e-4 * (3 * Hq * C + kept)


@pytest.mark.parametrize("fmt", FMTS)
def test_long_sequence_alone(E, fmt):
    """One sequence over many workgroups, joined; and ragged neighbours."""
    check(E, fmt, 1, 1, 4, 1, 128, 16, [20011])
    check(E, fmt, 5, 1, 8, 2, 64, 16, [9001, 1, 0, 64, 12345], [1, 1, 0, 1, 1])
    check(E, fmt, 2, 20, 4, 2, 64, 16, [9001, 30])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,heads", [(1, (4, 2, 64)), (3, (8, 2, 128)), (1, (2, 1, 256)), (20, (2, 2, 64))])
def test_large_batches(E, fmt, C, heads):
    """Up to and past the number whose sequences are cut into shares."""
    rng = np.random.default_rng(11)
    for B in (300, 1100):
        n = rng.integers(0, 60, B).tolist()
        n[5], n[B - 1] = 0, 400
        check(E, fmt, B, C, *heads, 16, n, [min(x, C) for x in n])


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
    """With NaN in a later token's key the tokens that see it do not count; those
    before it do.  (Unused bytes of every page are NaN throughout these tests.)"""
    n = [C + 50, C + 3]

    def edit(b, k, v):
        at = n[b] - C + C // 2 + (1 if C > 1 else 0)
        if at < n[b]:
            k[at, 0, 3] = np.nan
            v[at, H - 1, 5], v[at, 0, 9] = np.nan, np.inf
    check(E, fmt, 2, C, Hq, H, d, 16, n, edit=edit, watch=0)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,watch", [(8, 2), (60, 16), (200, 64)])
def test_uncounted_tokens_hold_anything(E, fmt, C, watch):
    """NaN queries of padding and of tokens before the window do not reach the
    sums."""
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(C)
    n, nn, Hq, H, d = [C + 70, C + 5, 40], [C - 1, C, 3], 4, 2, 64
    c = Cache(E, rng, fm, 3, H, d, 16, max(n))
    held = fill(c, rng, n, H, d)
    q, q64 = bf16(rng.standard_normal((3, C, Hq, d)))
    q[0, C - 1:] = float("nan")
    q[1, :C - watch] = float("nan")
    q[2, 3:] = float("inf")
    w = torch.zeros(3, max(n), device=DEV)
    run(E, c, C, n, q, nn=nn, weights=w, watch=watch)
    for b in range(3):
        m = nn[b]
        first = max(0, m - watch)  # (those before it see less: the window's own rows are what counts)
        want, tol = expected(q64[b, :m], *held[b], m, d ** -0.5, None, 1.0, 0.0, 1.0, watch)
        assert first >= 0 and np.all(np.abs(f64(w)[b, :n[b]] - want) <= tol), b


@pytest.mark.parametrize("C,n", [(1, 40), (1, 5000), (4, 3000), (40, 3000), (200, 300)])
def test_nan_and_infinity_that_are_seen(E, C, n):
    """Queries that see a NaN key or an infinite score do not count, and leave no
    NaN in the sums; an infinite value changes no weight."""
    def edit(b, k, v):
        if b == 0:
            k[2 * n // 3, 0, 9] = np.inf
        if b == 1:
            k[n // 2, 0, 3] = np.nan
        if b == 2:
            v[n // 3, 1, 5] = np.inf
        if b == 3:
            k[n // 4, 1, 6] = -1e30
    check(E, "bf16", 4, C, 4, 2, 128, 16, [n] * 4, edit=edit)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads", [(3, 1, 64), (10, 2, 128), (7, 1, 256), (65, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("C,every", [(1, 1), (3, 2), (80, 9), (80, 21), (80, 79)])
def test_bad_queries_beside_good_ones(E, fmt, heads, C, every):
    """Groups that do not fill a tile's rows, and tokens whose first head holds a
    NaN or an infinity, a tile's first row among them: the others' weights are
    whole."""
    Hq, H, d = heads
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(C + every)
    n = [C + 700, C]
    c = Cache(E, rng, fm, 2, H, d, 16, max(n))
    held = fill(c, rng, n, H, d)
    q, q64 = bf16(rng.standard_normal((2, C, Hq, d)))
    for t in (q, q64):
        t[:, ::every, 0, 1] = float("nan")
        t[1, ::every, 0, 2:] = float("inf")
    w = torch.zeros(2, max(n), device=DEV)
    run(E, c, C, n, q, weights=w)
    for b in range(2):
        with np.errstate(invalid="ignore"):
            want, tol = expected(q64[b], *held[b], C, d ** -0.5, None, 1.0, 0.0, 1.0, 0)
        assert np.isfinite(want).all() and np.all(np.abs(f64(w)[b, :n[b]] - want) <= tol), b


@pytest.mark.parametrize("C", [1, 3, 40])
def test_rows_that_see_only_minus_infinity(E, C):
    """Every score -infinity: nothing is added, and no NaN."""
    rng = np.random.default_rng(5)
    n, Hq, H, d = [C + 30], 4, 2, 64
    c = Cache(E, rng, E.KV_BF16, 1, H, d, 16, n[0])

    def edit(b, k, v):
        k[:, 0] = 0.0
        k[:, 0, 5] = -np.inf
    held = fill(c, rng, n, H, d, edit)
    q, q64 = bf16(np.abs(rng.standard_normal((1, C, Hq, d))) + 0.1)
    w = torch.full((1, n[0]), 3.0, device=DEV)
    _, lse, _ = run(E, c, C, n, q, weights=w, old=w, keep_old=0.5, keep_new=0.25)
    assert torch.all(lse[0, :2] == -float("inf"))
    with np.errstate(invalid="ignore"):
        x = R.attend_weights(q64[0], held[0][0], C, d ** -0.5)
    assert not x[:, :2].any()
    want, tol = expected(q64[0][:, 2:], held[0][0][:, 1:], held[0][1][:, 1:], C, d ** -0.5, np.full(n[0], 3.0), 0.5, 0.25, 1.0, 0)
    assert np.all(np.abs(f64(w)[0] - want) <= tol)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 6, 90])
def test_pages_out_of_range_and_places_past_the_row(E, fmt, C):
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(C)
    B, Hq, H, d, page = 5, 8, 2, 128, 16
    n = [C + 170, C + 40, 5000, C - 1, C + 60]
    c = Cache(E, rng, fm, B, H, d, page, max(n[:2]))
    q, q64 = bf16(rng.standard_normal((B, C, Hq, d)))
    held = fill(c, rng, [n[0], n[1], 0, 0, n[4]], H, d)
    table = c.table.clone()
    table[0, 3], table[0, 7] = -1, 2 ** 30
    table[1, :] = 10 ** 9
    ld_s = C + 50
    w = torch.full((B, ld_s), 5.0, device=DEV)
    before = torch.rand(B, ld_s, device=DEV)
    out, lse, status = run(E, c, C, n, q, table=table, weights=w, old=before, keep_old=0.5)
    assert status.tolist() == [2, 2, 2, 2, 2]  # (0 and 4: slots past ld_s)
    out0, lse0, _ = attend_only(E, c, C, n, q, table=table)
    assert same(out, out0) and same(lse, lse0)
    ok = np.ones(n[0], bool)
    ok[48:64] = ok[112:128] = False
    b64 = f64(before)
    for b, mask in ((0, ok), (4, np.ones(n[4], bool))):
        old = np.zeros(n[b])
        m = min(n[b], ld_s)
        old[:m] = b64[b, :m]
        want, tol = expected(q64[b], *held[b], C, d ** -0.5, old, 0.5, 0.0, 1.0, 0, mask)
        assert np.all(np.abs(f64(w)[b, :m] - want[:m]) <= tol[:m]), b
    # nothing seen: the old sums stay in part; lengths out of range: nothing is written
    assert np.allclose(f64(w)[1, :40], 0.5 * b64[1, :40]) and torch.all(w[1, 40:C + 40] == 0)
    assert torch.all(w[2] == 5.0) and torch.all(w[3] == 5.0)


def test_strides(E):
    """Queries of a fused projection, outputs [B][heads][chunk][d], broadcast
    queries."""
    rng = np.random.default_rng(9)
    for C in (1, 3, 50):
        B, Hq, H, d = 2, 8, 2, 64
        n = [C + 20, C + 90]
        c = Cache(E, rng, E.KV_BF16, B, H, d, 16, max(n), fill=0)
        fill(c, rng, n, H, d)
        fused = torch.randn(B, C, Hq + 4, d, device=DEV).bfloat16()
        q = fused[:, :, 1:1 + Hq]
        wa, wb = torch.zeros(B, C + 90, device=DEV), torch.zeros(B, C + 90, device=DEV)
        a = run(E, c, C, n, q.contiguous(), weights=wa)[0]
        room = torch.full((B, Hq, C, d), 9.0, dtype=torch.bfloat16, device=DEV)
        o = run(E, c, C, n, q, out=room.transpose(1, 2), weights=wb)[0]
        assert same(a, o) and same(wa, wb)
        one = torch.randn(1, C, Hq, d, device=DEV).bfloat16()
        run(E, c, C, n, one.expand(B, C, Hq, d), weights=wa)
        run(E, c, C, n, one.expand(B, C, Hq, d).contiguous(), weights=wb)
        assert same(wa, wb)
        wide = torch.zeros(B, C + 200, device=DEV)  # part of a wider row
        run(E, c, C, n, q, weights=wide[:, :C + 90], ld_s=C + 200)
        run(E, c, C, n, q, weights=wa)
        assert same(wide[:, :C + 90], wa) and not wide[:, C + 90:].any()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 48])
def test_other_streams_and_graphs(E, fmt, C):
    """On a stream of its own, and captured: replays with eager work between
    them, and other lengths, give the eager call's bits; two graphs share a
    workspace."""
    fm = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    rng = np.random.default_rng(3)
    B, Hq, H, d = 3, 8, 2, 128
    n = [C + 500, C + 2, C + 3000]
    c = Cache(E, rng, fm, B, H, d, 16, max(n))
    fill(c, rng, n, H, d)
    q = torch.randn(B, C, Hq, d, device=DEV).bfloat16()
    before = torch.rand(B, max(n), device=DEV)

    def eager(n, **kw):
        w = torch.zeros_like(before)
        return (w,) + run(E, c, C, n, q, weights=w, old=before, keep_old=0.5, **kw)[:2]
    want = eager(n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = eager(n, stream=side)
    assert all(same(a, b) for a, b in zip(want, got))
    need = E.attend_weigh_workspace_bytes(c.cfg, C, Hq, c.ld_pt)
    ws = torch.zeros(need, dtype=torch.uint8, device=DEV)
    nd = ints(n)
    graphs, outs = [], []
    for _ in range(2):
        w, out, lse = (torch.zeros_like(x) for x in want)
        io = E.make_attend_io(C, c.pool, 0, c.table, c.ld_pt, nd, q, out, lse=lse, workspace=ws, workspace_bytes_=need)
        wio = E.make_weigh_io(w, w.shape[1], old=before, keep_old=0.5)
        E.epikv_attend_weigh(c.cfg, io, wio)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            E.epikv_attend_weigh(c.cfg, io, wio)
        graphs.append(g)
        outs.append((w, out, lse))
    for i in range(4):
        now = [x if i % 2 == 0 else max(C, x // 2) for x in n]
        fresh = eager(now)
        nd.copy_(ints(now))
        for t in outs[0] + outs[1]:
            t.zero_()
        ws.fill_(i * 37)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for got in outs:
            assert all(same(a, b) for a, b in zip(fresh, got))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 5, 48])
def test_two_calls_at_once(E, fmt, C):
    """On two streams, a workspace each, over the same pages: what each gives
    alone."""
    rng = np.random.default_rng(4)
    B, Hq, H, d = 2, 8, 2, 128
    n = [C + 4000, C + 900]
    c = Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, B, H, d, 16, max(n))
    fill(c, rng, n, H, d)
    need, nd = E.attend_weigh_workspace_bytes(c.cfg, C, Hq, c.ld_pt), ints(n)
    calls = []
    for _ in range(2):
        q = torch.randn(B, C, Hq, d, device=DEV).bfloat16()
        want = torch.zeros(B, max(n), device=DEV)
        run(E, c, C, n, q, weights=want)
        got, ws = torch.zeros_like(want), torch.empty(need, dtype=torch.uint8, device=DEV)
        io = E.make_attend_io(C, c.pool, 0, c.table, c.ld_pt, nd, q, torch.empty_like(q), workspace=ws, workspace_bytes_=need)
        calls.append((want, got, io, E.make_weigh_io(got, max(n)), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(8):
        for _, _, io, wio, s in calls:
            E.epikv_attend_weigh(c.cfg, io, wio, stream=s)
    torch.cuda.synchronize()
    for want, got, *_ in calls:
        assert same(want, got)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 48])
def test_shared_pages(E, fmt, C):
    """Sequences with the same pages, and one page twice in a table: every slot
    has its own sum."""
    rng = np.random.default_rng(14)
    Hq, H, d, page = 8, 2, 64, 16
    n = C + 77
    c = Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, 2, H, d, page, n)
    fill(c, rng, [n, n], H, d)
    q = torch.randn(1, C, Hq, d, device=DEV).bfloat16().expand(2, C, Hq, d)
    both = c.table[:1].expand(2, -1).contiguous()
    w = torch.zeros(2, n, device=DEV)
    run(E, c, C, [n, n], q, table=both, weights=w)
    assert same(w[0], w[1])
    twice = both.clone()
    twice[:, 1] = twice[:, 0]
    run(E, c, C, [n, n], q, table=twice, weights=w)
    assert same(w[:, :page], w[:, page:2 * page]) and same(w[0], w[1])


def test_wide_tables(E):
    """A page table that covers far more than the sequences hold; what the
    scratch is indexed by passes 32 bits."""
    rng = np.random.default_rng(6)
    B, Hq, H, d, page = 40, 32, 8, 128, 1024
    n = [0] * B
    n[0], n[B - 1] = 130, 1500
    width = 1024  # a million slots
    for C in (1, 24):
        c = Cache(E, rng, E.KV_BF16, B, H, d, page, max(n))
        held = fill(c, rng, n, H, d)
        q, q64 = bf16(rng.standard_normal((B, C, Hq, d)))
        table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
        table[:, :c.ld_pt] = c.table
        c.ld_pt = width
        w = torch.zeros(B, 1600, device=DEV)
        run(E, c, C, n, q, nn=[min(C, x) for x in n], table=table, weights=w)
        for b in (0, B - 1):
            want, tol = expected(q64[b], *held[b], C, d ** -0.5, None, 1.0, 0.0, 1.0, 0)
            assert np.all(np.abs(f64(w)[b, :n[b]] - want) <= tol), b
        assert not w[1:B - 1].any()


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
        fill(c, rng, [n], H, d)
        for C in (1, 40):
            q = torch.randn(1, C, Hq, d, device=DEV).bfloat16()
            a, b = torch.zeros(1, n, device=DEV), torch.zeros(1, n, device=DEV)
            run(E, c, C, [n], q, weights=a)
            view = big.view(2, n_pages, stride)
            pages = ints([[39999, 35000]])
            for m in range(2):
                view[:, int(pages[0, m])] = c.bytes[0, :, int(c.table_host[0, m])]
            c2 = type("C2", (), dict(cfg=cfg, pool=E.Pool(big.data_ptr(), 0, n_pages * stride, stride, n_pages),
                                     layer=0, table=pages, ld_pt=2))
            run(E, c2, C, [n], q, weights=b)
            assert same(a, b)
        del big


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("heads", [(65, 1, 64), (130, 1, 64), (128, 2, 128), (71, 1, 256)])
@pytest.mark.parametrize("C", [1, 3, 9])
def test_groups_past_a_tile(E, fmt, heads, C):
    """More query heads to a KV head than a tile has rows."""
    check(E, fmt, 3, C, *heads, 16, [C + 300, C, 40], [C, C, min(C, 2)])
    check(E, fmt, 2, C, *heads, 16, [C + 300, C], watch=1)


def test_queries_far_apart(E):
    """Rows of one tile that span more than 2^31 bytes, by tokens and by heads."""
    rng = np.random.default_rng(12)
    Hq, H, d, C = 8, 1, 64, 20
    n = [C + 100]
    c = Cache(E, rng, E.KV_BF16, 1, H, d, 16, n[0])
    fill(c, rng, n, H, d)
    q = torch.randn(1, C, Hq, d, device=DEV).bfloat16()
    want = torch.zeros(1, n[0], device=DEV)
    out = run(E, c, C, n, q, weights=want)[0]
    for strides in ((0, 170 << 20, d, 1), (0, d, 160 << 20, 1)):
        size = (C - 1) * strides[1] + (Hq - 1) * strides[2] + d
        far = torch.empty(size, dtype=torch.bfloat16, device=DEV).as_strided((1, C, Hq, d), strides)
        far.copy_(q)
        got = torch.zeros(1, n[0], device=DEV)
        o = run(E, c, C, n, far, weights=got)[0]
        assert same(got, want) and same(o, out)
        del far


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 4, 60])
@pytest.mark.parametrize("scale", [1e4, 1e6, 1e8, 1e12])
def test_scores_too_large_to_tell_apart(E, fmt, C, scale):
    """What float32 leaves of such weights is still between 0 and 1 a row."""
    rng = np.random.default_rng(C)
    Hq, H, d, n = 8, 2, 64, [C + 200, C]
    c = Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, 2, H, d, 16, max(n))
    fill(c, rng, n, H, d)
    q = torch.randn(2, C, Hq, d, device=DEV).bfloat16()
    w = torch.zeros(2, max(n), device=DEV)
    run(E, c, C, n, q, weights=w, scale=scale)
    assert torch.isfinite(w).all() and (w >= 0).all() and (w <= C * Hq).all()


@pytest.mark.parametrize("seed", range(24))
def test_random_mixes(E, seed):
    rng = np.random.default_rng(2000 + seed)
    d = int(rng.choice([64, 128, 256]))
    H = int(rng.choice([1, 2, 3, 4]))
    G = int(rng.choice([1, 2, 3, 4, 6, 8, 11]))
    C = int(rng.choice([1, 1, 2, 3, 7, 16, 31, 64, 130]))
    B = int(rng.integers(1, 6))
    nn = [int(rng.integers(0, C + 1)) for _ in range(B)]
    n = [x + int(rng.integers(0, 700)) for x in nn]
    check(E, FMTS[seed % 2], B, C, G * H, H, d, int(rng.choice([1, 7, 16, 32, 100])), n, nn, seed=seed,
          watch=int(rng.choice([0, 0, 1, 5, 40])), keep_old=float(rng.choice([0.0, 0.5, 1.0])),
          keep_new=float(rng.choice([0.0, 1.0])), gain=float(rng.choice([1.0, 0.25])),
          old=str(rng.choice(["apart", "in place", "none"])))

"""Appending to the paged cache and reading it back, against the oracle: bytes
of bf16 and of 4-bit rows, positions, padding, flags, and every byte that must
stay."""
import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import DEV, Cache, f64, quick_encode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def rotated32(x, table, pos, il, r):
    """The float32 steps of the rotation (x bf16 on the CPU)."""
    cs = table.cpu()[torch.from_numpy(pos).long()]
    c, s = cs[..., 0].unsqueeze(2), cs[..., 1].unsqueeze(2)
    x = x.float()
    y = x.clone()
    lo, hi = (slice(0, r, 2), slice(1, r, 2)) if il else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    return y


def rows_of_values(E, c, x):
    """Raw rows of float32 values [..., H, d]."""
    flat = x.reshape(x.shape[0], c.H * c.d)
    if c.fmt == E.KV_BF16:
        return flat.bfloat16().view(torch.uint8).numpy()
    codes, byte = quick_encode(flat.double().numpy())
    return R.mxfp4_pack(codes, byte, c.row)


SHAPES = [  # B, C, Hq, H, d, r, page, cached before, n_new
    (1, 1, 4, 1, 64, 64, 16, [0], None),
    (3, 1, 32, 8, 128, 128, 16, [15, 16, 4000], None),
    (2, 33, 8, 8, 64, 32, 5, [3, 0], None),
    (4, 7, 6, 3, 128, 64, 1, [0, 1, 2, 9], [7, 0, 1, 6]),
    (2, 70, 16, 8, 256, 256, 1024, [1000, 30], [70, 69]),
    (2, 20, 5, 5, 256, 16, 12, [11, 40], [3, 20]),
    (1, 300, 24, 8, 128, 112, 48, [100], None),
]


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_append(E, shape, il, fmt):
    B, C, Hq, H, d, r, page, before, n_new = shape
    rng = np.random.default_rng(B * 1000 + C)
    g = torch.Generator().manual_seed(C * 7 + d)
    fmt = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    nn = n_new or [C] * B
    n = [p + m for p, m in zip(before, nn)]
    c = Cache(E, rng, fmt, B, H, d, page, max(n) + 5, layers=3, layer=1, gap=32)
    start = c.bytes.clone()
    k = (torch.randn(B, C, H, d, generator=g) * torch.exp(torch.randn(H, d, generator=g))).bfloat16()
    v = torch.randn(B, C, H, d, generator=g).bfloat16()
    q = torch.randn(B, C, Hq, d, generator=g).bfloat16()
    first = np.array([m - p + 37 * b for b, (m, p) in enumerate(zip(n, nn))], dtype=np.int32)
    rope = E.default_rope(rotary_dim=r, n_pos=int(first.max()) + C, theta=500000.0, layout=int(il))
    table = torch.empty(rope.n_pos, r // 2, 2, device=DEV)
    E.epikv_rope_table(rope, table)
    q_out = torch.full((B, C, Hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    ids = torch.full((B, max(n) + 2), -5, dtype=torch.int32, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    kd, vd, qd = k.to(DEV), v.to(DEV), q.to(DEV)
    io = E.make_append_io(C, c.pool, 1, c.table, c.ld_pt, ints(*n), kd, vd,
                          n_new=ints(*nn) if n_new else None, rope=rope, table=table,
                          positions=torch.from_numpy(first).to(DEV), q=qd, q_out=q_out, pos=ids,
                          ld_s=ids.shape[1], seq_status=status)
    E.epikv_append(c.cfg, io)
    pos = first[:, None] + np.arange(C)
    want_k = rotated32(k, table, pos, il, r)
    want_q = rotated32(q, table, pos, il, r).bfloat16()
    got_q, got_ids = q_out.cpu(), ids.cpu()
    expect = start.cpu().numpy().copy()
    used = c.row if fmt == E.KV_BF16 else H * d // 2 + H * d // 32  # (the padding is never written)
    for b in range(B):
        m = nn[b]
        rk, rv = rows_of_values(E, c, want_k[b, :m]), rows_of_values(E, c, v[b, :m].float())
        for i in range(m):
            slot = n[b] - m + i
            pg, at = c.table_host[b, slot // page], slot % page * c.row
            expect[1, 0, pg, at:at + used] = rk[i, :used]
            expect[1, 1, pg, at:at + used] = rv[i, :used]
        assert torch.equal(got_q[b, :m], want_q[b, :m])
        assert torch.all(got_q[b, m:] == 9.0)
        assert got_ids[b, n[b] - m:n[b]].tolist() == pos[b, :m].tolist()
        assert torch.all(got_ids[b, :n[b] - m] == -5) and torch.all(got_ids[b, n[b]:] == -5)
    assert np.array_equal(c.bytes.cpu().numpy(), expect)
    assert not status.any().item()
    # queries in place
    io = E.make_append_io(C, c.pool, 1, c.table, c.ld_pt, ints(*n), kd, vd,
                          n_new=ints(*nn) if n_new else None, rope=rope, table=table,
                          positions=torch.from_numpy(first).to(DEV), q=qd, q_out=qd)
    E.epikv_append(c.cfg, io)
    for b in range(B):
        assert torch.equal(qd.cpu()[b, :nn[b]], want_q[b, :nn[b]])
        assert torch.equal(qd.cpu()[b, nn[b]:], q[b, nn[b]:])
    assert np.array_equal(c.bytes.cpu().numpy(), expect)
    # read back: the values of the rows
    for b in range(B):
        if not nn[b]:
            continue
        back = [torch.full((B, C, H, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        rd = E.make_read_io(C, c.pool, 1, c.table, c.ld_pt,
                            ints(*[x - C if x >= C else 0 for x in n]), back[0], back[1])
        E.epikv_read(c.cfg, rd)
        lo = n[b] - C if n[b] >= C else 0
        for kv in range(2):
            raw = c.rows(b, kv, lo + C)[lo:] if lo + C <= c.ld_pt * page else None
            if raw is None:
                continue
            if fmt == E.KV_BF16:
                assert np.array_equal(back[kv][b].cpu().reshape(C, -1).view(torch.uint8).numpy(), raw)
            else:
                held = R.mxfp4_decode(raw, H * d).reshape(C, H, d)
                assert np.array_equal(f64(back[kv][b]), held, equal_nan=True)


@pytest.mark.parametrize("scale", [2.0 ** -127, 2.0 ** -100, 1e-30, 1e-3, 1.0, 1e4, 1e30, 3e38])
def test_quantising_every_magnitude(E, scale):
    """Values, not rotated, over the whole range of bf16, with ties and zeros."""
    g = torch.Generator().manual_seed(11)
    C, H, d = 64, 2, 64
    x = torch.randn(1, C, H, d, generator=g)
    x[0, 0, 0, :8] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5])
    x[0, 1, 0, :32] = 0
    x[0, 2, 0, 8:40] = -x[0, 2, 0, 8:40].abs()
    x[0, 3, 0, :8] = torch.tensor([7.0, -7.0, 7.03125, 0, 0.5, -0.25, -0.75, 3.5])
    x = (x.clamp(-1, 1) if scale > 1e38 else x).bfloat16().float() * scale
    x = x.bfloat16()
    assert torch.isfinite(x).all()
    c = Cache(E, np.random.default_rng(1), E.KV_MXFP4, 1, H, d, 16, C)
    xd = x.to(DEV)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(C), xd, xd))
    want = rows_of_values(E, c, x[0].float())
    used = H * d // 2 + H * d // 32
    for kv in range(2):
        assert np.array_equal(c.rows(0, kv, C)[:, :used], want[:, :used])


def test_nan_and_infinity_make_their_block_nan(E):
    C, H, d = 4, 1, 128
    x = torch.ones(1, C, H, d)
    x[0, 0, 0, 3], x[0, 1, 0, 40], x[0, 2, 0, 127] = float("nan"), float("inf"), float("-inf")
    xd = x.bfloat16().to(DEV)
    c = Cache(E, np.random.default_rng(1), E.KV_MXFP4, 1, H, d, 16, C, fill=0)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(C), xd, xd))
    k = torch.zeros(1, C, H, d, dtype=torch.bfloat16, device=DEV)
    E.epikv_read(c.cfg, E.make_read_io(C, c.pool, 0, c.table, c.ld_pt, ints(0), k))
    bad = torch.isnan(k[0, :, 0].view(C, 4, 32))
    for i, blocks in enumerate([[0], [1], [3], []]):
        for j in range(4):
            assert bool(bad[i, j].all()) == (j in blocks) and bool(bad[i, j].any()) == (j in blocks)
    assert torch.all(k[0, 3] == 1)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
def test_out_of_range_is_flagged_and_left(E, fmt):
    """Counts, pages and positions out of range: the sequence (or the token)
    is left, its neighbours are written."""
    fmt = E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4
    B, C, H, d, page = 8, 2, 2, 64, 4
    c = Cache(E, np.random.default_rng(2), fmt, B, H, d, page, 16)
    table = c.table.clone()
    table[5, 2] = 10 ** 6           # slots 8..11 of sequence 5
    table[6, 2] = -1
    n = ints(10, 17, 1, -1, 10, 10, 10, 12)
    nn = ints(2, 2, 2, 0, 3, 2, 2, 2)
    first = ints(0, 0, 0, 0, 0, 0, 0, 7)
    x = torch.ones(B, C, H, d, dtype=torch.bfloat16, device=DEV)
    rope = E.default_rope(rotary_dim=64, n_pos=8)
    tab = torch.empty(8, 32, 2, device=DEV)
    E.epikv_rope_table(rope, tab)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    ids = torch.full((B, 16), -5, dtype=torch.int32, device=DEV)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, table, c.ld_pt, n, x, x, n_new=nn, rope=rope,
                                           table=tab, positions=first, q=x, q_out=x.clone(), pos=ids,
                                           ld_s=16, seq_status=status))
    assert status.tolist() == [0, 2, 2, 2, 2, 2, 2, 2]
    wrote = [[s for s in range(16) if not np.all(c.rows(b, 0, 16)[s, :32] == 255)] for b in range(B)]
    assert wrote == [[8, 9], [], [], [], [], [], [], [10]]
    assert (ids != -5).sum().item() == 3
    # read: slots outside and bad pages are zeros
    k = torch.full((B, C, H, d), 3.0, dtype=torch.bfloat16, device=DEV)
    status.zero_()
    E.epikv_read(c.cfg, E.make_read_io(C, c.pool, 0, table, c.ld_pt, ints(8, 15, -1, 0, 8, 8, 11, 8), k,
                                       seq_status=status))
    assert status.tolist() == [0, 2, 2, 0, 0, 2, 2, 0]
    assert torch.all(k[1, 1] == 0) and torch.all(k[2, 0] == 0) and torch.all(k[5] == 0)
    assert torch.all(k[6, 0] == 0) and torch.all(k[0].abs().sum(-1) > 0)


def test_views_and_broadcast_inputs(E):
    """Rows of a fused projection; one value broadcast over heads and batch."""
    B, C, H, d = 2, 5, 2, 64
    fused = torch.randn(B, C, 3 * H, d, device=DEV).bfloat16()
    v1 = torch.randn(1, C, 1, d, device=DEV).bfloat16()
    c = Cache(E, np.random.default_rng(2), E.KV_BF16, B, H, d, 4, C)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(C, C),
                                           fused[:, :, H:2 * H], v1.expand(B, C, H, d)))
    for b in range(B):
        assert np.array_equal(c.rows(b, 0, C), fused[b, :, H:2 * H].reshape(C, -1).contiguous().cpu()
                              .view(torch.uint8).numpy())
        assert np.array_equal(c.rows(b, 1, C), v1[0].expand(C, H, d).reshape(C, -1).contiguous().cpu()
                              .view(torch.uint8).numpy())


def test_rows_past_four_gigabytes(E):
    """Offsets past 32 bits inside a plane."""
    H, d, page, n_pages = 1, 64, 1024, 40000
    stride = page * 128
    pool = torch.zeros(2 * n_pages * stride, dtype=torch.uint8, device=DEV)  # 10.5 GB
    cfg = E.default_cfg(batch=2, n_layers=1, n_kv_heads=H, head_dim=d, page_size=page)
    P = E.Pool(pool.data_ptr(), 0, n_pages * stride, stride, n_pages)
    table = ints(39999, 17, 33000, 2).view(2, 2)
    x = torch.randn(2, 3, H, d, device=DEV).bfloat16()
    n = ints(1024, 1025)
    E.epikv_append(cfg, E.make_append_io(3, P, 0, table, 2, n, x, x))
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    E.epikv_read(cfg, E.make_read_io(3, P, 0, table, 2, n - 3, k, v))
    assert torch.equal(k, x) and torch.equal(v, x)
    view = pool.view(2, n_pages, page, 128)
    assert torch.equal(view[1, 39999, 1021:].reshape(-1), x[0].reshape(-1).view(torch.uint8))
    assert torch.equal(view[0, 2, 0].reshape(-1), x[1, 2].reshape(-1).view(torch.uint8))

"""The cache calls on rows that lie between each other's in one buffer: slices
of a fused projection as input, as output, and as both."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache

pytestmark = pytest.mark.gpu
LAYOUTS = [(1, 1, False), (3, 1, False), (2, 9, False), (2, 9, True)]


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def fused(B, C, heads, d, heads_first):
    """Random [B][C][heads][d], as a view of [B][heads][C][d] or of itself."""
    g = torch.Generator(device=DEV).manual_seed(B * 100 + C)
    shape = (B, heads, C, d) if heads_first else (B, C, heads, d)
    x = torch.randn(shape, generator=g, device=DEV).bfloat16()
    return x.transpose(1, 2) if heads_first else x


def table_of(E, d, n_pos=64):
    rope = E.default_rope(rotary_dim=d, n_pos=n_pos)
    t = torch.empty(n_pos, d // 2, 2, device=DEV)
    E.epikv_rope_table(rope, t)
    return rope, t


@pytest.mark.parametrize("B,C,heads_first", LAYOUTS)
def test_rope_into_another_slice(E, B, C, heads_first):
    H, d = 4, 64
    x = fused(B, C, 2 * H, d, heads_first)
    start = x.clone()
    rope, t = table_of(E, d)
    want = torch.empty(B, C, H, d, dtype=torch.bfloat16, device=DEV)
    first = ints(list(range(B)))
    E.epikv_rope(rope, t, E.DTYPE_BF16, B, C, H, d, start[:, :, :H].contiguous(), want, first)
    E.epikv_rope(rope, t, E.DTYPE_BF16, B, C, H, d, x[:, :, :H], x[:, :, H:], first)
    assert torch.equal(x[:, :, H:], want) and torch.equal(x[:, :, :H], start[:, :, :H])


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("B,C,heads_first", LAYOUTS)
def test_append_attend_and_read_in_one_buffer(E, B, C, heads_first, fmt):
    Hq, H, d = 8, 2, 64
    n = [C + 5 * b for b in range(B)]
    rng = np.random.default_rng(3)
    c = Cache(E, rng, fmt, B, H, d, 4, max(n), fill=0)
    start = c.bytes.clone()
    x = fused(B, C, 2 * Hq + 2 * H, d, heads_first)
    was = x.clone()
    rope, t = table_of(E, d)
    kw = dict(rope=rope, table=t, positions=ints(list(range(B))))

    def split(a):
        return a[:, :, :Hq], a[:, :, Hq:2 * Hq], a[:, :, 2 * Hq:2 * Hq + H], a[:, :, 2 * Hq + H:]
    q, o, k, v = split(x)
    wq, _, wk, wv = (a.contiguous() for a in split(was))
    want_q = torch.empty_like(wq)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), wk, wv, q=wq, q_out=want_q, **kw))
    held = c.bytes.clone()
    need = E.attend_workspace_bytes(c.cfg, C, Hq)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    want_o = torch.empty_like(wq)
    E.epikv_attend(c.cfg, E.make_attend_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), want_q, want_o, workspace=ws,
                                           workspace_bytes_=need))
    c.bytes.copy_(start)
    # in place, then attention and the rows read back, all in the one buffer
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), k, v, q=q, q_out=q, **kw))
    assert torch.equal(c.bytes, held) and torch.equal(q, want_q)
    E.epikv_attend(c.cfg, E.make_attend_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), q, o, workspace=ws,
                                           workspace_bytes_=need))
    assert torch.equal(o, want_o) and torch.equal(q, want_q)
    back = [torch.empty_like(wk) for _ in range(2)]
    first = ints([m - C for m in n])
    E.epikv_read(c.cfg, E.make_read_io(C, c.pool, 0, c.table, c.ld_pt, first, *back))
    E.epikv_read(c.cfg, E.make_read_io(C, c.pool, 0, c.table, c.ld_pt, first, k, v))
    assert torch.equal(k, back[0]) and torch.equal(v, back[1])
    assert torch.equal(q, want_q) and torch.equal(o, want_o)
    # the rotated queries into another slice
    x.copy_(was)
    c.bytes.copy_(start)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), k, v, q=q, q_out=o, **kw))
    assert torch.equal(c.bytes, held) and torch.equal(o, want_q) and torch.equal(q, wq)

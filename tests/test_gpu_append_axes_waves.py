"""Appending by positions on several axes where a wavefront has one token and
gathers its turns in LDS: shapes whose queries and keys both fill two thirds of
their wavefronts' lanes, with wavefronts full and in part, and, beside them, one
that does not."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache
from test_gpu_rope_axes import Appended, ints, same, table_of

pytestmark = pytest.mark.gpu

# (items of a token, of queries and of keys and values, of 64 lanes each:
# 128 and 128; 48 and 96; 128 and 256; 120 and 96, one head at a time; 64 and 64;
# 32 and 128, which is left to threads)
SHAPES = [((32, 8, 128), (16, 24, 24)), ((12, 6, 128), (5, 9, 10)), ((16, 8, 256), (60, 30, 20, 18)),
          ((15, 3, 128), (1, 62, 1)), ((16, 4, 128), (20, 12)), ((16, 16, 64), (5, 5, 6))]


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("heads,pairs", SHAPES)
@pytest.mark.parametrize("turns", [False, True])
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("per_token", [False, True])
@pytest.mark.parametrize("queries", [True, False])
def test_append(E, fmt, heads, pairs, turns, il, per_token, queries):
    """Byte for byte the append of one axis by a table of each token's own
    turns, padded tokens among them; and the ids."""
    args = (E, fmt, heads, pairs, turns, il, per_token)
    a, b = (Appended(*args, plain, queries=queries) for plain in (False, True))
    assert same(a.c.bytes, b.c.bytes) and same(a.q_out, b.q_out)
    assert not a.status.any().item()
    ids = a.pos.cpu().numpy()
    for s in range(3):
        first = a.n[s] - a.nn[s]
        assert np.array_equal(ids[s, first:a.n[s]], a.ids[s, :a.nn[s]])
        assert np.all(ids[s, :first] == -1) and np.all(ids[s, a.n[s]:] == -1)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("heads,pairs", SHAPES)
def test_positions_out_of_range(E, fmt, heads, pairs):
    """On one axis: the token's row, queries and id stay as they were and its
    sequence is flagged; the others are what they are without it."""
    Hq, H, d = heads
    B, C, A, n_pos = 3, 6, len(pairs), 90
    rope, axes = E.default_rope(rotary_dim=2 * sum(pairs), n_pos=n_pos), E.axes_of(pairs, order=E.AXES_TURNS)
    table = table_of(E, rope, axes)
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(B, C, h, d, generator=g).bfloat16().to(DEV) for h in (Hq, H, H))
    good = torch.randint(0, n_pos, (B, A, C), generator=g, dtype=torch.int32).to(DEV)
    bad = good.clone()
    bad[0, 0, 2], bad[0, A - 1, 4], bad[2, A - 1, 0] = n_pos, -1, 2 ** 31 - 1
    left = {(0, 2), (0, 4), (2, 0)}
    n = [C, C + 9, C + 3]

    def append(positions):
        c = Cache(E, np.random.default_rng(2), fmt, B, H, d, 4, 20)
        q_out, pos, status = torch.full_like(q, 5.0), torch.full((B, 20), -1, dtype=torch.int32, device=DEV), ints([0] * B)
        io = E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), k, v, rope=rope, table=table, positions=positions,
                              ld_pos=C, axes=axes, ids=ints([100, 200, 300]), q=q, q_out=q_out, pos=pos, ld_s=20,
                              seq_status=status)
        E.epikv_append_axes(c.cfg, io)
        return [[c.rows(b, kv, n[b]) for kv in range(2)] for b in range(B)], q_out, pos.cpu().numpy(), status.tolist()
    rows, q_all, ids, status = append(good)
    assert status == [0, 0, 0]
    rows_bad, q_bad, ids_bad, status = append(bad)
    assert status == [2, 0, 2]
    for b in range(B):
        for t in range(C):
            at = n[b] - C + t
            if (b, t) in left:
                assert all((rows_bad[b][kv][at] == 255).all() for kv in range(2)), (b, t)
                assert torch.all(q_bad[b, t] == 5.0) and ids_bad[b, at] == -1, (b, t)
            else:
                assert all(np.array_equal(rows_bad[b][kv][at], rows[b][kv][at]) for kv in range(2)), (b, t)
                assert same(q_bad[b, t], q_all[b, t]) and ids_bad[b, at] == ids[b, at] == 100 * (b + 1) + t, (b, t)

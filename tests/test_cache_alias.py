"""Which tensors of the cache calls may share a buffer (CPU: a call that is
not refused ends at its launch, which fails without a GPU)."""
import ctypes
import random

import pytest

A = 1 << 20  # fake, aligned addresses, never dereferenced


def _no_gpu():
    try:
        import torch
        return not torch.cuda.is_available()
    except Exception:
        return True


pytestmark = pytest.mark.skipif(not _no_gpu(), reason="fake-pointer validation runs only without a GPU")


@pytest.fixture(scope="module")
def E():
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def pool(E):
    return E.Pool(A, 1 << 30, 1 << 29, 32768, 100)


def append(E, B, C, Hq, H, d, q, q_out, k, v):
    cfg = E.default_cfg(batch=B, n_layers=1, n_kv_heads=H, head_dim=d)
    io = E.AppendIO()
    io.chunk, io.pool, io.page_table, io.ld_pt, io.n_cached = C, pool(E), 2 * A, 8, 3 * A
    io.k, io.v, io.n_heads, io.q, io.q_out = k, v, Hq, q, q_out
    return E.lib().epikv_append(ctypes.byref(cfg), ctypes.byref(io), None)


def read(E, B, C, H, d, k, v):
    cfg = E.default_cfg(batch=B, n_layers=1, n_kv_heads=H, head_dim=d)
    io = E.ReadIO()
    io.chunk, io.pool, io.page_table, io.ld_pt, io.first, io.k, io.v = C, pool(E), 2 * A, 8, 3 * A, k, v
    return E.lib().epikv_read(ctypes.byref(cfg), ctypes.byref(io), None)


def attend(E, B, C, Hq, d, q, out):
    cfg = E.default_cfg(batch=B, n_layers=1, n_kv_heads=1, head_dim=d)
    io = E.AttendIO()
    io.chunk, io.pool, io.page_table, io.ld_pt, io.n_cached = C, pool(E), 2 * A, 8, 3 * A
    io.n_heads, io.q, io.out = Hq, q, out
    return E.lib().epikv_attend(ctypes.byref(cfg), ctypes.byref(io), None)


def rope(E, B, C, heads, d, x, y, dtype=0):
    r = E.default_rope(rotary_dim=d)
    return E.lib().epikv_rope(ctypes.byref(r), A, dtype, B, C, heads, d, ctypes.byref(x), ctypes.byref(y), 2 * A, 0, 0,
                              None, None)


class Fused:
    """Slices of one [B][C][heads][d] or [B][heads][C][d] projection."""

    def __init__(self, E, B, C, heads, d, heads_first=False):
        self.E, self.d = E, d
        self.ld = (C * heads * d, d, C * d) if heads_first else (C * heads * d, heads * d, d)

    def slice(self, head, more=0):
        return self.E.Rows(64 * A + 2 * (head * self.ld[2] + more), *self.ld)


@pytest.mark.parametrize("B,C,heads_first", [(1, 1, False), (4, 1, False), (1, 7, False), (3, 7, False), (3, 7, True)])
def test_queries_and_keys_of_one_projection(E, B, C, heads_first):
    """Queries rotated in place beside their keys and values pass; queries that
    are the keys or the values, or share some of their heads, do not: the
    launch would rotate what it is still reading."""
    Hq, H, d = 8, 2, 64
    f = Fused(E, B, C, Hq + 2 * H, d, heads_first)
    q, k, v = f.slice(0), f.slice(Hq), f.slice(Hq + H)
    far = E.Rows(512 * A, *f.ld)
    for q_out in (q, far):
        assert append(E, B, C, Hq, H, d, q, q_out, k, v) != E.EPIKV_EALIAS
    for kk, vv in ((f.slice(Hq - 1), v), (k, f.slice(Hq - 1)), (q, v), (k, q), (f.slice(Hq, -32), v)):
        assert append(E, B, C, Hq, H, d, q, q, kk, vv) == E.EPIKV_EALIAS
        assert append(E, B, C, Hq, H, d, far, q, kk, vv) == E.EPIKV_EALIAS
    # all heads alike, the same tensor three times
    assert append(E, B, C, H, H, d, q, q, q, q) == E.EPIKV_EALIAS
    # the rotated queries into another slice of the same buffer
    assert append(E, B, C, H, H, d, q, f.slice(H), k, v) != E.EPIKV_EALIAS
    assert append(E, B, C, H, H, d, q, f.slice(1), k, v) == E.EPIKV_EALIAS
    # the other calls' pairs
    assert rope(E, B, C, H, d, q, k) != E.EPIKV_EALIAS
    assert rope(E, B, C, H, d, q, f.slice(H - 1)) == E.EPIKV_EALIAS
    assert read(E, B, C, H, d, k, v) != E.EPIKV_EALIAS
    assert read(E, B, C, H, d, k, f.slice(Hq + 1)) == E.EPIKV_EALIAS
    assert attend(E, B, C, 4, d, q, f.slice(4)) != E.EPIKV_EALIAS
    assert attend(E, B, C, 4, d, q, f.slice(3)) == E.EPIKV_EALIAS


def elements(r, B, C, heads, d, es):
    at = r.base // es
    return {at + b * r.ld_seq + c * r.ld_tok + h * r.ld_head + i
            for b in range(B) for c in range(C) for h in range(heads) for i in range(d)}


@pytest.mark.parametrize("seed", range(4))
def test_shared_elements_are_always_refused(E, seed):
    """Random strides, nested, interleaved and broadcast, against the sets of
    elements themselves."""
    rng = random.Random(seed)
    met = 0
    for _ in range(400):
        B, C, heads, d = rng.choice([1, 2, 3]), rng.choice([1, 2, 4]), rng.choice([1, 2, 3]), 16
        strides = [8 * rng.choice([0, 2, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96]) for _ in range(3)]
        x = E.Rows(A, *strides)
        if rng.random() < 0.5:
            rng.shuffle(strides)
        y = E.Rows(A + 16 * rng.randrange(0, 160), *strides)
        es = rng.choice([2, 4])
        ex, ey = elements(x, B, C, heads, d, es), elements(y, B, C, heads, d, es)
        st = rope(E, B, C, heads, d, x, y, dtype=0 if es == 2 else 1)
        if st == E.EPIKV_EINVAL_SHAPE:
            continue  # (y's rows overlap each other)
        same = (x.base, x.ld_seq, x.ld_tok, x.ld_head) == (y.base, y.ld_seq, y.ld_tok, y.ld_head)
        if ex & ey and not same:
            met += 1
            assert st == E.EPIKV_EALIAS, (B, C, heads, x.base, y.base, strides, es)
        if max(ex) < min(ey) or max(ey) < min(ex):
            assert st != E.EPIKV_EALIAS
    assert met > 20

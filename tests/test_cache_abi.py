"""Refusals of the calls that fill and read the cache (CPU: every call here
fails on the host, before a launch)."""
import ctypes

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


def test_defaults_and_sizes(E):
    c = E.default_cfg()
    assert c.kv_format == E.KV_BF16 and E.kv_row_bytes(c) == 2048
    for H, d, row in ((8, 128, 544), (1, 64, 128), (3, 64, 128), (4, 64, 144), (8, 256, 1088), (5, 64, 176)):
        c = E.default_cfg(n_kv_heads=H, head_dim=d, kv_format=E.KV_MXFP4)
        assert E.check_cfg(c) == 0 and E.kv_row_bytes(c) == row and row % 16 == 0
    r = E.default_rope()
    assert E.check_rope(r) == 0 and E.rope_table_bytes(r) == 32768 * 128 * 4
    assert (r.theta, r.factor, r.amplitude) == (10000.0, 1.0, 1.0)
    assert E.lib().epikv_default_rope(None) == E.EPIKV_EINVAL_NULL
    assert E.lib().epikv_check_rope(None) == E.EPIKV_EINVAL_NULL


@pytest.mark.parametrize("field,value,code", [("kv_format", 2, -3), ("kv_format", -1, -3)])
def test_cfg_rejects(E, field, value, code):
    c = E.default_cfg(**{field: value})
    assert E.check_cfg(c) == code and E.kv_row_bytes(c) == 0


@pytest.mark.parametrize("signal", [1, 2, 3, 4])
def test_kv_signals_need_bf16_rows(E, signal):
    c = E.default_cfg(signal=signal, smoothing=E.SMOOTH_MEAN)
    assert E.check_cfg(c) == 0
    c.kv_format = E.KV_MXFP4
    assert E.check_cfg(c) == E.EPIKV_EINVAL_PARAM


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw,code", [
    (dict(rotary_dim=8), -2), (dict(rotary_dim=24), -2), (dict(rotary_dim=1040), -2), (dict(rotary_dim=-16), -2),
    (dict(n_pos=0), -2), (dict(n_pos=(1 << 24) + 1), -2), (dict(layout=2), -3), (dict(scaling=5), -3),
    (dict(scaling=-1), -3), (dict(theta=1.0), -3), (dict(theta=NAN), -3), (dict(theta=INF), -3),
    (dict(amplitude=0.0), -3), (dict(amplitude=NAN), -3), (dict(scaling=1, factor=0.0), -3),
    (dict(scaling=2, factor=INF), -3), (dict(scaling=3, factor=8.0, original=0), -3),
    (dict(scaling=3, turns_low=0.0), -3), (dict(scaling=4, turns_low=4.0, turns_high=4.0), -3),
    (dict(scaling=4, turns_high=INF), -3)])
def test_rope_cfg_rejects(E, kw, code):
    r = E.default_rope(**kw)
    assert E.check_rope(r) == code and E.rope_table_bytes(r) == 0
    assert E.lib().epikv_rope_table(ctypes.byref(r), A, None) == code


def test_rope_table_rejects(E):
    r, f = E.default_rope(), E.lib().epikv_rope_table
    assert f(ctypes.byref(r), None, None) == E.EPIKV_EINVAL_NULL
    assert f(ctypes.byref(r), A + 4, None) == E.EPIKV_EALIGN


def rows(E, base, heads=4, d=128, chunk=3):
    return E.Rows(base, chunk * heads * d, heads * d, d)


def test_rope_rejects(E):
    L = E.lib()
    r = E.default_rope()

    def call(x=None, y=None, table=A, dtype=0, B=2, C=3, heads=4, d=128, pos=5 * A, ld=0, rope=r):
        x, y = x or rows(E, 2 * A), y or rows(E, 3 * A)
        return L.epikv_rope(ctypes.byref(rope), table, dtype, B, C, heads, d, ctypes.byref(x),
                            ctypes.byref(y), pos, ld, 0, None, None)
    assert call(table=None) == E.EPIKV_EINVAL_NULL
    assert call(pos=None) == E.EPIKV_EINVAL_NULL
    assert call(x=E.Rows(None, 0, 0, 0)) == E.EPIKV_EINVAL_NULL
    assert call(dtype=2) == E.EPIKV_EINVAL_PARAM
    for kw in (dict(B=0), dict(C=0), dict(heads=0), dict(heads=2000), dict(d=120), dict(d=2048), dict(d=64),
               dict(ld=2), dict(B=1 << 16, C=1 << 16)):
        assert call(**kw) == E.EPIKV_EINVAL_SHAPE, kw
    assert call(table=A + 8) == E.EPIKV_EALIGN
    assert call(x=rows(E, 2 * A + 8)) == E.EPIKV_EALIGN
    assert call(x=E.Rows(2 * A, 1536, 516, 128)) == E.EPIKV_EALIGN
    assert call(x=E.Rows(2 * A, -1536, 512, 128)) == E.EPIKV_EINVAL_SHAPE
    # written rows that overlap each other: heads, tokens, sequences
    for st in ((1536, 512, 64), (1536, 256, 128), (512, 512, 128), (0, 512, 128), (1536, 0, 128)):
        assert call(y=E.Rows(3 * A, *st)) == E.EPIKV_EINVAL_SHAPE, st
    # read rows may be broadcast; the call goes on to the next check
    assert call(x=E.Rows(2 * A, 0, 0, 0), y=rows(E, 2 * A)) == E.EPIKV_EALIAS
    assert call(y=rows(E, 2 * A + 256)) == E.EPIKV_EALIAS
    assert call(y=E.Rows(2 * A, 1536, 128, 384)) == E.EPIKV_EALIAS


def pool(E, base=A, page=32768):
    return E.Pool(base, 1 << 30, 1 << 29, page, 100)


def append_io(E, **kw):
    io = E.AppendIO()
    io.chunk, io.layer, io.pool = 3, 1, pool(E)
    io.page_table, io.ld_pt, io.n_cached = 2 * A, 8, 3 * A
    io.k, io.v = rows(E, 4 * A, 8), rows(E, 5 * A, 8)
    io._rope = E.default_rope()
    io.rope, io.rope_table = ctypes.pointer(io._rope), 6 * A
    io.positions, io.ld_pos = 7 * A, 0
    io.n_heads, io.q, io.q_out = 32, rows(E, 8 * A, 32), rows(E, 9 * A, 32)
    io.pos, io.ld_s = 10 * A, 64
    for k, v in kw.items():
        setattr(io, k, v)
    return io


def test_append_rejects(E):
    f = E.lib().epikv_append
    c = E.default_cfg(batch=2, n_layers=4)

    def call(cfg=c, **kw):
        return f(ctypes.byref(cfg), ctypes.byref(append_io(E, **kw)), None)
    none = E.Rows(None, 0, 0, 0)
    assert f(None, ctypes.byref(append_io(E)), None) == E.EPIKV_EINVAL_NULL
    assert f(ctypes.byref(c), None, None) == E.EPIKV_EINVAL_NULL
    for kw in (dict(page_table=None), dict(n_cached=None), dict(k=none), dict(v=none), dict(q_out=none),
               dict(rope_table=None), dict(positions=None), dict(rope=None, positions=None),
               dict(pool=E.Pool(None, 0, 0, 0, 0))):
        assert call(**kw) == E.EPIKV_EINVAL_NULL, kw
    for kw in (dict(chunk=0), dict(chunk=-1), dict(chunk=(1 << 24) + 1), dict(layer=4), dict(layer=-1),
               dict(ld_pt=0), dict(n_heads=0), dict(n_heads=1025), dict(ld_pos=2), dict(ld_s=0),
               dict(q_out=E.Rows(9 * A, 3 * 4096, 4096, 64))):
        assert call(**kw) == E.EPIKV_EINVAL_SHAPE, kw
    assert call(_rope2=0, rope=ctypes.pointer(E.default_rope(rotary_dim=256))) == E.EPIKV_EINVAL_SHAPE
    assert call(rope=ctypes.pointer(E.default_rope(theta=0.5))) == E.EPIKV_EINVAL_PARAM
    for kw in (dict(k=rows(E, 4 * A + 8, 8)), dict(v=E.Rows(5 * A, 4, 1024, 128)), dict(rope_table=6 * A + 8),
               dict(pool=pool(E, A + 8)), dict(pool=pool(E, A, 32776))):
        assert call(**kw) == E.EPIKV_EALIGN, kw
    for kw in (dict(q_out=rows(E, 8 * A + 64, 32)), dict(q_out=rows(E, 4 * A, 32)), dict(q_out=rows(E, 5 * A, 32))):
        assert call(**kw) == E.EPIKV_EALIAS, kw
    bad = E.default_cfg(batch=0)
    assert call(cfg=bad) == E.EPIKV_EINVAL_SHAPE


def test_read_rejects(E):
    f = E.lib().epikv_read
    c = E.default_cfg(batch=2, n_layers=4)

    def call(**kw):
        io = E.ReadIO()
        io.chunk, io.layer, io.pool = 3, 1, pool(E)
        io.page_table, io.ld_pt, io.first = 2 * A, 8, 3 * A
        io.k, io.v = rows(E, 4 * A, 8), rows(E, 5 * A, 8)
        for k, v in kw.items():
            setattr(io, k, v)
        return f(ctypes.byref(c), ctypes.byref(io), None)
    none = E.Rows(None, 0, 0, 0)
    assert f(ctypes.byref(c), None, None) == E.EPIKV_EINVAL_NULL
    assert call(k=none, v=none) == E.EPIKV_EINVAL_NULL
    assert call(first=None) == E.EPIKV_EINVAL_NULL
    assert call(chunk=0) == E.EPIKV_EINVAL_SHAPE
    assert call(k=E.Rows(4 * A, 0, 1024, 128)) == E.EPIKV_EINVAL_SHAPE
    assert call(v=rows(E, 5 * A + 2, 8)) == E.EPIKV_EALIGN
    assert call(v=rows(E, 4 * A + 256, 8)) == E.EPIKV_EALIAS


def test_attend_rejects(E):
    f = E.lib().epikv_attend
    c = E.default_cfg(batch=2, n_layers=4)
    W = 40 * A

    def call(cfg=c, **kw):
        io = E.AttendIO()
        io.chunk, io.layer, io.pool = 3, 1, pool(E)
        io.page_table, io.ld_pt, io.n_cached = 2 * A, 8, 3 * A
        io.n_heads, io.q, io.out = 32, rows(E, 8 * A, 32), rows(E, 9 * A, 32)
        io.lse = 10 * A
        io.workspace, io.workspace_bytes = W, 1 << 40
        for k, v in kw.items():
            setattr(io, k, v)
        return f(ctypes.byref(cfg), ctypes.byref(io), None)
    none = E.Rows(None, 0, 0, 0)
    for kw in (dict(q=none), dict(out=none), dict(page_table=None), dict(n_cached=None)):
        assert call(**kw) == E.EPIKV_EINVAL_NULL, kw
    for kw in (dict(n_heads=0), dict(n_heads=12), dict(n_heads=1032), dict(chunk=0), dict(layer=4), dict(ld_pt=0),
               dict(out=E.Rows(9 * A, 0, 4096, 128))):
        assert call(**kw) == E.EPIKV_EINVAL_SHAPE, kw
    for scale in (-1.0, NAN, INF):
        assert call(scale=scale) == E.EPIKV_EINVAL_PARAM
    assert call(q=rows(E, 8 * A + 2, 32)) == E.EPIKV_EALIGN
    assert call(out=rows(E, 8 * A, 32)) == E.EPIKV_EALIAS
    assert call(out=rows(E, 8 * A + 1024, 32)) == E.EPIKV_EALIAS
    need = E.attend_workspace_bytes(c, 3, 32)
    if need:
        assert call(workspace=None) == E.EPIKV_EWORKSPACE
        assert call(workspace_bytes=need - 1) == E.EPIKV_EWORKSPACE
        assert call(workspace=W + 8) == E.EPIKV_EALIGN
        for other in (8 * A, 9 * A, 10 * A, 2 * A, 3 * A):
            assert call(workspace=other) == E.EPIKV_EALIAS
    assert E.attend_workspace_bytes(c, 0, 32) == 0 and E.attend_workspace_bytes(c, 3, 12) == 0


def test_binding_refuses_other_shapes(E):
    """Tensors that a kernel would read or write past their end."""
    import torch
    c = E.default_cfg(batch=2, n_layers=1)

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype)
    i = t(2, 8, dtype=torch.int32)
    with pytest.raises(ValueError):
        E.make_append_io(3, pool(E), 0, i, 8, i, t(2, 3, 8, 128), t(2, 3, 4, 128))
    with pytest.raises(ValueError):
        E.make_append_io(3, pool(E), 0, i, 8, i, t(2, 2, 8, 128), t(2, 2, 8, 128))
    with pytest.raises(ValueError):
        E.make_append_io(3, pool(E), 0, i, 8, i, t(2, 3, 8, 128), t(2, 3, 8, 128), q=t(2, 3, 32, 64),
                         q_out=t(2, 3, 32, 64))
    with pytest.raises(ValueError):
        E.make_attend_io(3, pool(E), 0, i, 8, i, t(2, 3, 32, 128), t(2, 3, 32, 128, dtype=torch.float32))
    with pytest.raises(ValueError):
        E.make_attend_io(3, pool(E), 0, i, 8, i, t(2, 3, 32, 128), t(2, 3, 32, 128),
                         lse=t(2, 32, 2, dtype=torch.float32))
    with pytest.raises(ValueError):
        E.rows_of(t(2, 3, 128, 8).transpose(2, 3))
    with pytest.raises(ValueError):
        E.make_read_io(3, pool(E), 0, i, 8, i, t(2, 3, 8, 128), t(2, 3, 8, 64))
    io = E.make_append_io(3, pool(E), 0, i, 8, i, t(2, 3, 4, 128), t(2, 3, 4, 128))
    with pytest.raises(ValueError):
        E.epikv_append(c, io)  # 4 KV heads against 8
    io = E.make_attend_io(3, pool(E), 0, i, 8, i, t(3, 3, 32, 128), t(3, 3, 32, 128))
    with pytest.raises(ValueError):
        E.epikv_attend(c, io)
    with pytest.raises(ValueError):
        E.epikv_rope_table(E.default_rope(), t(16, dtype=torch.float32))

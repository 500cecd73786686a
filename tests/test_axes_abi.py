"""Refusals of the rotary calls with several axes (CPU: every call here fails
on the host, before a launch), and the oracle's deal of the pairs."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.cache_ref as R

A = 1 << 20  # fake, aligned addresses, never dereferenced
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation runs only without a GPU")
NULL, SHAPE, PARAM, ALIGN, ALIAS = -1, -2, -3, -4, -6


@pytest.fixture(scope="module")
def E():
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


@pytest.mark.parametrize("pairs,kw,code", [
    ((16, 24, 24), {}, 0), ((64,), {}, 0), ((1, 1, 61, 1), {}, 0), ((16, 24, 23), {}, SHAPE), ((16, 24, 25), {}, SHAPE),
    ((64, 0), {}, SHAPE), ((65, -1), {}, SHAPE), ((), {}, SHAPE), ((32, 32), dict(order=2), PARAM),
    ((32, 32), dict(order=-1), PARAM), ((32, 32), dict(frequencies=2), PARAM), ((2 ** 31 - 1, 2 ** 31 - 1), {}, SHAPE)])
def test_axes(E, pairs, kw, code):
    r, x = E.default_rope(), E.axes_of(pairs, **kw)
    assert E.check_axes(r, x) == code
    got = E.lib().epikv_rope_axes_table(ctypes.byref(r), ctypes.byref(x), A + 4, None)
    assert got == (ALIGN if code == 0 else code)
    assert E.lib().epikv_check_axes(ctypes.byref(r), None) == NULL
    assert E.lib().epikv_check_axes(None, ctypes.byref(x)) == NULL


def test_number_of_axes(E):
    with pytest.raises(ValueError, match="axes"):
        E.axes_of((13, 13, 13, 13, 12))
    x = E.axes_of((32, 32))
    x.n_axes = 5
    assert E.check_axes(E.default_rope(), x) == SHAPE


def test_ntk_needs_two_pairs(E):
    """Its base is raised to r / (r - 2)."""
    r = E.default_rope(scaling=E.ROPE_NTK, factor=4.0)
    assert E.check_axes(r, E.axes_of((63, 1))) == 0
    assert E.check_axes(r, E.axes_of((63, 1), frequencies=E.AXES_APART)) == SHAPE
    assert E.check_axes(r, E.axes_of((62, 2), frequencies=E.AXES_APART)) == 0


def rows(E, base, heads=4, d=128, chunk=3):
    return E.Rows(base, chunk * heads * d, heads * d, d)


def test_rope_axes_rejects(E):
    def call(x=None, y=None, table=A, dtype=0, B=2, C=3, heads=4, d=128, pos=5 * A, ld=0, axes=None):
        x, y = x or rows(E, 2 * A), y or rows(E, 3 * A)
        axes = axes or E.axes_of((16, 24, 24))
        return E.lib().epikv_rope_axes(ctypes.byref(E.default_rope()), ctypes.byref(axes), table, dtype, B, C, heads, d,
                                       ctypes.byref(x), ctypes.byref(y), pos, ld, 0, None, None)
    for kw, code in ((dict(table=None), NULL), (dict(pos=None), NULL), (dict(x=E.Rows(None, 0, 0, 0)), NULL),
                     (dict(dtype=2), PARAM), (dict(B=0), SHAPE), (dict(C=0), SHAPE), (dict(heads=0), SHAPE),
                     (dict(d=64), SHAPE), (dict(ld=2), SHAPE), (dict(ld=-1), SHAPE), (dict(table=A + 8), ALIGN),
                     (dict(x=rows(E, 2 * A + 2)), ALIGN), (dict(y=rows(E, 2 * A + 256)), ALIAS),
                     (dict(axes=E.axes_of((16, 24, 23))), SHAPE)):
        assert call(**kw) == code, kw


def test_append_axes_rejects(E):
    c = E.default_cfg(batch=2, n_kv_heads=4, head_dim=128)
    rope = E.default_rope()

    def call(axes=(16, 24, 24), ids=9 * A, ld_ids=0, with_rope=True, pos=8 * A, **kw):
        io = E.AppendIO()
        io.chunk, io.layer, io.pool = 3, 0, E.Pool(A, 1 << 16, 1 << 16, 1 << 14, 4)
        io.page_table, io.ld_pt, io.n_cached = 2 * A, 4, 3 * A
        io.k, io.v = rows(E, 4 * A), rows(E, 5 * A)
        io.rope = ctypes.pointer(rope) if with_rope else None
        io.rope_table, io.positions, io.pos, io.ld_s = 6 * A, 7 * A, pos, 64
        for k, v in kw.items():
            setattr(io, k, v)
        return E.lib().epikv_append_axes(ctypes.byref(c), ctypes.byref(io), ctypes.byref(E.axes_of(axes)) if axes else None,
                                         ids, ld_ids, None)
    for kw, code in ((dict(axes=None), NULL), (dict(with_rope=False), NULL), (dict(ids=None), NULL),
                     (dict(ld_ids=2), SHAPE), (dict(ld_ids=-1), SHAPE), (dict(axes=(16, 24)), SHAPE),
                     (dict(positions=None), NULL), (dict(rope_table=None), NULL), (dict(rope_table=6 * A + 8), ALIGN),
                     (dict(ld_pos=2), SHAPE), (dict(n_cached=None), NULL), (dict(layer=32), SHAPE), (dict(ld_s=0), SHAPE),
                     (dict(chunk=0), SHAPE)):
        assert call(**kw) == code, kw


def ints(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


def test_binding(E):
    """Tensors too small or of another type are refused before the library
    takes their addresses."""
    B, C, H, d = 3, 2, 2, 64
    t = torch.zeros(B, C, H, d, dtype=torch.bfloat16)
    rope, axes = E.default_rope(rotary_dim=d, n_pos=32), E.axes_of((8, 12, 12))
    table = torch.zeros(32, d // 2, 2)

    def rotate(positions, ld=0, table=table):
        E.epikv_rope_axes(rope, axes, table, E.DTYPE_BF16, B, C, H, d, t, t.clone(), positions, ld, stream=0)
    for bad, ld in ((ints(B, 2), 0), (ints(B, 3, dtype=torch.int64), 0), (ints(B, 3, 1), 2), (ints(B, 2, 2), 2)):
        with pytest.raises(ValueError, match="positions"):
            rotate(bad, ld)
    with pytest.raises(ValueError, match="table"):
        rotate(ints(B, 3), table=table[1:])
    with pytest.raises(ValueError, match="table"):
        E.epikv_rope_axes_table(rope, axes, table[1:], stream=0)

    def io(**kw):
        a = dict(chunk=C, pool=E.Pool(), layer=0, page_table=ints(B, 8), ld_pt=8, n_cached=ints(B), k=t, v=t, rope=rope,
                 table=table, positions=ints(B, 3), axes=axes, ids=ints(B), pos=ints(B, 20), ld_s=20)
        return E.make_append_io(**{**a, **kw})
    cfg = E.default_cfg(batch=B, n_kv_heads=H, head_dim=d)
    for kw, what in ((dict(positions=ints(B, 2)), "positions"), (dict(ids=ints(B - 1)), "ids"),
                     (dict(ids=ints(B, dtype=torch.int64)), "ids"), (dict(ids=ints(B, 1), ld_ids=2), "ids"),
                     (dict(positions=ints(B, 3, 1), ld_pos=2), "positions"), (dict(axes=None), "without axes")):
        with pytest.raises(ValueError, match=what):
            E.epikv_append_axes(cfg, io(**kw), stream=0)
    with pytest.raises(ValueError, match="with axes"):
        E.epikv_append(cfg, io(), stream=0)
    for call in (io(), io(positions=ints(B, 3, C), ld_pos=C, ids=ints(B, C), ld_ids=C)):
        with pytest.raises(E.EpikvError) as e:  # as far as the library, which refuses the empty pool
            E.epikv_append_axes(cfg, call, stream=0)
        assert e.value.status == NULL


def test_oracle_deals_pairs():
    assert R.axes_of_pairs((2, 1, 3), False) == ([0, 0, 1, 2, 2, 2], [0, 1, 0, 0, 1, 2])
    assert R.axes_of_pairs((2, 1, 3), True) == ([0, 1, 2, 0, 2, 2], [0, 0, 0, 1, 1, 2])
    f = R.rope_axes_frequencies((2, 2), False, True, 100.0)
    assert np.allclose(f, [1.0, 0.1, 1.0, 0.1])
    assert np.array_equal(R.rope_axes_frequencies((2, 2), True, False, 100.0), R.rope_frequencies(8, 100.0))

"""The binding's checks of the cache calls' integer tensors and rotary tables:
the kernels take their addresses, so a wrong type or too few entries would be
read (or written) past the end.  CPU: refused before the library is reached."""
import pytest
import torch

B, C, H, HQ, D = 3, 2, 2, 4, 64


@pytest.fixture(scope="module")
def E():
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


def rows(heads=H, b=B):
    return torch.zeros(b, C, heads, D, dtype=torch.bfloat16)


def append(E, **kw):
    a = dict(chunk=C, pool=E.Pool(), layer=0, page_table=ints(B, 8), ld_pt=8, n_cached=ints(B), k=rows(), v=rows(),
             n_new=ints(B), rope=E.default_rope(rotary_dim=D, n_pos=32), table=torch.zeros(32, D // 2, 2),
             positions=ints(B), q=rows(HQ), q_out=rows(HQ), pos=ints(B, 20), ld_s=20, seq_status=ints(B))
    return E.epikv_append, E.make_append_io(**{**a, **kw})


def attend(E, **kw):
    a = dict(chunk=C, pool=E.Pool(), layer=0, page_table=ints(B, 8), ld_pt=8, n_cached=ints(B), q=rows(HQ),
             out=rows(HQ), n_new=ints(B), seq_status=ints(B))
    return E.epikv_attend, E.make_attend_io(**{**a, **kw})


def read(E, **kw):
    a = dict(chunk=C, pool=E.Pool(), layer=0, page_table=ints(B, 8), ld_pt=8, first=ints(B), k=rows(), v=rows(),
             seq_status=ints(B))
    return E.epikv_read, E.make_read_io(**{**a, **kw})


def refused(E, make, what, **kw):
    """By the binding: at the latest when the call learns the batch."""
    cfg = E.default_cfg(batch=B, n_kv_heads=H, head_dim=D)
    with pytest.raises(ValueError, match=what):
        call, io = make(E, **kw)
        call(cfg, io, stream=0)


def passes(E, make, **kw):
    """As far as the library, which refuses the empty pool."""
    call, io = make(E, **kw)
    with pytest.raises(E.EpikvError) as e:
        call(E.default_cfg(batch=B, n_kv_heads=H, head_dim=D), io, stream=0)
    assert e.value.status == E.EPIKV_EINVAL_NULL


CALLS = [(append, "n_cached"), (append, "n_new"), (append, "positions"), (append, "seq_status"),
         (attend, "n_cached"), (attend, "n_new"), (attend, "seq_status"), (read, "first"), (read, "seq_status")]


@pytest.mark.parametrize("make,name", CALLS)
def test_counts(E, make, name):
    passes(E, make)
    for bad in (ints(B, dtype=torch.int64), ints(B, dtype=torch.float32), ints(B - 1), ints(2 * B)[::2],
                ints(1).expand(B)):
        refused(E, make, name, **{name: bad})
    passes(E, make, **{name: ints(2 * B)[B:]})
    passes(E, make, **{name: 1 << 20})  # an address


@pytest.mark.parametrize("make", [append, attend, read])
def test_page_tables(E, make):
    for bad in (ints(B, 8, dtype=torch.int64), ints(B, 7), ints(B - 1, 8), ints(8, B).T, ints(B, 12)[:, 5:]):
        refused(E, make, "page_table", page_table=bad)
    refused(E, make, "page_table", page_table=ints(B, 12)[:, 4:], ld_pt=12)  # (the last row ends past it)
    passes(E, make, page_table=ints(B, 12)[:, :8], ld_pt=12)  # part of a wider table
    passes(E, make, page_table=ints(B * 8))


def test_ids_and_positions(E):
    for bad in (ints(B, 20, dtype=torch.int64), ints(B, 19), ints(B - 1, 20)):
        refused(E, append, "pos", pos=bad)
    passes(E, append, positions=ints(B, C), ld_pos=C)
    refused(E, append, "positions", positions=ints(B), ld_pos=C)
    refused(E, append, "positions", positions=ints(B, C, dtype=torch.int64), ld_pos=C)


@pytest.mark.parametrize("table", [torch.zeros(31, D // 2, 2), torch.zeros(32, D // 2, 2, dtype=torch.float64),
                                   torch.zeros(32, D // 2, 2, dtype=torch.bfloat16),
                                   torch.zeros(32, D // 2, 4)[..., :2]])
def test_rotary_tables(E, table):
    refused(E, append, "table", table=table)
    with pytest.raises(ValueError, match="table"):
        E.epikv_rope(E.default_rope(rotary_dim=D, n_pos=32), table, E.DTYPE_BF16, B, C, H, D, rows(), rows(), ints(B))


@pytest.mark.parametrize("name,bad", [("positions", ints(B, dtype=torch.int64)), ("positions", ints(B - 1)),
                                      ("seq_status", ints(B, dtype=torch.int64)), ("seq_status", ints(B - 1))])
def test_rope(E, name, bad):
    a = dict(positions=ints(B), seq_status=None)
    with pytest.raises(ValueError, match=name):
        E.epikv_rope(E.default_rope(rotary_dim=D, n_pos=32), torch.zeros(32, D // 2, 2), E.DTYPE_BF16, B, C, H, D,
                     rows(), rows(), **{**a, name: bad})

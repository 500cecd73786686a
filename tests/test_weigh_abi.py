"""Refusals of epikv_attend_weigh (CPU: every call here fails on the host,
before a launch), and the oracle's sums."""
import ctypes

import numpy as np
import pytest
import torch

import oracle.cache_ref as R

A = 1 << 24  # fake, aligned addresses, never dereferenced
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation runs only without a GPU")
NULL, SHAPE, PARAM, ALIGN, WORKSPACE, ALIAS = -1, -2, -3, -4, -5, -6
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def E():
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


B, C, HQ, H, D, LD_PT, LD_S = 2, 3, 8, 4, 128, 40, 600


def call(E, io_kw=None, need=0, **kw):
    cfg = E.default_cfg(batch=B, n_kv_heads=H, head_dim=D)

    def rows(base):
        return E.Rows(base, C * HQ * D, HQ * D, D)
    io = E.AttendIO()
    io.chunk, io.layer, io.pool = C, 0, E.Pool(A, 1 << 16, 1 << 16, 1 << 14, 4)
    io.page_table, io.ld_pt, io.n_cached, io.n_new, io.n_heads = 2 * A, LD_PT, 3 * A, 4 * A, HQ
    io.q, io.out, io.lse, io.seq_status = rows(5 * A), rows(6 * A), 7 * A, 8 * A
    io.workspace, io.workspace_bytes = 9 * A, need
    for k, v in (io_kw or {}).items():
        setattr(io, k, v)
    w = E.WeighIO(old=20 * A, weights=21 * A, ld_s=LD_S, keep_old=1.0, keep_new=0.0, gain=1.0, watch=0)
    for k, v in kw.items():
        setattr(w, k, v)
    return E.lib().epikv_attend_weigh(ctypes.byref(cfg), ctypes.byref(io), ctypes.byref(w), None)


@pytest.mark.parametrize("kw,code", [
    (dict(weights=None), NULL), (dict(ld_s=0), SHAPE), (dict(watch=-1), SHAPE), (dict(keep_old=-0.5), PARAM),
    (dict(keep_old=1.5), PARAM), (dict(keep_old=NAN), PARAM), (dict(keep_new=2.0), PARAM), (dict(keep_new=NAN), PARAM),
    (dict(gain=0.0), PARAM), (dict(gain=-1.0), PARAM), (dict(gain=NAN), PARAM), (dict(gain=INF), PARAM),
    (dict(weights=21 * A + 2), ALIGN), (dict(old=20 * A + 1), ALIGN), (dict(old=21 * A + 4), ALIAS),
    (dict(old=21 * A - 4 * B * LD_S + 4), ALIAS), (dict(old=6 * A), ALIAS), (dict(old=7 * A), ALIAS),
    (dict(weights=2 * A), ALIAS), (dict(weights=3 * A), ALIAS), (dict(weights=4 * A), ALIAS), (dict(weights=5 * A), ALIAS),
    (dict(weights=6 * A), ALIAS), (dict(weights=7 * A), ALIAS), (dict(weights=8 * A), ALIAS), ({}, WORKSPACE),
    (dict(old=21 * A), WORKSPACE), (dict(old=21 * A + 4 * B * LD_S), WORKSPACE), (dict(old=None), WORKSPACE)])
def test_sums_rejects(E, kw, code):
    """(What passes every check ends at the workspace, of which there is none.)"""
    assert call(E, **kw) == code


def test_attend_rejects(E):
    for kw, code in ((dict(n_cached=None), NULL), (dict(page_table=None), NULL), (dict(chunk=0), SHAPE),
                     (dict(layer=32), SHAPE), (dict(n_heads=6), SHAPE), (dict(scale=-1.0), PARAM),
                     (dict(ld_pt=0), SHAPE)):
        assert call(E, kw) == code, kw
    L, cfg = E.lib(), E.default_cfg()
    io, w = E.AttendIO(), E.WeighIO()
    assert L.epikv_attend_weigh(None, ctypes.byref(io), ctypes.byref(w), None) == NULL
    assert L.epikv_attend_weigh(ctypes.byref(cfg), None, ctypes.byref(w), None) == NULL
    assert L.epikv_attend_weigh(ctypes.byref(cfg), ctypes.byref(io), None, None) == NULL


def test_workspace(E):
    cfg = E.default_cfg(batch=B, n_kv_heads=H, head_dim=D)
    need = E.attend_weigh_workspace_bytes(cfg, C, HQ, LD_PT)
    assert need >= E.attend_workspace_bytes(cfg, C, HQ)
    assert call(E, need=need - 1) == WORKSPACE
    assert call(E, dict(workspace=None), need=need) == WORKSPACE
    assert call(E, dict(workspace=9 * A + 8), need=need) == ALIGN
    for at in (2, 3, 4, 5, 6, 7, 8, 20, 21):  # every other argument
        assert call(E, dict(workspace=at * A), need=need) == ALIAS, at
    for bad in (dict(chunk=0), dict(n_heads=6), dict(ld_pt=0), dict(watch=-1)):
        a = {**dict(chunk=C, n_heads=HQ, ld_pt=LD_PT, watch=0), **bad}
        assert E.attend_weigh_workspace_bytes(cfg, **a) == 0
    # the most a table can cover is bounded, whatever it says
    big = E.attend_weigh_workspace_bytes(cfg, C, HQ, 1 << 62)
    assert big == E.attend_weigh_workspace_bytes(cfg, C, HQ, 1 << 30)


def test_binding(E):
    cfg = E.default_cfg(batch=B, n_kv_heads=H, head_dim=D)
    q = torch.zeros(B, C, HQ, D, dtype=torch.bfloat16)
    n = torch.zeros(B, dtype=torch.int32)
    io = E.make_attend_io(C, E.Pool(), 0, torch.zeros(B, 4, dtype=torch.int32), 4, n, q, q.clone())
    good = torch.zeros(B, 64)
    for bad in (good.double(), good[:, ::2], torch.zeros(64, B).T):
        with pytest.raises(ValueError, match="weights"):
            E.make_weigh_io(bad, bad.shape[1])
        with pytest.raises(ValueError, match="old"):
            E.make_weigh_io(good, bad.shape[1], old=bad)
    for w in (E.make_weigh_io(good, 65), E.make_weigh_io(good[:1].clone(), 64),
              E.make_weigh_io(good, 64, old=good[:1].clone())):
        with pytest.raises(ValueError, match="sums for"):
            E.epikv_attend_weigh(cfg, io, w, stream=0)
    with pytest.raises(ValueError, match="batch"):
        E.epikv_attend_weigh(E.default_cfg(batch=B + 1, n_kv_heads=H, head_dim=D), io, E.make_weigh_io(good, 64), stream=0)
    with pytest.raises(E.EpikvError) as e:
        E.epikv_attend_weigh(cfg, io, E.make_weigh_io(good, 64), stream=0)
    assert e.value.status == NULL  # (the empty pool)


def test_oracle():
    """The weights are the softmax that the oracle's attention uses, and every
    query's add up to 1."""
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    w = R.attend_weights(q, k, 3, 0.5)
    out, *_ = R.attend(q, k, v, 3, 0.5)
    assert np.allclose(np.einsum("chn,nhd->chd", w, np.repeat(v, 2, 1)), out)
    assert np.allclose(w.sum(-1), 1) and np.all(w[0, :, 5:] == 0)
    old = np.arange(7.0)
    got = R.weigh(w, old, 3, 0.5, 0.0, 2.0, 1)
    assert np.allclose(got, np.where(np.arange(7) < 4, 0.5 * old, 0) + 2 * w[2].sum(0))
    assert np.allclose(R.weigh(w, None, 3, 1.0, 1.0, 1.0, 0).sum(), 12)

"""The eviction step over a cache held in 4 bits: the rows it keeps are moved
byte for byte in all three rebuild modes, alone and inside the step, and
attention over the rebuilt cache reads what it read before."""
import numpy as np
import pytest
import torch

import oracle as O
from cache_harness import DEV, Cache, bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def all_rows(c, layers, b, table, n):
    """[layers][2][n][row] of a sequence through a host table."""
    host = c.bytes.cpu().numpy()
    s = np.arange(n)
    pg = table[b, s // c.page]
    at = (s % c.page)[:, None] * c.row + np.arange(c.row)
    return host[:, :, pg[:, None], at]


@pytest.mark.parametrize("H,d,page", [(8, 128, 16), (1, 64, 16), (4, 64, 7), (5, 64, 32), (8, 256, 16),
                                      (3, 128, 1)])
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_rebuilds_move_whole_rows(E, H, d, page, mode):
    rng = np.random.default_rng(H * 10 + d + mode)
    g = torch.Generator(device=DEV).manual_seed(3)
    B, K, L = 3, 96, 2
    n = [400, 97, 300]
    c = Cache(E, rng, E.KV_MXFP4, B, H, d, page, 400, layers=L, budget=K)
    c.bytes.random_(0, 256, generator=g)
    before = [all_rows(c, L, b, c.table_host, n[b]) for b in range(B)]
    scores = torch.randn(B, 400, device=DEV, generator=g)
    if mode == 2:  # whole pages evicted, so that some are remapped
        scores[0, 32:32 + 4 * page] = -50
    keep = torch.zeros(B, K, dtype=torch.int32, device=DEV)
    nk, status = ints([0] * B), ints([0] * B)
    E.epikv_select(c.cfg, scores, 400, ints(n), ints([4, 0, 8]), keep, nk, status)
    kept = keep.cpu().numpy()
    need = E.compact_workspace_bytes(c.cfg)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    if mode == 0:
        dst = Cache(E, rng, E.KV_MXFP4, B, H, d, page, K, layers=L, budget=K)
        E.epikv_compact(c.cfg, c.pool, c.table, c.ld_pt, dst.pool, dst.table, dst.ld_pt, keep, nk,
                        seq_status=status, workspace=ws, workspace_bytes_=need)
        table = dst.table_host
    else:
        dst = c
        f = E.epikv_compact_inplace if mode == 1 else E.epikv_compact_remap
        f(c.cfg, c.pool, c.table, c.ld_pt, keep, nk, seq_status=status, workspace=ws, workspace_bytes_=need)
        table = c.table.cpu().numpy()
    assert not status.any().item()
    for b in range(B):
        assert np.array_equal(all_rows(dst, L, b, table, K), before[b][:, :, kept[b]])


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_step_and_attention_over_what_it_keeps(E, mode):
    """Scores, kept set and rows of the step; then attention over the rebuilt
    cache equals attention over the old one with the evicted slots gone."""
    import oracle.cache_ref as R
    rng = np.random.default_rng(mode)
    B, K, C, L, H, d, page, D, na, nb = 2, 128, 16, 2, 2, 128, 16, 512, 2, 2
    n = [333, 200]
    c = Cache(E, rng, E.KV_MXFP4, B, H, d, page, 340, layers=L, layer=1, budget=K, hidden=D, n_band_a=na,
              n_band_b=nb)
    held = []
    for b in range(B):
        got = []
        for kv in range(2):
            raw, val = c.encode(rng.standard_normal((n[b], H, d)))
            c.fill_rows(b, kv, raw)
            c.bytes[0, kv] = c.bytes[1, kv]
            got.append(val)
        held.append(got)
    hid = torch.randn(na + nb, B, C, D, device=DEV).bfloat16()
    st = torch.zeros(2, E.state_bytes(c.cfg), dtype=torch.uint8, device=DEV)
    scores = torch.randn(B, 400, device=DEV)
    keep = torch.zeros(B, K, dtype=torch.int32, device=DEV)
    nk, status = ints([0] * B), ints([0] * B)
    need = E.workspace_bytes(c.cfg, C)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    dst = Cache(E, rng, E.KV_MXFP4, B, H, d, page, K, layers=L, layer=1, budget=K) if mode == 0 else c
    ids = torch.arange(400, dtype=torch.int32, device=DEV).expand(B, 400).contiguous()
    dsc, dids = torch.zeros_like(scores), torch.zeros_like(ids)
    io = E.make_step_io(C, list(hid), D, C * D, ints(n), ints([0, 0]), c.pool, c.table, c.ld_pt, dst.pool,
                        dst.table, dst.ld_pt, scores, 400, st[0], st[1], keep, nk, status, ws, need,
                        dst_scores=dsc if mode == 0 else None, src_pos=ids, dst_pos=dids if mode == 0 else ids,
                        in_place=mode)
    E.epikv_evict_step(c.cfg, io)
    assert not status.any().item() and nk.tolist() == [K, K]
    kept = keep.cpu().numpy()
    final = (scores if mode == 0 else None)
    got_ids = (dids if mode == 0 else ids).cpu().numpy()
    for b in range(B):
        if final is not None:
            assert np.array_equal(kept[b], O.select_keep(final.cpu().numpy()[b, :n[b]], 0, K))
        assert np.array_equal(got_ids[b, :K], kept[b])
    q, q64 = bf16(rng.standard_normal((B, 1, 4, d)))
    need = E.attend_workspace_bytes(dst.cfg, 1, 4)
    ws = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    for layer in range(L):
        out = torch.zeros(B, 1, 4, d, dtype=torch.bfloat16, device=DEV)
        E.epikv_attend(dst.cfg, E.make_attend_io(1, dst.pool, layer, dst.table, dst.ld_pt, nk, q, out,
                                                 workspace=ws, workspace_bytes_=need))
        for b in range(B):
            ref, _, mag, _ = R.attend(q64[b], held[b][0][kept[b]], held[b][1][kept[b]], 1, d ** -0.5)
            # bf16 of weights and result, 2^-8 each, and 1e-4 for the scores
            assert np.all(np.abs(out[b].double().cpu().numpy() - ref)
                          <= 2.0 ** -8 * 1.01 * (mag + np.abs(ref)) + 1e-4 * mag)

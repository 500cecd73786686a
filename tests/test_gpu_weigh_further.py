"""Sequences longer than the workgroups that a batch's sums are dealt to: each goes
on to further slots."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache, bf16, f64
from test_gpu_weigh import FMTS, expected, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


# (16384 tiles of 256 slots, 128 where many rows have 256 channels, for all
# sequences: 3584, 1792 and 13824 slots of one here)
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,C,heads,long", [
    (1100, 1, (4, 2, 64), 8000), (1100, 3, (4, 2, 128), 7201), (1100, 20, (4, 2, 64), 8000), (1100, 20, (2, 1, 128), 11111),
    (1100, 20, (2, 1, 256), 4001), (300, 1, (4, 2, 64), 28000), (300, 30, (4, 2, 64), 28000)])
def test_further_slots(E, fmt, B, C, heads, long):
    Hq, H, d = heads
    page, short = 64, 80
    rng = np.random.default_rng(B + C)
    width, narrow = -(-long // page), -(-short // page)
    at = [0, 7, B - 1]  # the long ones
    n = rng.integers(C, short + 1, B)
    n[at] = [long, long - 1000, long - page + 1]
    n[3], nn = 0, np.full(B, C)
    nn[3], nn[7] = 0, max(1, C - 1)
    c = Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, B, H, d, page, short, spare=len(at) * width)
    rest = np.setdiff1d(np.arange(B * narrow + len(at) * width), c.table_host)
    table = np.full((B, width), -1, np.int32)
    table[:, :narrow] = c.table_host
    table[at] = rng.permutation(rest).reshape(len(at), width)
    c.table_host, c.table, c.ld_pt = table, torch.from_numpy(table).to(DEV), width
    held = {}
    looked_at = at + [1, 2, B // 2]
    for b in range(B):
        if b in looked_at or b % 16 == 0:
            kv = [c.encode(rng.standard_normal((n[b], H, d))) for _ in range(2)]
            for i in range(2):
                c.fill_rows(b, i, kv[i][0])
            held[b] = [x[1] for x in kv]
    q, q64 = bf16(rng.standard_normal((B, C, Hq, d)))
    before = torch.from_numpy(rng.exponential(1.0, (B, long + 3)).astype(np.float32)).to(DEV)
    w = torch.full_like(before, 7.0)
    _, _, status = run(E, c, C, n.tolist(), q, nn=nn.tolist(), weights=w, old=before, keep_old=0.5, keep_new=0.25)
    assert not status.any().item()
    w = f64(w)
    for b in looked_at:
        want, tol = expected(q64[b, :nn[b]], *held[b], int(nn[b]), d ** -0.5, f64(before[b, :int(n[b])]), 0.5, 0.25, 1.0, 0)
        off = np.abs(w[b, :n[b]] - want)
        assert np.all(off <= tol), (b, np.nanmax(off / tol), int(np.nanargmax(off / tol)))
        assert np.all(w[b, n[b]:] == 7.0), b
    assert np.all(w[3] == 7.0)

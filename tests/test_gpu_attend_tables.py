"""Attention where the page tables are much wider than the sequences, and where
the sequences hold so much that their rows bypass the caches."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache
from test_gpu_attend import check, run

pytestmark = pytest.mark.gpu
FMTS = ["bf16", "mxfp4"]


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C,n", [(1, [700, 33, 4224, 0]), (4, [4, 1000, 129]), (1, [50] * 100), (1, [40] * 1030),
                                 (40, [2000, 41])])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 1, 64), (4, 2, 256)])
def test_wide_tables_change_nothing(E, fmt, C, n, heads):
    """A table for 128k slots whose further entries are no pages (they must
    not be read as such): the bits of the tight table's call."""
    Hq, H, d = heads
    B, page = len(n), 16
    rng = np.random.default_rng(C + B)
    c = Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, B, H, d, page, max(n))
    for b in range(B):
        for i in range(2):
            c.fill_rows(b, i, c.encode(rng.standard_normal((n[b], H, d)))[0])
    q = torch.randn(B, C, Hq, d, device=DEV).bfloat16()
    nn = [min(m, C) for m in n]
    want, wl, _ = run(E, c, C, n, q, nn)
    wide = torch.full((B, 131072 // page), -1, dtype=torch.int32, device=DEV)
    wide[:, :c.ld_pt] = c.table
    c.ld_pt = wide.shape[1]
    got, gl, status = run(E, c, C, n, q, nn, table=wide)
    assert torch.equal(want.view(torch.int16), got.view(torch.int16))
    assert torch.equal(wl, gl) and not status.any().item()


@pytest.mark.parametrize("C,heads,n,nn", [(1, (8, 8, 128), [17003, 1, 0, 16001], [1, 1, 0, 1]),
                                          (2, (8, 4, 256), [33100, 2], [2, 1])])
def test_many_bytes_in_shares(E, C, heads, n, nn):
    """More rows than the caches keep, cut into shares and joined."""
    assert 4 * heads[1] * heads[2] * sum(n) > 128 << 20
    check(E, "bf16", len(n), C, *heads, 16, n, nn)

"""Attention in the plans that small calls do not reach: many query rows walked
whole (no pieces, no join), with four and with eight wavefronts, row tiles
from 24 on in both orders, few pieces; and for few rows head counts that do not
fill a workgroup's wavefronts.

What plan a shape gets depends on the compute units; a call whose workspace is
empty walks every row whole."""
import numpy as np
import pytest
import torch

from test_gpu_attend import check

pytestmark = pytest.mark.gpu
FMTS = ["bf16", "mxfp4"]


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def workspace(E, fmt, B, C, Hq, H, d):
    cfg = E.default_cfg(batch=B, n_layers=1, n_kv_heads=H, head_dim=d,
                        kv_format=E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4)
    assert E.check_cfg(cfg) == 0
    return E.attend_workspace_bytes(cfg, C, Hq)


def ragged(B, C, most, seed):
    """Counts: a full chunk alone, one with a past, partly padding, empty."""
    rng = np.random.default_rng(seed)
    nn = [C] * B
    n = [C + int(rng.integers(0, most)) for _ in range(B)]
    n[0] = C
    if B > 2:
        nn[1], n[1] = 0, 0
        nn[2] = C // 2 + 1
    if B > 3:
        nn[3], n[3] = 1, most + C
    return n, nn


WHOLE = [  # B, C, Hq, H, d
    (17, 257, 8, 8, 64),     # eight wavefronts, two row tiles
    (9, 33, 128, 16, 128),   # eight, two, 8 query heads a KV head
    (33, 20, 16, 8, 128),    # four wavefronts: no more than 128 rows
    (40, 17, 16, 8, 64),
    (33, 18, 8, 8, 256),     # rows of 256 channels
    (17, 65, 32, 8, 256),   # and three row tiles
]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", WHOLE)
def test_rows_walked_whole(E, fmt, shape):
    B, C, Hq, H, d = shape
    assert workspace(E, fmt, *shape) == 0
    n, nn = ragged(B, C, 130, sum(shape))
    check(E, fmt, B, C, Hq, H, d, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,C,H,whole", [
    (1, 370, 6, True),   # 47 row tiles in one round, one sequence: long with short
    (1, 380, 6, True),   # 48
    (2, 370, 3, True),   # 47 row tiles of two sequences
    (1, 370, 5, False),  # 47, in two pieces
    (3, 370, 1, False),
])
def test_many_row_tiles(E, fmt, B, C, H, whole):
    """16 query heads a KV head: 24 row tiles of 256 rows and more, where four
    wavefronts take 128 each."""
    shape = (B, C, 16 * H, H, 64)
    assert (workspace(E, fmt, *shape) == 0) == whole
    n, nn = ragged(B, C, 300, C + H)
    check(E, fmt, *shape, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("B,H", [(5, 10), (4, 10), (3, 9)])
def test_few_pieces(E, fmt, B, H):
    shape = (B, 257, H, H, 64)
    assert workspace(E, fmt, *shape) > 0
    n, nn = ragged(B, 257, 700, B)
    check(E, fmt, *shape, 16, n, nn)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", [(17, 257, 8, 8, 64), (33, 20, 16, 8, 128), (33, 18, 8, 8, 256)])
def test_hidden_slots_of_whole_walks(E, fmt, shape):
    """NaN and infinities in a later token's key and value (and in every unused
    byte) do not reach the tokens before it."""
    B, C, Hq, H, d = shape
    assert workspace(E, fmt, *shape) == 0
    n = [C + 3 * b for b in range(B)]

    def edit(b, k, v):
        at = n[b] - C + C // 2
        k[at, 0, 3] = np.nan
        v[at, H - 1, 5], v[at, 0, 9] = np.nan, np.inf
    check(E, fmt, *shape, 16, n, edit=edit)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("C", [1, 3])
@pytest.mark.parametrize("H,d", [(9, 64), (11, 64), (9, 128), (11, 128), (17, 64), (5, 256), (7, 256), (8, 256)])
def test_heads_that_do_not_fill_a_workgroup(E, fmt, C, H, d):
    """Some wavefronts of the last group have no head, and leave before the
    others' barriers."""
    n = [3000, 17, 0, 515]
    check(E, fmt, 4, C, 2 * H, H, d, 16, n, [C, C, 0, C])

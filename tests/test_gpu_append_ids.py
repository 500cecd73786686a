"""Token ids of epikv_append where the row of ids is shorter than the cache."""
import numpy as np
import pytest
import torch

from cache_harness import DEV, Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("ld_s", [7, 8, 9, 16])
def test_ids_without_a_place_flag_their_sequence(fmt, ld_s):
    """The rows are written all the same, ids only inside their own row."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv as E
    B, C, H, d = 3, 3, 2, 64
    n = [3, 8, 10]  # slots 0..2, 5..7, 7..9
    c = Cache(E, np.random.default_rng(1), fmt, B, H, d, 4, 16, fill=0)
    k = torch.randn(B, C, H, d, device=DEV).bfloat16()

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)
    room = torch.full((B + 1, ld_s), -5, dtype=torch.int32, device=DEV)
    status = ints([0] * B)
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), k, k,
                                           positions=ints([100, 200, 300]), pos=room, ld_s=ld_s, seq_status=status))
    with_ids = c.bytes.clone()
    want = torch.full((B + 1, ld_s), -5, dtype=torch.int32)
    for b in range(B):
        for i in range(C):
            if n[b] - C + i < ld_s:
                want[b, n[b] - C + i] = 100 * (b + 1) + i
    assert torch.equal(room.cpu(), want)
    assert status.tolist() == [E.SEQ_RANGE if m > ld_s else E.SEQ_OK for m in n]
    c.bytes.zero_()
    E.epikv_append(c.cfg, E.make_append_io(C, c.pool, 0, c.table, c.ld_pt, ints(n), k, k))
    assert torch.equal(c.bytes, with_ids)

"""The binding refuses fewer layers of hidden states than the configuration
scores (the library reads an address for each), and the example refuses
settings that would leave a band without a layer or a token without a
position (CPU: every call here is refused before the library is reached)."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="refusals only, checked without a GPU")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def E():
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


def test_scoring_needs_every_band_layer(E):
    c = E.default_cfg(batch=2, n_band_a=1, n_band_b=1, hidden=64)
    h = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    for hidden in ([], [h]):
        with pytest.raises(ValueError, match="2 band layers"):
            E.epikv_score(c, 3, hidden, 64, 192, state_in=1 << 20, state_out=2 << 20, sig=3 << 20)
        with pytest.raises(ValueError, match="2 band layers"):
            E.epikv_score_tokens(c, 3, hidden, 64, 192, 4 << 20, 1 << 20, 2 << 20, 3 << 20, 8)
        io = E.make_step_io(3, hidden, 64, 192, 4 << 20, 5 << 20, E.Pool(), None, 1, E.Pool(), None, 1,
                            3 << 20, 8, 1 << 20, 2 << 20, 6 << 20, 7 << 20, 8 << 20, None, 0)
        for step in (E.epikv_evict_step, E.epikv_evict_step_noalloc):
            with pytest.raises(ValueError, match="2 band layers"):
                step(c, io)


def test_more_layers_or_none_go_on_to_the_library(E):
    """What the library itself refuses stays its own to refuse."""
    c = E.default_cfg(batch=2, n_band_a=1, n_band_b=1, hidden=64)
    h = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    for hidden, code in ((None, E.EPIKV_EINVAL_NULL), ([h, h, h], E.EPIKV_EINVAL_NULL)):
        with pytest.raises(E.EpikvError) as e:
            E.epikv_score(c, 3, hidden, 64, 192, state_in=1 << 20, state_out=2 << 20, stream=0)  # (no sig)
        assert e.value.status == code


@pytest.mark.parametrize("kw", [dict(layers=1), dict(layers=0), dict(prompt=0), dict(prompt=101, max_positions=100)])
def test_the_example_refuses_its_settings(kw):
    from decode_evict import Decoder
    with pytest.raises(ValueError):
        Decoder(**kw)


def test_the_example_refuses_tokens_past_its_positions():
    import decode_evict as X
    X.check_positions(100, 3996, 4096)
    with pytest.raises(ValueError):
        X.check_positions(100, 3997, 4096)
    with pytest.raises(ValueError):  # 100 of the prompt, 64 to warm up, 4000 timed
        X.main(["--tokens", "4000"])
    with pytest.raises(ValueError):
        X.main(["--layers", "1"])

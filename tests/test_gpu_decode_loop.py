"""The example's decode loop, end to end: after a prompt, tokens and several
evictions, the cache's ids say which tokens are held, and attention equals the
64-bit attention over exactly those."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import f64, quick_encode

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
@pytest.mark.parametrize("prompt,tokens", [(40, 100), (70, 33)])
def test_decode_loop(fmt, prompt, tokens):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from decode_evict import Decoder
    m = Decoder(batch=3, layers=3, hidden=256, heads=8, kv_heads=2, head_dim=64, prompt=prompt, budget=96,
                every=16, fmt=fmt, history=True)
    m.run(tokens)
    torch.cuda.synchronize()
    assert not m.status.any().item()
    n = m.n_cached.tolist()
    total = prompt + tokens
    assert m.position.tolist() == [total] * 3 and all(x <= 96 + 16 for x in n)
    assert total <= 112 or all(x < total for x in n)  # something was evicted
    table = f64(m.table).reshape(-1, 32, 2)
    ids = m.pos.cpu().numpy()
    for l in range(m.L):
        k = torch.cat([x[0] for x in m.history[l]], 1)
        v = f64(torch.cat([x[1] for x in m.history[l]], 1))
        cs = m.table.view(-1, 32, 2)[:total]
        c, s = cs[..., 0].view(1, total, 1, 32), cs[..., 1].view(1, total, 1, 32)
        a, b = k[..., :32], k[..., 32:]
        k = torch.cat([a * c - b * s, b * c + a * s], -1)  # the library's float32 steps
        k = f64(k.bfloat16() if fmt == "bf16" else k)
        if fmt != "bf16":
            def held(x):
                flat = x.reshape(-1, 128)
                return R.mxfp4_decode(R.mxfp4_pack(*quick_encode(flat), 128), 128).reshape(x.shape)
            k, v = held(k), held(v)
        q, out = m.last[l]
        for b in range(3):
            kept = ids[b, :n[b]]
            assert np.all(np.diff(kept) > 0) and kept[-1] == total - 1
            assert np.array_equal(kept[:prompt], np.arange(prompt))  # the prompt stays
            ref, _, mag, _ = R.attend(f64(q)[b], k[b, kept], v[b, kept], 1, 64 ** -0.5)
            # weights and result in bf16: 2^-8 each; 1e-4 for the scores
            assert np.all(np.abs(f64(out)[b] - ref) <= 1.01 * 2.0 ** -8 * (mag + np.abs(ref)) + 1e-4 * mag)
    assert table.shape[0] == 4096

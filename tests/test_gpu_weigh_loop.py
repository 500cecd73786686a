"""The example's decode loop with the weights' policy and an image before the
text, end to end: positions on three axes go into the cache, attention equals the
64-bit attention over the held tokens, the sums are those of the weights of all
layers since each token came, and the step keeps the largest of them."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle as O
import oracle.cache_ref as R
from cache_harness import f64, quick_encode

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def turned(m, k, at, fmt):
    """Keys as the cache holds them: the library's float32 steps by the turns of
    each pair's axis."""
    axis = torch.tensor(R.axes_of_pairs([m.axes.pairs[i] for i in range(3)], True)[0], device=k.device)
    table = m.table.view(-1, m.d // 2, 2)
    cs = table[at[:, axis].transpose(1, 2).long(), torch.arange(m.d // 2, device=k.device)]
    c, s = cs[..., 0].unsqueeze(2), cs[..., 1].unsqueeze(2)
    a, b = k[..., :m.d // 2], k[..., m.d // 2:]
    k = torch.cat([a * c - b * s, b * c + a * s], -1)
    return f64(k.bfloat16() if fmt == "bf16" else k)


@pytest.mark.parametrize("fmt", ["bf16", "mxfp4"])
@pytest.mark.parametrize("image,prompt,tokens", [(5, 40, 100), (0, 70, 33), (8, 64, 40)])
def test_weights_loop(fmt, image, prompt, tokens):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from decode_evict import Decoder
    B, budget, every, sinks = 3, 48, 16, 4
    m = Decoder(batch=B, layers=3, hidden=256, heads=8, kv_heads=2, head_dim=64, prompt=prompt, budget=budget,
                every=every, fmt=fmt, history=True, policy="weights", sinks=sinks, image=image)
    # what the loop's sums have to be, token by token, and what every step kept
    sums = [np.zeros(prompt) for _ in range(B)]
    err = [np.zeros(prompt) for _ in range(B)]
    held = [np.arange(prompt) for _ in range(B)]
    evicted, fed = [0], [0]

    def weigh(n_new):
        """The last feed's weights by the oracle, over what is held."""
        keys, vals = [], []
        for l in range(m.L):
            k = torch.cat([x[0] for x in m.history[l]], 1)
            v = f64(torch.cat([x[1] for x in m.history[l]], 1))
            at = torch.cat([x[2] for x in m.history[l]], 2)
            k = turned(m, k, at, fmt)
            if fmt != "bf16":
                def kept_as(x):
                    return R.mxfp4_decode(R.mxfp4_pack(*quick_encode(x.reshape(-1, 128)), 128), 128).reshape(x.shape)
                k, v = kept_as(k), kept_as(v)
            keys.append(k)
            vals.append(v)
        for b in range(B):
            for l in range(m.L):
                q, out = m.last[l]
                k, v = keys[l][b, held[b]], vals[l][b, held[b]]
                w = R.attend_weights(f64(q)[b], k, n_new, 64 ** -0.5)
                ref, lse, mag, size = R.attend(f64(q)[b], k, v, n_new, 64 ** -0.5)
                # (weights and result in bf16: 2^-8 each; 1e-4 for the scores)
                assert np.all(np.abs(f64(out)[b] - ref) <= 1.01 * 2.0 ** -8 * (mag + np.abs(ref)) + 1e-4 * mag)
                eps = (64 + 4) * 2.0 ** -24 * size + 2.0 ** -20
                row = 2 * eps + 2.0 ** -20 * (1 + np.abs(lse))
                sums[b] += w.sum((0, 1))
                err[b] += (w * np.moveaxis(row, -1, 0)[..., None]).sum((0, 1)) + (8 * n_new + 4) * 2.0 ** -24 * sums[b]

    plain_evict, plain_feed = m.evict, m.feed

    def feed(x):
        n = x.shape[1]
        if fed[0]:
            for b in range(B):
                held[b] = np.append(held[b], m.ids[b].item())
                sums[b], err[b] = np.append(sums[b], 0.0), np.append(err[b], 0.0)
        fed[0] += 1
        y = plain_feed(x)
        weigh(n)
        got = f64(m.scores)
        for b in range(B):
            assert np.all(np.abs(got[b, :sums[b].size] - sums[b]) <= err[b]), b
        return y

    def evict():
        before = [m.scores[b, :held[b].size].cpu().numpy() for b in range(B)]
        plain_evict()
        evicted[0] += 1
        for b in range(B):
            keep = O.select_keep(before[b], sinks, budget)
            assert m.n_cached[b].item() == keep.size
            held[b], sums[b], err[b] = held[b][keep], sums[b][keep], err[b][keep]
            assert np.array_equal(m.pos[b, :keep.size].cpu().numpy(), held[b])
            assert np.array_equal(m.scores[b, :keep.size].cpu().numpy(), before[b][keep])

    m.evict, m.feed = evict, feed
    m.run(tokens)
    assert not m.status.any().item() and m.ids.tolist() == [prompt + tokens] * B
    assert evicted[0] == (tokens - 1) // every
    assert m.position.tolist() == [prompt + tokens - image * image + image] * B


def test_refusals():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from decode_evict import Decoder
    for kw in (dict(policy="all"), dict(image=11, prompt=100)):
        with pytest.raises(ValueError):
            Decoder(layers=2, hidden=256, **kw)

"""The weights that attention sums are normalised however large its scores are,
and which rows count."""
import math

import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import DEV, Cache, bf16, f64
from test_gpu_weigh import FMTS, fill, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


# (chunk, heads, lengths): a few rows whole and in shares, with the log-sums made
# beside the join (one sequence) and after it (many slots, many sequences); tiles
# of rows, in pieces and not, of every number of channels.
FORMS = [(1, (8, 2, 64), [40]), (1, (8, 2, 128), [900]), (3, (4, 2, 128), [700, 33]), (1, (4, 1, 256), [5000]),
         (2, (8, 2, 64), [40000, 30000]), (1, (4, 2, 64), [30] * 1100), (40, (8, 2, 64), [40]),
         (60, (8, 2, 128), [1000, 60]), (30, (4, 1, 256), [600]), (700, (8, 2, 64), [700]),
         # (as many rows as a walk can have, 16 of 32 KV heads)
         (1, (512, 32, 64), [900]), (4, (128, 32, 64), [33, 400])]


def cache_of(E, fmt, rng, C, heads, n):
    _, H, d = heads
    return Cache(E, rng, E.KV_BF16 if fmt == "bf16" else E.KV_MXFP4, len(n), H, d, 16, max(n))


def offset_scores(E, fmt, C, heads, n, offset, seed=1):
    """Queries and keys of small whole numbers, and in one block of 32 channels
    one channel that adds `offset` (a power of two) to every score: the products
    and their sums are exact in 32 bits."""
    Hq, H, d = heads
    rng = np.random.default_rng(seed + C)
    c = cache_of(E, fmt, rng, C, heads, n)
    sign, power = math.copysign(1.0, offset), int(math.log2(abs(offset)))

    def edit(b, k, v):
        k[:] = rng.integers(-2, 3, k.shape)
        k[:, :, 32:64] = 0.0
        k[:, :, 40] = sign * 2.0 ** (power // 2)
        v[:] = 1.0
    held = fill(c, rng, n, H, d, edit)
    x = rng.integers(-1, 2, (len(n), C, Hq, d)).astype(np.float64)
    x[..., 32:64] = 0.0
    x[..., 40] = 2.0 ** (power - power // 2)
    return (c, held) + bf16(x)


def no_weights(n):
    return torch.zeros(len(n), max(n), device=DEV)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(str(x) for x in (f[0],) + f[1] + (max(f[2]), len(f[2]))))
@pytest.mark.parametrize("offset", [1.0, 2.0 ** 14, -2.0 ** 20, 2.0 ** 22])
def test_offsets_change_no_weight(E, fmt, form, offset):
    """Every score with the same large number on it, the sums against 64 bits.
    A weight's exponent is rounded once, by 2^-24 of 64 at most where it matters
    (weights above 2^-64), and holds the rounding of scale * log2(e), 2^-23 of
    a score's distance from the largest (64 at most there): 2^-17 together, and
    as much again in the sum that it is divided by and by the shares' maxima; the
    exponentials 2^-22; a slot's sum 2^-24 for each of its terms, and a row's
    for each of its slots."""
    C, heads, n = form
    c, held, q, q64 = offset_scores(E, fmt, C, heads, n, offset)
    w = no_weights(n)
    run(E, c, C, n, q, weights=w, scale=0.125)
    w = f64(w)
    for b in sorted({0, len(n) // 2, len(n) - 1}):
        want = R.weigh(R.attend_weights(q64[b], held[b][0], C, 0.125), None, C, 1.0, 0.0, 1.0, 0)
        tol = (2.0 ** -15 + (n[b] + C * heads[0]) * 2.0 ** -24) * want + C * heads[0] * 2.0 ** -60
        off = np.abs(w[b, :n[b]] - want)
        assert np.all(off <= tol), (b, (off / tol).max(), want.max())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(str(x) for x in (f[0],) + f[1] + (max(f[2]), len(f[2]))))
@pytest.mark.parametrize("scale", [0.0, 1e2, 1e4, 1e6])
def test_weights_of_a_row_add_up_to_one(E, fmt, form, scale):
    """Whatever the scores: a sequence's sums add up to its tokens times heads.
    (Exponents as above; a row's sum and a slot's by 2^-24 of each term.)"""
    C, heads, n = form
    rng = np.random.default_rng(7)
    c = cache_of(E, fmt, rng, C, heads, n)
    fill(c, rng, n, *heads[1:])
    q, _ = bf16(rng.standard_normal((len(n), C) + (heads[0], heads[2])))
    w = no_weights(n)
    run(E, c, C, n, q, weights=w, scale=scale)
    rows = C * heads[0]
    off = np.abs(f64(w).sum(1) / rows - 1.0)
    assert off.max() <= 2.0 ** -15 + (max(n) + rows) * 2.0 ** -24, off.max()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "x".join(str(x) for x in (f[0],) + f[1] + (max(f[2]), len(f[2]))))
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_rows_past_two_to_the_thirtieth_do_not_count(E, fmt, form, sign):
    """Every slot's score the same: a row's weights are one over what it sees.
    Every other query head's log-sum is 0.98 times 2^30 and the rest's 1.96
    times, then 0.51 and 1.02; the former count, the latter do not.  (No score
    is rounded; a sum by 2^-24 of itself for each term, and its inverse.)"""
    C, heads, n = form
    Hq, H, d = heads
    rng = np.random.default_rng(5)
    c = cache_of(E, fmt, rng, C, heads, n)

    def edit(b, k, v):
        k[:] = 0.0
        k[:, :, 40] = sign * 2.0 ** 15
        v[:] = 1.0
    fill(c, rng, n, H, d, edit)
    x = np.zeros((len(n), C, Hq, d))
    x[:, :, 0::2, 40] = 2.0 ** 15
    x[:, :, 1::2, 40] = 2.0 ** 16
    q, _ = bf16(x)
    for scale in (0.98, 0.51):
        w = no_weights(n)
        _, lse, _ = run(E, c, C, n, q, weights=w, scale=scale)
        assert torch.all(lse[:, 0::2].abs() < 2.0 ** 30) and torch.all(lse[:, 1::2].abs() > 2.0 ** 30)
        assert torch.isfinite(lse).all()
        w = f64(w)
        for b in sorted({0, len(n) // 2, len(n) - 1}):
            seen = n[b] - C + 1 + np.arange(C)
            want = (Hq // 2) * ((np.arange(n[b])[None] < seen[:, None]) / seen[:, None]).sum(0)
            assert np.all(np.abs(w[b, :n[b]] - want) <= (2.0 ** -20 + (n[b] + C * Hq) * 2.0 ** -24) * want), (scale, b)

"""Rotary positions on the GPU against the 64-bit oracle: the table, both
layouts, parts of the head, both types, the gradient, strides, refusals of
positions."""
import numpy as np
import pytest
import torch

import oracle.cache_ref as R
from cache_harness import DEV, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26472_amd import epikv
    epikv.lib()
    return epikv


MODES = {"plain": 0, "linear": 1, "ntk": 2, "bands": 3, "yarn": 4}


def table_of(E, rope):
    t = torch.full((rope.n_pos, rope.rotary_dim // 2, 2), float("nan"), device=DEV)
    E.epikv_rope_table(rope, t)
    return t


@pytest.mark.parametrize("mode", sorted(MODES))
@pytest.mark.parametrize("r,n_pos", [(16, 1), (64, 777), (128, 40001), (256, 130)])
def test_table(E, mode, r, n_pos):
    """Rounded once from 64 bits: half a unit in the last place, and the 64-bit
    angle's own error (an angle of 40,000 to 2^-53 of itself)."""
    kw = dict(factor=8.0, original=8192, low=1.0, high=32.0 if mode == "yarn" else 4.0)
    theta = 500000.0
    rope = E.default_rope(rotary_dim=r, n_pos=n_pos, theta=theta, scaling=MODES[mode], factor=8.0,
                          original=8192, turns_low=1.0, turns_high=kw["high"], amplitude=1.25)
    got = f64(table_of(E, rope))
    ang = R.rope_angles(n_pos, r, theta, mode, **kw)
    ref = 1.25 * np.stack([np.cos(ang), np.sin(ang)], -1)
    assert np.abs(got - ref).max() <= 2.0 ** -23 * 1.25 / 2 + 1e-10


def reference(x, table, pos, il, transpose):
    t = table[pos]
    return R.rotate(x, t[..., 0], t[..., 1], il, transpose)



SHAPES = [(1, 1, 1, 16, 16), (32, 1, 32, 128, 128), (2, 37, 5, 64, 32), (3, 11, 7, 256, 64),
          (1, 300, 8, 128, 128), (2, 3, 3, 80, 48), (5, 2, 40, 96, 96), (1, 7, 1, 1024, 1024)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("il", [False, True])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotation(E, shape, il, transpose, dtype):
    """Two products and a sum in float32, rounded once to the type: 2^-24 of
    each product and of the sum, then 2^-8 (bf16: 8 significant bits) of the result; and bit for
    bit the same arithmetic in torch."""
    B, C, heads, d, r = shape
    g = torch.Generator().manual_seed(B * 100 + d)
    x = torch.randn(B, C, heads, d, generator=g) * torch.exp(torch.randn(d, generator=g))
    x = x.bfloat16() if dtype == "bf16" else x
    rope = E.default_rope(rotary_dim=r, n_pos=500, theta=10000.0, layout=int(il))
    table = table_of(E, rope)
    first = torch.randint(0, 500 - C + 1, (B,), generator=g, dtype=torch.int32)
    y = torch.full_like(x, float("nan")).to(DEV)
    xd = x.to(DEV)
    dt = E.DTYPE_BF16 if dtype == "bf16" else E.DTYPE_FP32
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    E.epikv_rope(rope, table, dt, B, C, heads, d, xd, y, first.to(DEV), transpose=transpose,
                 seq_status=status)
    pos = first.numpy()[:, None] + np.arange(C)
    th = table.cpu()
    ref = reference(f64(x), th.double().numpy(), pos, il, transpose)
    t = np.abs(th.double().numpy()[pos])
    big = np.maximum(np.abs(R.rotate(np.abs(f64(x)), t[..., 0], t[..., 1], il, True)),
                     np.abs(R.rotate(np.abs(f64(x)), t[..., 0], t[..., 1], il)))
    tol = 3 * 2.0 ** -24 * (big + np.abs(ref)) + (2.0 ** -8 * np.abs(ref) * 1.01 if dtype == "bf16" else 0)
    got = f64(y)
    assert np.all(np.abs(got - ref) <= tol + 1e-38)
    assert not status.any().item()
    # the same float32 steps
    cs = th[pos]
    c, s = cs[..., 0].unsqueeze(2), cs[..., 1].unsqueeze(2)
    s = -s if transpose else s
    xf, want = x.float(), x.float().clone()
    lo, hi = (slice(0, r, 2), slice(1, r, 2)) if il else (slice(0, r // 2), slice(r // 2, r))
    a, b = xf[..., lo], xf[..., hi]
    want[..., lo], want[..., hi] = a * c - b * s, b * c + a * s
    assert torch.equal(want.to(x.dtype), y.cpu())
    # in place
    E.epikv_rope(rope, table, dt, B, C, heads, d, xd, xd, first.to(DEV), transpose=transpose)
    assert torch.equal(xd.cpu(), y.cpu())


def test_gradient_is_the_derivative(E):
    """<w, dy/dx . e> by differences of a linear map is exact up to float32,
    and the transposed call gives the same inner products."""
    B, C, heads, d, r = 2, 5, 3, 64, 48
    g = torch.Generator().manual_seed(3)
    for il in (0, 1):
        rope = E.default_rope(rotary_dim=r, n_pos=64, layout=il, amplitude=1.125)
        table = table_of(E, rope)
        first = torch.tensor([7, 40], dtype=torch.int32, device=DEV)

        def run(v, tr=False):
            out = torch.empty_like(v)
            E.epikv_rope(rope, table, E.DTYPE_FP32, B, C, heads, d, v, out, first, transpose=tr)
            return out
        x = torch.randn(B, C, heads, d, generator=g).to(DEV)
        e = torch.randn(B, C, heads, d, generator=g).to(DEV)
        w = torch.randn(B, C, heads, d, generator=g).to(DEV)
        h = 1.0 / 64
        diff = (run(x + h * e).double() - run(x - h * e).double()) / (2 * h)
        num = (w.double() * diff).sum().item()
        ana = (run(w, True).double() * e.double()).sum().item()
        # 1920 terms of size ~1, each off by a few 2^-24 / h
        assert abs(num - ana) <= 1920 * 8 * 2.0 ** -24 * 64
        # and element for element the transposed matrix
        table64 = table.cpu().double().numpy()
        pos = np.array([[7], [40]]) + np.arange(C)
        ref = reference(f64(w), table64, pos, bool(il), True)
        assert np.abs(f64(run(w, True)) - ref).max() <= 2.0 ** -20


def test_strides_and_positions_per_token(E):
    """A view into a fused projection, a transposed output, packed documents
    (positions that restart)."""
    B, C, heads, d = 2, 9, 4, 64
    fused = torch.randn(B, C, heads + 3, d, device=DEV).bfloat16()
    x = fused[:, :, 2:2 + heads]
    y = torch.zeros(B, heads, C, d, device=DEV, dtype=torch.bfloat16)
    rope = E.default_rope(rotary_dim=64, n_pos=100)
    table = table_of(E, rope)
    pos = torch.tensor([[0, 1, 2, 0, 1, 50, 51, 0, 99, -7], [9, 8, 7, 6, 5, 4, 3, 2, 1, -7]],
                       dtype=torch.int32, device=DEV)
    E.epikv_rope(rope, table, E.DTYPE_BF16, B, C, heads, d, x, y.transpose(1, 2), pos, ld_pos=10)
    p = pos.cpu().numpy()[:, :C]
    ref = reference(f64(x), f64(table), p, False, False)
    assert np.abs(f64(y.transpose(1, 2)) - ref).max() <= 2.0 ** -8 * np.abs(ref).max()


def test_positions_out_of_range_leave_the_token(E):
    B, C, heads, d = 3, 4, 2, 32
    x = torch.randn(B, C, heads, d, device=DEV)
    y = torch.full_like(x, 7.0)
    rope = E.default_rope(rotary_dim=32, n_pos=10)
    table = table_of(E, rope)
    first = torch.tensor([8, -2, 6], dtype=torch.int32, device=DEV)
    status = torch.zeros(B, dtype=torch.int32, device=DEV)
    E.epikv_rope(rope, table, E.DTYPE_FP32, B, C, heads, d, x, y, first, seq_status=status)
    assert status.tolist() == [2, 2, 0]
    left = (y == 7.0).flatten(2).all(-1).cpu().numpy()
    assert left.tolist() == [[False, False, True, True], [True, True, False, False], [False] * 4]


def test_nan_and_infinity_stay_in_their_pairs(E):
    x = torch.ones(1, 1, 1, 64, device=DEV)
    x[..., 3], x[..., 40] = float("nan"), float("inf")
    rope = E.default_rope(rotary_dim=48, n_pos=8)
    y = torch.empty_like(x)
    E.epikv_rope(rope, table_of(E, rope), E.DTYPE_FP32, 1, 1, 1, 64, x, y,
                 torch.tensor([5], dtype=torch.int32, device=DEV))
    bad = (~torch.isfinite(y[0, 0, 0])).nonzero().flatten().tolist()
    assert bad == [3, 16, 27, 40]

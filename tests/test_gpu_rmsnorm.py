"""evomoe_add_rmsnorm, its backward and evomoe_quantize_mx8 against the float64 oracle."""
import numpy as np
import pytest
import torch

import synth_inputs as synth
from oracle import block_oracle as blk
from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {"f32": U, "bf16": 2.0 ** -8}
EPS = 1e-5
# tokens, columns: single rows, one vector, no multiple of a wave's, of a block's, and rows longer than a block holds at once
SIZES = {"f32": [(1, 4), (3, 64), (777, 260), (64, 768), (5, 4096), (2, 20480 + 4)],
         "bf16": [(1, 8), (7, 64), (777, 136), (300, 768), (33, 1032), (9, 4096), (2, 40960 + 8)]}
ALL = [(t, *s) for t in SIZES for s in SIZES[t]]


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def rows(rng, T, d, dtype, wide=False):
    v = rng.standard_normal((T, d)).astype(np.float32)
    if wide:
        v *= np.float32(10.0) ** rng.uniform(-6, 6, (T, 1)).astype(np.float32)
    return synth.round_to_storage(v, dtype)


def dev(a, dtype):
    return None if a is None else torch.from_numpy(a).cuda().to(B.torch_dtype(dtype))


def terms(d):
    """Additions behind a sum over a row: at most d / 256 + 1 vectors of 8 in one thread, then a tree; and some to spare."""
    return 8 * (d / 256 + 1) + 16


def check_mx8(q, scale, v, tol):
    """q and scale are a rounding of v, which the computation may have off by tol: the scale is one of the two that values within
    tol give, and an element is within half a step (2^-4 of it, or of the smallest normal number) and tol of v."""
    g = v.reshape(*v.shape[:-1], -1, 32)
    t = tol.reshape(g.shape)
    lo, hi = blk.mx8_scale(np.maximum((abs(g) - t).max(-1), 0)), blk.mx8_scale((abs(g) + t).max(-1))
    assert ((scale == lo) | (scale == hi)).all()
    s = np.repeat(scale, 32, axis=-1)
    assert (abs(q * s - v) <= np.maximum(2.0 ** -4 * abs(v), 2.0 ** -10 * s) * (1 + 2.0 ** -20) + 2 * tol).all()


@pytest.mark.parametrize("dtype,T,d", ALL)
@pytest.mark.parametrize("residual", [False, True])
def test_forward(ctx, dtype, T, d, residual):
    rng = np.random.default_rng(T + d)
    x, res = rows(rng, T, d, dtype, wide=True), rows(rng, T, d, dtype) if residual else None
    if T > 2:
        x[1] = 0
        if residual:
            res[1] = 0
    gamma = rng.standard_normal(d).astype(np.float32)
    shape = B.make_shape(T, d, 1, d, dtype, "gelu", 1)
    xd, rd, gd = dev(x, dtype), dev(res, dtype), torch.from_numpy(gamma).cuda()
    h, y, rstd = torch.full_like(xd, 7), torch.full_like(xd, 7), torch.full((T,), 7.0, device="cuda")
    eight = d % 32 == 0
    q, qs = B.mx8_empty((T, d)) if eight else (None, None)
    B.evomoe_add_rmsnorm(ctx, shape, xd, rd, gd, EPS, h, y, rstd, q, qs)
    want_h = synth.round_to_storage(x + res, dtype) if residual else x
    assert np.array_equal(h.float().cpu().numpy(), want_h)
    want, want_r = blk.rmsnorm(want_h, gamma, EPS)
    # the sum of squares: U for each addition; its root halves that; 6 roundings of the quotient, the root, the products
    tol = U * (terms(d) / 2 + 6)
    assert (abs(rstd.cpu().numpy()[:, None] - want_r) <= tol * want_r).all()
    assert (abs(y.double().cpu().numpy() - want) <= (tol + HALF_STEP[dtype]) * abs(want) + 1e-40).all()
    if eight:
        check_mx8(q.double().cpu().numpy(), qs.double().cpu().numpy(), want, tol * abs(want))
        # every choice of outputs gives the same values; in place, and to 8 bits alone
        q2, qs2 = B.mx8_empty((T, d))
        B.evomoe_add_rmsnorm(ctx, shape, xd, rd, gd, EPS, None, None, None, q2, qs2)
        assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(qs2.view(torch.uint8), qs.view(torch.uint8))
    xc, rc = xd.clone(), None if rd is None else rd.clone()
    y2 = torch.empty_like(y)
    B.evomoe_add_rmsnorm(ctx, shape, xc, rc, gd, EPS, rc if residual else xc, y2)       # the residual stream, updated in place
    assert torch.equal(y2, y) and torch.equal(rc if residual else xc, h)
    xc, rc = xd.clone(), None if rd is None else rd.clone()
    B.evomoe_add_rmsnorm(ctx, shape, xc, rc, gd, EPS, rc, xc)                           # y over x, h over the residual
    assert torch.equal(xc, y) and (not residual or torch.equal(rc, h))
    xc = xd.clone()
    B.evomoe_add_rmsnorm(ctx, shape, xc, rd, gd, EPS, None, xc)
    assert torch.equal(xc, y)


@pytest.mark.parametrize("dtype,T,d", ALL + [("bf16", 5000, 64), ("f32", 4100, 68)])
@pytest.mark.parametrize("with_dh", [False, True])
def test_backward(ctx, dtype, T, d, with_dh):
    rng = np.random.default_rng(T * 3 + d)
    h, dy, dh = rows(rng, T, d, dtype), rows(rng, T, d, dtype), rows(rng, T, d, dtype) if with_dh else None
    gamma = rng.standard_normal(d).astype(np.float32)
    if T > 2:
        h[2] = 0
    shape = B.make_shape(T, d, 1, d, dtype, "gelu", 1)
    hd, dyd, dhd, gd = dev(h, dtype), dev(dy, dtype), dev(dh, dtype), torch.from_numpy(gamma).cuda()
    y, rstd = torch.empty_like(hd), torch.empty(T, device="cuda")
    B.evomoe_add_rmsnorm(ctx, shape, hd, None, gd, EPS, None, y, rstd)
    ws = torch.empty(B.evomoe_workspace_bytes(shape), dtype=torch.uint8, device="cuda").fill_(255)
    dx, dgamma = torch.full_like(hd, 7), torch.full((d,), 7.0, device="cuda")
    B.evomoe_add_rmsnorm_bwd(ctx, shape, dyd, dhd, hd, gd, rstd, dx, dgamma, ws)
    (want_dx, want_dg), (mag_dx, mag_dg) = blk.rmsnorm_bwd(dy, dh, h, gamma, EPS)
    # rstd off by half its sum's error, the inner sum by its own, and 8 roundings
    far = U * (2 * terms(d) + 8) * mag_dx + HALF_STEP[dtype] * abs(want_dx)
    assert (abs(dx.double().cpu().numpy() - want_dx) <= far + 1e-40).all()
    # at most one addition for each token, whatever their order; rstd as above, 3 roundings of a term
    far = U * (T + terms(d) / 2 + 16) * mag_dg
    assert (abs(dgamma.double().cpu().numpy() - want_dg) <= far + 1e-40).all()
    # again, without dgamma and its workspace, over dy, over dh: the same
    dx2, dg2 = torch.empty_like(dx), torch.empty_like(dgamma)
    B.evomoe_add_rmsnorm_bwd(ctx, shape, dyd, dhd, hd, gd, rstd, dx2, dg2, ws)
    assert torch.equal(dx2, dx) and torch.equal(dg2, dgamma)
    B.evomoe_add_rmsnorm_bwd(ctx, shape, dyd, dhd, hd, gd, rstd, dx2.fill_(7), None)
    assert torch.equal(dx2, dx)
    over = dyd.clone()
    B.evomoe_add_rmsnorm_bwd(ctx, shape, over, dhd, hd, gd, rstd, over, dg2.fill_(7), ws)
    assert torch.equal(over, dx) and torch.equal(dg2, dgamma)
    if with_dh:
        over = dhd.clone()
        B.evomoe_add_rmsnorm_bwd(ctx, shape, dyd, over, hd, gd, rstd, over, dg2.fill_(7), ws)
        assert torch.equal(over, dx) and torch.equal(dg2, dgamma)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row(ctx, dtype):
    rng = np.random.default_rng(1)
    x = rows(rng, 6, 96, dtype)
    x[1, 5], x[3, 70], x[4, 0] = np.nan, np.inf, -np.inf
    shape = B.make_shape(6, 96, 1, 96, dtype, "gelu", 1)
    xd = dev(x, dtype)
    y, gd = torch.empty_like(xd), torch.ones(96, device="cuda")
    q, qs = B.mx8_empty((6, 96))
    B.evomoe_add_rmsnorm(ctx, shape, xd, None, gd, EPS, None, y, None, q, qs)
    yn, qn = y.float().cpu().numpy(), q.float().cpu().numpy()
    assert np.isfinite(yn[[0, 2, 5]]).all() and np.isfinite(qn[[0, 2, 5]]).all()
    assert np.isnan(yn[1]).all() and np.isnan(qn[1]).all()
    # an infinite square makes rstd 0: the infinity becomes a NaN, the others 0
    assert np.isnan(yn[3, 70]) and np.isnan(qn[3, 70]) and (np.delete(yn[3], 70) == 0).all() and np.isnan(yn[4, 0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 32), (3, 5, 96), (1000, 64), (7, 4096), (257, 1056)])
def test_quantize_bit_for_bit(ctx, dtype, shape):
    rng = np.random.default_rng(shape[-1])
    v = rng.standard_normal(shape).astype(np.float32) * np.float32(10.0) ** rng.uniform(-38, 37, shape[:-1] + (1,)).astype(np.float32)
    flat = v.reshape(-1, shape[-1])
    flat[0, :8] = [448, 449, -464, 464.1, 0, -0.0, 2.0 ** -9, 2.0 ** -10]
    if flat.shape[0] > 2:
        flat[1] = 0
        flat[2, :5] = [np.inf, -np.inf, np.nan, 3e38, 1e-45]
    v = synth.round_to_storage(v, dtype)
    q, s = B.mx8_empty(shape)
    B.evomoe_quantize_mx8(ctx, dev(v, dtype), q, s)
    want_q, want_s = blk.mx8(v)
    assert np.array_equal(s.double().cpu().numpy(), want_s)
    assert np.array_equal(q.double().cpu().numpy(), want_q, equal_nan=True)

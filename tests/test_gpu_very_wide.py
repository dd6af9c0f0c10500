"""Rows and tables so wide that one thread to an element, or one block to a slice of columns, would not fit a grid dimension (2^32
threads, 65536 blocks): the backward passes that add up partial tables, against the same formulas in float64, a run of columns at a time."""
import pytest
import torch

from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
RUN = 1 << 22


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def runs(d):
    return [slice(a, min(a + RUN, d)) for a in range(0, d, RUN)]


@pytest.mark.parametrize("d", [(1 << 26) + 4096 + 8, (1 << 28) + 64])
def test_norm_of_wide_rows(ctx, d):
    """dgamma of more columns than the blocks of one round hold, and than a thread each for sixteen partial rows allows."""
    T, eps = 2, 1e-5
    g = torch.Generator(device="cuda").manual_seed(d)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x, dy, gamma = new(T, d), new(T, d), new(d)
    y, rstd, dx, dgamma = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty_like(x), torch.full((d,), 7.0, device="cuda")
    s = B.make_shape(T, d, 1, 4, "f32", "relu", 1)
    ws = torch.empty(T * d * 4, dtype=torch.uint8, device="cuda")              # one partial row is enough for two rows
    B.evomoe_add_rmsnorm(ctx, s, x, None, gamma, eps, None, y, rstd)
    B.evomoe_add_rmsnorm_bwd(ctx, s, dy, None, x, gamma, rstd, dx, dgamma, ws)
    torch.cuda.synchronize()
    # sums over the row: d / 256 in a thread, a tree over the threads, each addition off by U of the sum of magnitudes so far
    chain = (d / 256 + 16) * U
    square, inner, size = (torch.zeros(T, 1, dtype=torch.float64, device="cuda") for _ in range(3))
    for c in runs(d):
        square += x[:, c].double().square().sum(1, keepdim=True)
    want = (square / d + eps).rsqrt()
    assert ((rstd[:, None] - want).abs() <= (chain + 4 * U) * want).all()
    r = rstd.double()[:, None]                                                 # as the backward reads it
    for c in runs(d):
        p = gamma[c].double() * dy[:, c].double() * x[:, c].double() * r
        inner += p.sum(1, keepdim=True) / d
        size += p.abs().sum(1, keepdim=True) / d
    for c in runs(d):
        n, b, gm = x[:, c].double() * r, dy[:, c].double(), gamma[c].double()
        assert ((y[:, c] - n * gm).abs() <= 3 * U * (n * gm).abs()).all()
        assert ((dgamma[c] - (b * n).sum(0)).abs() <= 4 * U * (b * n).abs().sum(0)).all(), c
        far = 6 * U * r * ((gm * b).abs() + n.abs() * size) + r * n.abs() * (chain + 4 * U) * size
        assert ((dx[:, c] - r * (gm * b - n * inner)).abs() <= far).all(), c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_wide_rows(ctx, dtype):
    """More than 2^30 elements of dW_g, and (float32) more than 65536 slices of columns."""
    T, d, E = 2, (1 << 24) + 256, 64
    dt = B.torch_dtype(dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device="cuda", dtype=dtype)
    x, dx_in, Wg, bg, dz = new(T, d, dtype=dt), new(T, d, dtype=dt), new(d, E), new(E), new(T, E)
    z, dWg, dbg, dx = torch.empty(T, E, device="cuda"), torch.full_like(Wg, 7.0), torch.empty(E, device="cuda"), dx_in.clone()
    s = B.make_shape(T, d, E, 8, dtype, "relu", 1)
    ws = torch.empty((T * E + (d + 1) * E) * 4, dtype=torch.uint8, device="cuda")     # one partial table
    B.evomoe_gate_logits(ctx, s, x, Wg, bg, z)
    B.evomoe_gate_logits_bwd(ctx, s, dz, x, Wg, dx, dWg, dbg, dx, ws)
    torch.cuda.synchronize()
    zd = dz.double()
    sums, size = bg.double().repeat(T, 1), bg.double().abs().repeat(T, 1)
    # dx of a bf16 layer: both factors to 16 bits, and the result half a step of bf16
    rough, step = (0.0, U) if dtype == "f32" else (2.0 ** -15, 2.0 ** -8)
    for c in runs(d):
        xd, Wd, into = x[:, c].double(), Wg[c].double(), dx_in[:, c].double()
        sums += xd @ Wd
        size += xd.abs() @ Wd.abs()
        outer, mag = xd[0, :, None] * zd[0], xd[0, :, None].abs() * zd[0].abs()
        outer, mag = outer + xd[1, :, None] * zd[1], mag + xd[1, :, None].abs() * zd[1].abs()
        assert ((dWg[c] - outer).abs() <= 8 * U * mag).all(), c
        Wt = Wd.t().contiguous()
        want, mag = into + zd @ Wt, into.abs() + zd.abs() @ Wt.abs()
        assert ((dx[:, c] - want).abs() <= (rough + 2 * E * U) * mag + step * want.abs()).all(), c
    assert ((z - sums).abs() <= (d / 16 + 20) * U * size).all()
    assert ((dbg - zd.sum(0)).abs() <= 4 * U * zd.abs().sum(0)).all()


def test_gate_of_a_wide_bf16_layer(ctx):
    """The split copy of W_g has more than 2^31 elements to a term.  x of -1 and 1, W_g of -1, 0 and 1 times 2^-12: every sum is exact."""
    T, d, E = 1, (1 << 25) + 64, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randint(0, 2, (T, d), generator=g, device="cuda").mul_(2).sub_(1).to(torch.bfloat16)
    Wg = torch.randint(-1, 2, (d, E), generator=g, device="cuda", dtype=torch.int8).float().mul_(2.0 ** -12)
    gp, gw = torch.empty(T, E, device="cuda"), torch.empty(T, E, device="cuda")
    mask, counts = torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    B.evomoe_dts_gate(ctx, B.make_shape(T, d, E, 8, "bf16", "relu", E), x, Wg, None, None, 1.0, 0.01, gp, gw, mask, counts, None)
    torch.cuda.synchronize()
    z = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    for c in runs(d):
        z += x[:, c].double() @ Wg[c].double()
    want = torch.softmax(z, 1)
    # softmax: the argument z - max, of up to 8, is rounded once (8 U), the exponential, a sum of 64 terms and the quotient take 24 more
    assert float((z.max() - z.min())) < 8
    assert ((gp - want).abs() <= 32 * U * want).all(), (gp, want)

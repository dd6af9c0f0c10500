"""The DTS gate's backward asks for what its own plan uses: dz and one partial table to a chunk of tokens.  A buffer of that size is enough,
whatever the other backward passes that share evomoe_workspace_bytes need."""
import ctypes

import pytest
import torch

from paper_2112_14397_amd import binding as B

CASES = [(36486, 380, 22), (18220, 448, 49), (777, 68, 5)]


def dts_bytes(T, d, E):
    """float32 layer: chunks of 32 tokens, more where there would be over 256 of them, within 60 KB of dz."""
    tc = 32
    while -(-T // tc) > 256:
        tc *= 2
    while tc * (-(-E // 16) * 16) * 4 > 60 * 1024 and tc > 16:
        tc //= 2
    return 4 * (T * E + -(-T // tc) * (d + 1) * E)


@pytest.mark.parametrize("T,d,E", CASES)
def test_less_is_refused(T, d, E):
    """On the host, before anything is launched: the addresses are never read."""
    ctx, A, s = ctypes.create_string_buffer(4096), 1 << 20, B.make_shape(T, d, E, 4, "f32", "relu", T)
    n = dts_bytes(T, d, E) - 4
    assert B.lib().evomoe_dts_gate_bwd(ctx, ctypes.byref(s), A, A, A, A, A, 1.0, A, A, A, A, A, A, n) == B.EVOMOE_EWORKSPACE
    assert B.lib().evomoe_dts_gate_bwd_balance(ctx, ctypes.byref(s), A, A, A, A, A, 1.0, A, A, A, 1.0, A, A, A, A, n) == B.EVOMOE_EWORKSPACE
    assert dts_bytes(T, d, E) <= min(B.evomoe_workspace_bytes(s), B.evomoe_workspace_bytes_recompute(s))


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,E", CASES)
def test_that_much_is_enough(T, d, E):
    s = B.make_shape(T, d, E, 4, "f32", "relu", T)
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    x, Wg, gp, dG = new(T, d), new(d, E), new(T, E).softmax(1), new(T)
    expert = torch.randint(0, E, (T,), generator=g, device="cuda")
    bits = torch.ones(T, dtype=torch.int64, device="cuda") << expert
    off, rows = (torch.arange(T + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    ctx, out = B.Context(), []
    for n in (B.evomoe_workspace_bytes(s), dts_bytes(T, d, E)):
        ws = torch.full((n + 4096,), 255, dtype=torch.uint8, device="cuda")
        dWg, dbg, dx = torch.empty(d, E, device="cuda"), torch.empty(E, device="cuda"), torch.zeros(T, d, device="cuda")
        B.evomoe_dts_gate_bwd(ctx, s, dG, off, rows, gp, bits, 0.7, x, Wg, dWg, dbg, dx, ws[:n])
        coef = new(E).zero_()
        B.evomoe_dts_gate_bwd_balance(ctx, s, dG, off, rows, gp, bits, 0.7, x, Wg, coef, 1.0, dWg, dbg, dx, ws[:n])
        torch.cuda.synchronize()
        assert (ws[n:] == 255).all()
        out.append((dWg, dbg, dx))
    ctx.close()
    for a, b in zip(*out):
        assert torch.equal(a, b) and torch.isfinite(a).all()

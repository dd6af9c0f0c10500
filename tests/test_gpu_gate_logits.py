"""evomoe_gate_logits and its backward against the float64 oracle."""
import numpy as np
import pytest
import torch

import synth_inputs as synth
from oracle import block_oracle as blk
from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CASES = [("bf16", 1, 64, 1), ("bf16", 5, 8, 64), ("bf16", 48, 768, 16), ("bf16", 256, 256, 16), ("bf16", 257, 136, 7),
         ("bf16", 4500, 72, 33), ("bf16", 9000, 264, 48), ("f32", 1, 4, 1), ("f32", 17, 68, 5), ("f32", 256, 256, 17),
         ("f32", 300, 1028, 64), ("f32", 5000, 100, 20), ("f32", 16500, 64, 40), ("f32", 4200, 516, 33),
         ("f32", 700, 132, 64), ("f32", 33, 256, 63), ("bf16", 33, 64, 49)]


@pytest.mark.parametrize("dtype,T,d,E", CASES)
@pytest.mark.parametrize("more", [False, True])
def test_against_the_oracle(dtype, T, d, E, more):
    """more: with a bias, and dx added to what flows into x besides."""
    rng = np.random.default_rng(T + d + E)
    x, dx_in = (synth.round_to_storage(rng.standard_normal((T, d)), dtype) for _ in range(2))
    Wg = (0.02 * rng.standard_normal((d, E))).astype(np.float32)
    bg, dz = rng.standard_normal(E).astype(np.float32), rng.standard_normal((T, E)).astype(np.float32)
    bg, dx_in = (bg, dx_in) if more else (None, None)
    dt = B.torch_dtype(dtype)
    dev = lambda a, t=torch.float32: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(t)
    shape = B.make_shape(T, d, E, d, dtype, "gelu", 1)
    ctx = B.Context()
    xd, Wd, zd, ind = dev(x, dt), dev(Wg), dev(dz), dev(dx_in, dt)
    new = lambda *s, dtype=torch.float32: torch.full(s, 7.0, dtype=dtype, device="cuda")
    z = new(T, E)
    B.evomoe_gate_logits(ctx, shape, xd, Wd, dev(bg), z)
    want, mag = blk.logits(x, Wg, bg)
    # products of 24-bit factors exact or rounded once, sums of up to d of them in any order: d / 16 + 20 roundings at most, as the
    # k's are dealt to four lane groups of four waves
    assert (abs(z.cpu().numpy() - want) <= U * (d / 16 + 20) * mag).all()
    ws = torch.empty(B.evomoe_workspace_bytes(shape), dtype=torch.uint8, device="cuda").fill_(255)
    dWg, dbg, dx = new(d, E), new(E), new(T, d, dtype=dt)
    B.evomoe_gate_logits_bwd(ctx, shape, zd, xd, Wd, ind, dWg, dbg, dx, ws)
    (w_W, w_b, w_x), (m_W, m_b, m_x) = blk.logits_bwd(dz, x, Wg, dx_in)
    assert (abs(dWg.cpu().numpy() - w_W) <= U * (T + 20) * m_W).all()
    assert (abs(dbg.cpu().numpy() - w_b) <= U * (T + 20) * m_b).all()
    # a bf16 layer's dx: W_g to 16 bits and dz to 16 (2^-16 of the magnitudes each at most), and the result's half step
    far = U * (E + 8) * m_x if dtype == "f32" else 2.0 ** -15 * m_x + 2.0 ** -8 * abs(w_x)
    assert (abs(dx.double().cpu().numpy() - w_x) <= far).all()
    # again; over dx_in; without dbg: the same
    first = [t.clone() for t in (dWg, dbg, dx)]
    over = None if ind is None else ind.clone()
    B.evomoe_gate_logits_bwd(ctx, shape, zd, xd, Wd, over, dWg.fill_(7), None, over if more else dx.fill_(7), ws)
    assert torch.equal(dWg, first[0]) and torch.equal(over if more else dx, first[2])
    z2 = new(T, E)
    B.evomoe_gate_logits(ctx, shape, xd, Wd, dev(bg), z2)
    assert torch.equal(z, z2)
    ctx.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_dts_gate_s_softmax_follows_from_the_logits(dtype):
    rng = np.random.default_rng(2)
    T, d, E = 600, 136, 12
    dt = B.torch_dtype(dtype)
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(dt)
    Wg, bg = (torch.from_numpy((0.1 * rng.standard_normal(s)).astype(np.float32)).cuda() for s in ((d, E), (E,)))
    shape, ctx = B.make_shape(T, d, E, 64, dtype, "gelu", T * E), B.Context()
    z, gp = torch.empty(T, E, device="cuda"), torch.empty(T, E, device="cuda")
    mask, counts = torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    B.evomoe_gate_logits(ctx, shape, x, Wg, bg, z)
    B.evomoe_dts_gate(ctx, shape, x, Wg, bg, None, 0.5, 0.1, gp, None, mask, counts, None)
    # the same products and sums; / tau is exact, the softmax rounds as in the top-k gate's test (spread below 16)
    assert (gp.double() - torch.softmax(z.double() / 0.5, 1)).abs().max().item() <= U * 32
    ctx.close()


def test_a_captured_pass_outlives_a_larger_one():
    """The split copy of W_g grows with d; a graph that was captured before goes on with the smaller one."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.Generator(device="cuda").manual_seed(3)
        ctx, new = B.Context(), lambda *s: torch.randn(*s, generator=g, device="cuda")
        T, d, E = 5000, 64, 16
        shape, x, W, z = B.make_shape(T, d, E, d, "bf16", "gelu", 1), new(T, d).bfloat16(), new(d, E), new(T, E)
        B.evomoe_gate_logits(ctx, shape, x, W, None, z)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.evomoe_gate_logits(ctx, shape, x, W, None, z)
        wide = 8192
        x2, W2, z2 = new(T, wide).bfloat16(), new(wide, E), new(T, E)
        B.evomoe_gate_logits(ctx, B.make_shape(T, wide, E, wide, "bf16", "gelu", 1), x2, W2, None, z2)
        mine = B.Context()
        for i in range(3):
            x.copy_(new(T, d))
            W.copy_(new(d, E))
            graph.replay()
            torch.randn(2048, 2048, device="cuda").sum()
            want = torch.empty_like(z)
            B.evomoe_gate_logits(mine, shape, x, W, None, want)
            torch.cuda.synchronize()
            assert torch.equal(z, want)
        torch.cuda.synchronize()
        ctx.close()
        mine.close()


def test_few_tokens_captured_before_any_other_call():
    """Up to 4096 tokens nothing is allocated, so that the first call of a context may be a captured one."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        g = torch.Generator(device="cuda").manual_seed(4)
        new = lambda *s: torch.randn(*s, generator=g, device="cuda")
        T, d, E = 48, 4096, 16
        shape, x, W, z = B.make_shape(T, d, E, d, "bf16", "gelu", 1), new(T, d).bfloat16(), new(d, E), new(T, E)
        other, want = B.Context(), torch.empty(T, E, device="cuda")
        B.evomoe_gate_logits(other, shape, x, W, None, want)
        ctx = B.Context()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.evomoe_gate_logits(ctx, shape, x, W, None, z)
        for _ in range(3):
            z.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(z, want)
        ctx.close()
        other.close()

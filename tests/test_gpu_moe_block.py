"""The operators of a pre-norm MoE block as they are used, one behind the other: residual + norm, gate logits, top-k gate, dispatch, experts,
combine, and back; and the serving form with the experts in 8 bits.  Against the oracle, and captured into graphs."""
import numpy as np
import pytest
import torch

import gpu_harness as H
import synth_inputs as synth
from helpers import tol_ok
from oracle import block_oracle as blk
from oracle import evomoe_oracle as orc
from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-6


class Block:
    """Buffers of one block, and its two passes as a program would write them."""

    def __init__(self, T, d, E, F, dtype, act, o: blk.TopK, seed, mx8=False, stream=None):
        rng = np.random.default_rng(seed)
        draw = lambda *s, std=1.0: (std * rng.standard_normal(s)).astype(np.float32)
        st = lambda a: synth.round_to_storage(a, dtype)
        self.o, self.act = o, act
        self.np = dict(x=st(draw(T, d)), res=st(draw(T, d)), gamma=1 + draw(d, std=0.1), Wg=draw(d, E, std=0.05), bg=draw(E, std=0.1),
                       W1=st(draw(E, F, d, std=0.05)), b1=draw(E, F, std=0.1), W2=st(draw(E, d, F, std=0.05)), b2=draw(E, d, std=0.1),
                       bias=draw(E, std=0.02), dout=st(draw(T, d)))
        stored = ("x", "res", "W1", "W2", "dout")
        t = {n: H.to_dev(a, B.torch_dtype(dtype) if n in stored else None) for n, a in self.np.items()}
        self.t = t
        self.ctx = B.Context(stream)
        self.shape = B.make_shape(T, d, E, F, dtype, act, T * o.k)
        self.topk = B.make_topk(o.k, o.score, o.groups, o.top_groups, o.group_keys, o.renormalise, o.scale)
        self.p = B.LayerParams(Wg=t["Wg"], bg=t["bg"], W1=t["W1"], b1=t["b1"], W2=t["W2"], b2=t["b2"])
        self.b = B.LayerBuffers(self.shape, backward=not mx8, mx8=mx8)
        self.h, self.y, self.rstd = torch.zeros_like(t["x"]), torch.zeros_like(t["x"]), torch.zeros(T, device="cuda")
        self.dx, self.dgamma = torch.zeros_like(t["x"]), torch.zeros(d, device="cuda")
        if mx8:
            self.experts = B.Mx8Experts(self.ctx, self.p)
            self.q, self.qs = B.mx8_empty((T, d))

    def step(self):
        t = self.t
        B.evomoe_add_rmsnorm(self.ctx, self.shape, t["x"], t["res"], t["gamma"], EPS, self.h, self.y, self.rstd)
        B.topk_layer_forward(self.ctx, self.b, self.p, self.topk, self.y, t["bias"])
        B.topk_layer_backward(self.ctx, self.b, self.p, self.topk, self.y, t["dout"], balance_alpha=0.1)
        # the block's output is h + layer(y): dout flows into h as well
        B.evomoe_add_rmsnorm_bwd(self.ctx, self.shape, self.b.dx, t["dout"], self.h, t["gamma"], self.rstd, self.dx, self.dgamma,
                                 self.b.workspace)

    def serve(self):
        t = self.t
        B.evomoe_add_rmsnorm(self.ctx, self.shape, t["x"], t["res"], t["gamma"], EPS, self.h, self.y, None, self.q, self.qs)
        B.topk_layer_forward_mx8(self.ctx, self.b, self.p, self.topk, self.experts, self.y, self.q, self.qs, t["bias"])

    def outputs(self):
        b = self.b
        names = ("y", "dx", "dWg", "dbg", "dW1", "db1", "dW2", "db2", "bal_loss", "gate_w", "mask_bits", "counts")
        out = {n: getattr(b, n) for n in names if hasattr(b, n)}
        return {n: v.clone() for n, v in {**out, "h": self.h, "norm": self.y, "block_dx": self.dx, "dgamma": self.dgamma}.items()}


OPTIONS = [blk.TopK(2), blk.TopK(3, "sigmoid", 4, 2, 2, True, 2.5), blk.TopK(1, "sigmoid", renormalise=False)]


@pytest.mark.parametrize("dtype,rt", [("f32", 3e-5), ("bf16", 2e-2)])
@pytest.mark.parametrize("o", OPTIONS)
def test_training_step_against_the_oracle(dtype, rt, o):
    """rt: what the layer's own comparison allows a type, in float32 three times that, for the norm before and the longer chain behind."""
    T, d, E, F = 190, 64, 8, 128
    k = Block(T, d, E, F, dtype, "gelu", o, seed=21)
    k.step()
    P = B.evomoe_num_pairs(k.ctx, k.b.num_pairs)
    n = k.np
    close = lambda name, got, want: (lambda r: r[0] or pytest.fail(f"{name}: {r[1]:.3g} times the bound"))(
        tol_ok(H.np_of(got), want, rt))
    h = synth.round_to_storage(n["x"] + n["res"], dtype)
    close("norm", k.y, blk.rmsnorm(h, n["gamma"], EPS)[0])
    y = H.np_of(k.y)                                                     # what the gate and the experts read, as it is stored
    z, _ = blk.logits(y, n["Wg"], n["bg"])
    mask = blk.topk_select(z, n["bias"], o)
    assert np.array_equal(H.mask_from_bits(H.np_of(k.b.mask_bits), E), mask)
    w = blk.topk_weights(z, mask, o)
    dp = orc.dispatch(mask, w)
    assert P == int(dp.expert_offsets[E])
    ffn = orc.expert_ffn(y, dp.pair_token, dp.expert_offsets, n["W1"], n["b1"], n["W2"], n["b2"], "gelu")
    close("y", k.b.y, orc.combine(ffn.O, dp.pair_gate, dp.tok_off, dp.tok_rows, T))
    dO, dG = orc.combine_bwd(n["dout"], ffn.O, dp.pair_gate, dp.pair_token)
    g = orc.expert_ffn_bwd(dO, ffn.H, y, dp.pair_token, dp.expert_offsets, n["W1"], n["W2"], "gelu")
    for name in ("dW1", "db1", "dW2", "db2"):
        close(name, getattr(k.b, name), getattr(g, name))
    dense = np.zeros((T, E))
    dense[dp.pair_token, dp.pair_expert] = dG
    coef = 0.1 * E * mask.sum(0) / T ** 2
    s = blk.scores(z, o.score)
    close("loss", k.b.bal_loss, np.array([(coef * s.sum(0)).sum()]))
    dz, _ = blk.topk_bwd(z, mask, dense, o, coef)
    (dWg, dbg, dyl), _ = blk.logits_bwd(dz, y, n["Wg"], orc.dispatch_bwd(g.dXp, dp.tok_off, dp.tok_rows, T))
    close("dWg", k.b.dWg, dWg)
    close("dbg", k.b.dbg, dbg)
    close("dx of the layer", k.b.dx, dyl)
    (dx, dgamma), _ = blk.rmsnorm_bwd(H.np_of(k.b.dx), n["dout"], h, n["gamma"], EPS)
    close("dx", k.dx, dx)
    close("dgamma", k.dgamma, dgamma)


def test_serving_against_the_oracle():
    T, d, E, F, o = 75, 96, 8, 160, blk.TopK(3, "sigmoid", 4, 2, 2, True, 2.5)
    k = Block(T, d, E, F, "bf16", "gelu", o, seed=22, mx8=True)
    k.serve()
    B.evomoe_num_pairs(k.ctx, k.b.num_pairs)
    n, y = k.np, H.np_of(k.y)
    z, _ = blk.logits(y, n["Wg"], n["bg"])
    mask = blk.topk_select(z, n["bias"], o)
    assert np.array_equal(H.mask_from_bits(H.np_of(k.b.mask_bits), E), mask)
    dp = orc.dispatch(mask, blk.topk_weights(z, mask, o))
    val = lambda q, s: blk.mx8_value(q.double().cpu().numpy(), s.double().cpu().numpy())
    W1, W2 = val(k.experts.W1, k.experts.W1_scale), val(k.experts.W2, k.experts.W2_scale)
    for got, of in ((W1, n["W1"]), (W2, n["W2"])):
        assert np.array_equal(got, blk.mx8_value(*blk.mx8(of)))
    u = 2.0 ** -24
    O, far = blk.experts_mx8(val(k.q, k.qs), dp.pair_token, dp.expert_offsets, W1, n["b1"], W2, n["b2"], "gelu", 2 * u * max(d, F), 1.4e-5)
    far += 2.0 ** -8 * abs(O)
    # the sum over a token's experts: each O within its bound, the weights within 32 roundings, the result half a bf16 step
    want, bound = (orc.combine(a, dp.pair_gate, dp.tok_off, dp.tok_rows, T) for a in (O, far))
    size = orc.combine(abs(O), dp.pair_gate, dp.tok_off, dp.tok_rows, T)
    assert (abs(H.np_of(k.b.y) - want) <= bound + 40 * u * size + 2.0 ** -8 * abs(want)).all()


def test_padding_tokens_select_nothing_and_give_nothing():
    """Logits of -inf: such tokens have no pairs, an output of 0 and no gradient, and the others are as without them."""
    T, E, d, F, o = 300, 8, 64, 64, blk.TopK(2)
    rng = np.random.default_rng(5)
    k = Block(T, d, E, F, "bf16", "gelu", o, seed=23)
    t, b, s = k.t, k.b, k.shape
    pad = torch.from_numpy(rng.random(T) < 0.3).cuda()
    B.evomoe_gate_logits(k.ctx, s, t["x"], t["Wg"], t["bg"], b.logits)

    def rest():
        B.evomoe_topk_gate(k.ctx, s, k.topk, b.logits, None, b.gprime, b.gate_w, b.mask_bits, b.counts, b.k, b.block_hist)
        B.evomoe_dispatch(k.ctx, s, b.mask_bits, b.gate_w, b.expert_offsets, b.pair_token, b.pair_gate, b.tok_off, b.tok_rows,
                          b.num_pairs, block_hist=b.block_hist)
        B.evomoe_expert_ffn(k.ctx, s, t["x"], b.pair_token, b.expert_offsets, t["W1"], t["b1"], t["W2"], t["b2"], b.H, b.A, b.O)
        B.evomoe_combine(k.ctx, s, b.O, b.pair_gate, b.tok_off, b.tok_rows, b.y)
        B.topk_layer_backward(k.ctx, b, k.p, k.topk, t["x"], t["dout"])
        return {n: getattr(b, n).clone() for n in ("y", "dlogits", "gate_w", "k", "dx")}

    full = rest()
    b.logits[pad] = -float("inf")
    some = rest()
    assert B.evomoe_num_pairs(k.ctx, b.num_pairs) == 2 * int((~pad).sum())
    for n in full:
        assert torch.equal(some[n][~pad], full[n][~pad]), n
        assert (some[n][pad] == 0).all(), n


@pytest.mark.parametrize("mx8", [False, True])
def test_captured_and_replayed(mx8):
    """A step captured once and replayed on new inputs gives the bits of the eager calls, with other work between the replays; two blocks
    with contexts of their own on two streams at once give theirs."""
    stream = torch.cuda.Stream()
    sizes = (1000, 128, 16, 256, "bf16", "gelu", blk.TopK(4, "sigmoid", 4, 2, 2))
    with torch.cuda.stream(stream):
        k = Block(*sizes, seed=31, mx8=mx8, stream=stream)
        eager = Block(*sizes, seed=31, mx8=mx8, stream=stream)
        pass_of = lambda x: x.serve() if mx8 else x.step()
        pass_of(k)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            pass_of(k)
        for i in range(4):
            g = torch.Generator(device="cuda").manual_seed(i)
            for n in ("x", "res", "bias"):
                new = torch.randn(k.t[n].shape, generator=g, device="cuda") * (0.02 if n == "bias" else 1)
                k.t[n].copy_(new)
                eager.t[n].copy_(new)
            graph.replay()
            torch.randn(4096, 4096, device="cuda").sum()
            pass_of(eager)
            torch.cuda.synchronize()
            want, got = eager.outputs(), k.outputs()
            for n in want:
                assert torch.equal(got[n], want[n]), (i, n)
    two = [torch.cuda.Stream(), torch.cuda.Stream()]
    pair = [Block(*sizes, seed=31 + i, mx8=mx8, stream=s) for i, s in enumerate(two)]
    alone = []
    for x in pair:
        pass_of(x)
        torch.cuda.synchronize()
        alone.append(x.outputs())
    for _ in range(5):
        for x in pair:
            pass_of(x)
    torch.cuda.synchronize()
    for x, want in zip(pair, alone):
        got = x.outputs()
        for n in want:
            assert torch.equal(got[n], want[n]), n

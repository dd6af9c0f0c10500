"""evomoe_topk_gate and its backward against the float64 oracle: selections exactly, weights and gradients to the rounding of float32
arithmetic, over the options, odd numbers of experts, ties, masked experts and tokens, NaNs, and scores below float32's range."""
import itertools

import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from oracle import evomoe_oracle as orc
from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                   # half a step of float32


def gpu_topk(o: blk.TopK):
    return B.make_topk(o.k, o.score, o.groups, o.top_groups, o.group_keys, o.renormalise, o.scale)


def bits_of(mask):
    return (mask.astype(np.uint64) << np.arange(mask.shape[1], dtype=np.uint64)).sum(1, dtype=np.uint64)


def run(ctx, o, z, bias, dG=None, coef=None, P_cap=None):
    """Every output of the gate, of dispatch behind it and of its backward, as numpy."""
    T, E = z.shape
    shape = B.make_shape(T, 64, E, 64, "f32", "relu", P_cap or T * o.k)
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    new = lambda *s, dtype=torch.float32: torch.full(s, -7, dtype=dtype, device="cuda")
    i32 = torch.int32
    out = dict(scores=new(T, E), gate_w=new(T, E), mask=new(T, dtype=torch.int64), counts=new(E, dtype=i32),
               k=new(T, dtype=i32), hist=new((T + 255) // 256, E, dtype=i32))
    logits = dev(z)
    B.evomoe_topk_gate(ctx, shape, gpu_topk(o), logits, dev(bias), out["scores"], out["gate_w"], out["mask"], out["counts"],
                       out["k"], out["hist"])
    if dG is not None:
        P = shape.P_cap
        offs, ptok, trows, toff = new(E + 1, dtype=i32), new(P, dtype=i32), new(P, dtype=i32), new(T + 1, dtype=i32)
        pgate, num = new(P), new(1, dtype=torch.int64)
        B.evomoe_dispatch(ctx, shape, out["mask"], out["gate_w"], offs, ptok, pgate, toff, trows, num, block_hist=out["hist"])
        out["dlogits"] = new(T, E)
        B.evomoe_topk_gate_bwd(ctx, shape, gpu_topk(o), dev(dG), toff, trows, logits, out["mask"], dev(coef), 0.5, out["dlogits"])
        out["pair_gate"], out["num_pairs"] = pgate, num
    torch.cuda.synchronize()
    return {n: v.cpu().numpy() for n, v in out.items()}


def check(ctx, o, z, bias=None, coef=None, seed=0):
    T, E = z.shape
    z = z.astype(np.float32)
    mask = blk.topk_select(z, bias, o)
    dG_dense = np.random.default_rng(seed).standard_normal((T, E)).astype(np.float32)
    dp = orc.dispatch(mask, mask * 1.0)
    P = int(dp.expert_offsets[E])
    dG = np.zeros(T * o.k, np.float32)
    dG[:P] = dG_dense[dp.pair_token, dp.pair_expert]
    got = run(ctx, o, z, bias, dG, coef)
    np.testing.assert_array_equal(got["mask"].view(np.uint64), bits_of(mask))
    np.testing.assert_array_equal(got["counts"], mask.sum(0))
    np.testing.assert_array_equal(got["k"], mask.sum(1))
    for r in range(got["hist"].shape[0]):
        np.testing.assert_array_equal(got["hist"][r], mask[256 * r:256 * (r + 1)].sum(0))
    assert int(got["num_pairs"][0]) == P
    np.testing.assert_array_equal(got["pair_gate"][:P], got["gate_w"][dp.pair_token, dp.pair_expert])
    np.testing.assert_array_equal(got["gate_w"][~mask], 0)
    # Rounding.  An exponential's argument z_i - z_max is rounded once (U of it), the exponential, the sum over up to 64 terms in
    # a tree, the quotient and the product with `scale` take 16 U more; below 2^-126 a step is 2^-149.
    finite = np.where(np.isfinite(z), z, 0).astype(np.float64)
    spread = 16 + abs(finite - finite.max(1, keepdims=True))
    with np.errstate(all="ignore"):
        s = blk.scores(z, o.score)
        for name, want in (("scores", s), ("gate_w", blk.topk_weights(z, mask, o))):
            bad = ~(abs(got[name] - want) <= U * spread * abs(want) + 1e-44) & ~(np.isnan(want) & np.isnan(got[name]))
            assert not bad.any(), (name, got[name][bad][:4], want[bad][:4])
        # of a gradient each factor and each sum is off by as much: 4 such terms
        want, mag = blk.topk_bwd(z, mask, dG_dense, o, None if coef is None else 0.5 * coef)
        far = 4 * U * (spread.max(1, keepdims=True)) * mag + 1e-43
        bad = ~(abs(got["dlogits"] - want) <= far) & ~(np.isnan(want) & np.isnan(got["dlogits"]))
        assert not bad.any(), ("dlogits", got["dlogits"][bad][:4], want[bad][:4], far[bad][:4])


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


CASES = [(1, 64), (5, 4), (255, 3), (256, 16), (257, 1), (700, 7), (130, 33), (64, 48), (1025, 8), (300, 62)]


@pytest.mark.parametrize("T,E", CASES)
@pytest.mark.parametrize("score,renormalise,with_bias", itertools.product(("softmax", "sigmoid"), (True, False), (True, False)))
def test_against_the_oracle(ctx, T, E, score, renormalise, with_bias):
    rng = np.random.default_rng(T * 100 + E)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) if with_bias else None
    coef = rng.standard_normal(E).astype(np.float32) if renormalise else None
    for k in sorted({1, min(E, 8), E}):
        check(ctx, blk.TopK(k, score, renormalise=renormalise, scale=2.5), rng.standard_normal((T, E)), bias, coef)


@pytest.mark.parametrize("E,groups,top,keys,k", [(64, 8, 4, 2, 8), (62, 2, 1, 1, 5), (60, 20, 3, 2, 9), (64, 64, 7, 2, 7), (10, 5, 5, 1, 10),
                                                 (48, 4, 2, 2, 24), (3, 3, 1, 2, 1)])
@pytest.mark.parametrize("score,with_bias", itertools.product(("softmax", "sigmoid"), (True, False)))
def test_groups(ctx, E, groups, top, keys, k, score, with_bias):
    rng = np.random.default_rng(E + groups)
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) if with_bias else None
    z = rng.standard_normal((321, E))
    z[::7, : E // 2] = -np.inf                            # groups with few experts left, or none
    check(ctx, blk.TopK(k, score, groups, top, keys), z, bias)


@pytest.mark.parametrize("score,groups", [("softmax", 1), ("sigmoid", 1), ("softmax", 4), ("sigmoid", 4)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_ties_masks_and_what_is_not_finite(ctx, score, groups, with_bias):
    inf, nan, low = np.inf, np.nan, float(np.finfo(np.float32).min)
    E = 20
    rng = np.random.default_rng(3)
    rows = [np.zeros(E), np.full(E, -inf), np.full(E, 3.5), np.full(E, low), np.where(np.arange(E) < 2, 1.0, -inf),
            np.where(np.arange(E) == 19, 0.25, -inf), np.where(np.arange(E) % 2, 1.0, low), np.round(rng.standard_normal(E)),
            np.where(np.arange(E) == 7, nan, rng.standard_normal(E)), np.full(E, nan), np.where(np.arange(E) < 10, nan, -inf),
            np.full(E, -200.0) + np.arange(E) % 3, np.full(E, 90.0), -88.0 - np.arange(E), -100.0 - rng.random(E) * 8,
            np.where(np.arange(E) < 12, -inf, -104.0 + np.arange(E) * 0.01)]
    if score == "sigmoid" or not with_bias and groups == 1:
        rows.append(np.where(np.arange(E) == 4, inf, 0.5))
    bias = None
    if with_bias:
        bias = np.round(rng.standard_normal(E) * 4).astype(np.float32) / 8
        bias[3] = -inf
    for o in (blk.TopK(1, score, groups), blk.TopK(5, score, groups, groups, 2), blk.TopK(4, score, groups, groups, 1, False, 0.5)):
        check(ctx, o, np.array(rows), bias)


def test_keys_that_float32_scores_would_not_tell_apart(ctx):
    """Logits one step apart: their float32 sigmoids and softmaxes are often the same number, and the larger logit is selected all the
    same; with a bias that offsets them, the order of the 64-bit keys."""
    E, T = 64, 512
    rng = np.random.default_rng(9)
    base = rng.uniform(1.0, 6.0, (T, 1)).astype(np.float32)
    z = base + np.spacing(base) * rng.permuted(np.tile(np.arange(E), (T, 1)), axis=1).astype(np.float32)
    bias = (np.float32(2.0) ** -24 * rng.integers(-2, 3, E)).astype(np.float32)
    for score in ("softmax", "sigmoid"):
        check(ctx, blk.TopK(8, score), z)
        check(ctx, blk.TopK(8, score), z, bias)
        check(ctx, blk.TopK(8, score, 8, 4, 2), z, bias)


def test_a_token_is_routed_the_same_in_any_batch_and_again(ctx):
    rng = np.random.default_rng(11)
    z, o = rng.standard_normal((3000, 64)).astype(np.float32), blk.TopK(8, "sigmoid", 8, 4, 2)
    bias = (0.05 * rng.standard_normal(64)).astype(np.float32)
    dG = rng.standard_normal(24000)
    all_, again = run(ctx, o, z, bias, dG), run(ctx, o, z, bias, dG)
    for n in all_:
        assert np.array_equal(all_[n], again[n], equal_nan=True), n
    few = run(ctx, o, z[1000:1017], bias)
    for n in ("mask", "gate_w", "scores", "k"):
        assert np.array_equal(few[n], all_[n][1000:1017]), n


def test_optional_outputs_and_rows_that_do_not_fit(ctx):
    """Without scores, k and the histogram the rest is the same; with a P_cap that the pairs exceed the backward stays in bounds and
    the tokens whose pairs all fit keep their gradients."""
    rng = np.random.default_rng(12)
    T, E, o = 600, 16, blk.TopK(2)
    z = rng.standard_normal((T, E)).astype(np.float32)
    full = run(ctx, o, z, None)
    shape = B.make_shape(T, 64, E, 64, "f32", "relu", 1)
    gw, mask, counts = torch.empty(T, E, device="cuda"), torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    B.evomoe_topk_gate(ctx, shape, gpu_topk(o), torch.from_numpy(z).cuda(), None, None, gw, mask, counts)
    assert np.array_equal(gw.cpu().numpy(), full["gate_w"]) and np.array_equal(mask.cpu().numpy(), full["mask"])
    assert np.array_equal(counts.cpu().numpy(), full["counts"])
    with pytest.raises(AssertionError):
        B.evomoe_topk_gate(ctx, shape, gpu_topk(o), torch.from_numpy(z).cuda().t(), None, None, gw, mask, counts)
    got = run(ctx, o, z, None, rng.standard_normal(900), P_cap=900)
    assert np.isfinite(got["dlogits"]).all()
    with pytest.raises(B.EvoMoEError) as e:                # the capacity flag is reported, and cleared
        B.evomoe_num_pairs(ctx, torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert e.value.status == B.EVOMOE_ECAPACITY


@pytest.mark.parametrize("T,E", [(257, 64), (2000, 40), (40000, 33)])
def test_counts_without_the_histogram(ctx, T, E):
    rng = np.random.default_rng(T)
    z, o = rng.standard_normal((T, E)).astype(np.float32), blk.TopK(5, "sigmoid")
    gw, mask, counts = torch.empty(T, E, device="cuda"), torch.empty(T, dtype=torch.int64, device="cuda"), torch.full((E,), 7, dtype=torch.int32, device="cuda")
    for _ in range(2):
        B.evomoe_topk_gate(ctx, B.make_shape(T, 64, E, 64, "f32", "relu", 1), gpu_topk(o), torch.from_numpy(z).cuda(), None, None, gw, mask, counts)
        want = blk.topk_select(z, None, o)
        assert np.array_equal(mask.cpu().numpy().view(np.uint64), bits_of(want))
        assert np.array_equal(counts.cpu().numpy(), want.sum(0))

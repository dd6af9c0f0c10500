"""evomoe_expert_ffn_mx8 against the float64 oracle on the same 8-bit values, each element within a bound of its own."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from paper_2112_14397_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# of the activation: erf's and the polynomials' errors are below 1.4e-5 max(|h|, 4.2) (the f32 one's far below)
ACT = 1.4e-5


def inputs(rng, T, d, E, F, P, skew=1.0):
    """x, weights and biases in 8 bits, values as float64; rows of experts of uneven sizes, some without any."""
    values = {}
    for n, shape, std in (("x", (T, d), 1.0), ("W1", (E, F, d), 0.05), ("W2", (E, d, F), 0.05)):
        q, s = blk.mx8(std * rng.standard_normal(shape).astype(np.float32))
        values[n] = (q, s)
    share = rng.random(E) ** 3 * skew
    share[rng.random(E) < 0.2] = 0
    share = share if share.sum() else np.ones(E)
    expert = np.sort(rng.choice(E, P, p=share / share.sum()))
    offsets = np.searchsorted(expert, np.arange(E + 1)).astype(np.int32)
    token = rng.integers(0, T, P).astype(np.int32)
    b1, b2 = (0.1 * rng.standard_normal((E, n)).astype(np.float32) for n in (F, d))
    return values, offsets, token, b1, b2


def to_gpu(q, s):
    """8-bit values that the oracle has made (both types hold them exactly)."""
    return (torch.from_numpy(q.astype(np.float32)).cuda().to(torch.float8_e4m3fn),
            torch.from_numpy((np.log2(s) + 127).astype(np.uint8)).cuda().view(torch.float8_e8m0fnu))


def run(ctx, values, offsets, token, b1, b2, act, P_cap, T, gather=True):
    W1, W2 = values["W1"][0], values["W2"][0]
    E, F, d = W1.shape
    shape = B.make_shape(T, d, E, F, "bf16", act, P_cap)
    (x, xs), (w1, s1), (w2, s2) = (to_gpu(*values[n]) for n in ("x", "W1", "W2"))
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    tok = torch.zeros(P_cap, dtype=torch.int32, device="cuda")
    tok[: min(len(token), P_cap)] = dev(token[:P_cap])
    O = torch.full((P_cap, d), 7.0, dtype=torch.bfloat16, device="cuda")
    n = B.evomoe_workspace_bytes_mx8(shape)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")            # NaNs, and a guard behind it
    B.evomoe_expert_ffn_mx8(ctx, shape, x, xs, tok if gather else None, dev(offsets), w1, s1, dev(b1), w2, s2, dev(b2), O, ws[:n])
    torch.cuda.synchronize()
    assert (ws[n:] == 255).all()
    return O


def some_rows(offsets, rng):
    """Rows that are compared where comparing all takes too long: the first and last ones of every expert, those around multiples of
    the tiles' 32 to 256 rows, and others."""
    rows = set(rng.integers(0, int(offsets[-1]), 60).tolist())
    for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist()):
        for r in (a, a + 1, a + 31, a + 32, a + 63, a + 64, a + 127, a + 128, a + 255, a + 256, b - 129, b - 2, b - 1):
            if a <= r < b:
                rows.add(r)
    return np.array(sorted(rows))


def check(ctx, T, d, E, F, P, act, seed=0, biases=True, gather=True, room=0, hint=0, some=False):
    rng = np.random.default_rng(seed + T + d + E + F)
    values, offsets, token, b1, b2 = inputs(rng, T if gather else P, d, E, F, P)
    if not biases:
        b1 = b2 = None
    if hint:
        B.evomoe_hint_pairs(ctx, hint)
    O = run(ctx, values, offsets, token, b1, b2, act, P + room, T, gather)
    again = run(ctx, values, offsets, token, b1, b2, act, P + room, T, gather)
    B.evomoe_hint_pairs(ctx, 0)
    assert torch.equal(O, again)
    assert (O[P:] == 7).all()                                     # rows behind the last pair are left as they were
    x, W1, W2 = (blk.mx8_value(*values[n]) for n in ("x", "W1", "W2"))
    rows = some_rows(offsets, rng) if some else np.arange(P)
    if not gather:
        token = np.arange(P)
    # sums over max(d, F) products of 8-bit values and scales, which are exact: one rounding each (two steps of slack for the
    # matrix instruction, which may cut off instead of rounding)
    want, bound = blk.experts_mx8(x, token[rows], np.searchsorted(rows, offsets), W1, b1, W2, b2, act, 2 * U * max(d, F), ACT)
    got = O[:P].double().cpu().numpy()[rows]
    bad = ~(abs(got - want) <= bound + 2.0 ** -8 * abs(want))
    assert not bad.any(), (int(bad.sum()), got[bad][:4], want[bad][:4], bound[bad][:4])


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


# T, d, E, F, pairs, and the tiles of both products
CASES = [(1, 32, 1, 32, 1, "32x32/4", "32x32/4"), (5, 64, 3, 96, 9, "32x32/4", "32x32/4"), (48, 768, 16, 1024, 8, "32x32/4", "32x32/4"), (48, 768, 16, 1024, 16, "32x32/4", "64x64/4"),
         (70, 160, 7, 288, 200, "32x32/4", "32x32/4"), (40, 1056, 5, 64, 90, "32x32/4", "32x32/4"),
         (33, 512, 33, 544, 33, "32x32/4", "32x32/4"), (300, 1184, 2, 32, 400, "32x32/4", "32x32/4"),
         (48, 768, 16, 1024, 48, "32x32/4", "64x64/4"), (300, 256, 4, 512, 700, "32x32/4", "64x64/4"),
         (90, 128, 64, 128, 400, "32x32/4", "64x64/4"), (60, 384, 5, 640, 77, "32x32/4", "64x64/4"),
         (600, 128, 2, 256, 1500, "32x32/4", "64x64/4"), (500, 640, 3, 384, 1100, "32x32/4", "64x128/4"),
         (100, 512, 1, 1152, 333, "32x32/4", "64x64/4"), (400, 768, 16, 256, 4000, "64x128/4", "128x128/4"),
         (500, 1024, 8, 640, 3000, "128x128/4", "128x128/4"), (30, 256, 33, 896, 500, "32x32/4", "64x64/4"),
         (300, 512, 4, 1152, 700, "64x128/4", "64x64/4"), (64, 256, 16, 2816, 300, "64x128/4", "64x64/4"),
         (700, 640, 2, 1280, 1100, "128x128/4", "64x128/4"), (700, 384, 2, 1280, 1300, "128x128/4", "64x128/4"),
         (500, 160, 3, 1120, 4000, "128x128/4", "32x32/4"), (300, 1120, 3, 96, 4000, "32x32/4", "128x128/4"),
         (300, 1056, 5, 1184, 3000, "128x128/4", "128x128/4"), (200, 32, 2, 2080, 3000, "128x128/4", "32x32/4")]
# ... where the oracle looks at some rows
LARGE = [(500, 128, 2, 4352, 8100, "256x256/8", "64x128/4"), (400, 384, 1, 8832, 4000, "256x256/8", "64x128/4"),
         (700, 1024, 3, 128, 8200, "128x128/4", "256x256/4"), (300, 4480, 2, 256, 2600, "128x128/4", "256x256/4"),
         (900, 1152, 5, 4736, 9000, "256x256/8", "256x256/4"), (300, 768, 16, 384, 5998, "128x128/4", "192x128/4"),
         (200, 1024, 8, 1408, 4000, "128x128/4", "192x128/4"), (300, 640, 10, 640, 6000, "128x128/4", "192x128/4")]


@pytest.mark.parametrize("T,d,E,F,P,first,second", CASES)
@pytest.mark.parametrize("act", ["gelu", "relu"])
def test_against_the_oracle(ctx, T, d, E, F, P, first, second, act):
    check(ctx, T, d, E, F, P, act, biases=act == "gelu", room=37, hint=P)


@pytest.mark.parametrize("T,d,E,F,P,first,second", LARGE)
def test_large_tiles(ctx, T, d, E, F, P, first, second):
    check(ctx, T, d, E, F, P, "gelu", room=300, hint=P, some=True)
    if d == 128:
        check(ctx, T, d, E, F, P, "relu", biases=False, some=True)


def test_a_hint_that_is_wrong(ctx):
    """An announced pair count picks the tiles and nothing else: far too few, far too many."""
    check(ctx, 300, 256, 4, 512, 700, "gelu", hint=1)
    check(ctx, 60, 256, 4, 512, 31, "gelu", room=40000, hint=40000)


def test_rows_that_are_permuted_already(ctx):
    check(ctx, 50, 128, 4, 160, 130, "gelu", gather=False, room=3)


def test_no_pairs_at_all(ctx):
    check(ctx, 5, 64, 3, 96, 0, "gelu", room=8)


def test_more_pairs_than_the_buffers_hold(ctx):
    """Offsets beyond P_cap: only rows below it are computed, as if there were no others."""
    rng = np.random.default_rng(8)
    values, offsets, token, b1, b2 = inputs(rng, 40, 64, 4, 96, 120)
    full = run(ctx, values, offsets, token, b1, b2, "gelu", 120, 40)
    part = run(ctx, values, offsets, token, b1, b2, "gelu", 75, 40)
    assert torch.equal(part, full[:75])


def test_nan_of_one_row_and_one_weight_stay_where_they_belong(ctx):
    rng = np.random.default_rng(4)
    values, offsets, token, b1, b2 = inputs(rng, 30, 96, 3, 128, 60)
    clean = run(ctx, values, offsets, token, b1, b2, "gelu", 60, 30)
    values["x"][0][int(token[7]), 50] = np.nan
    O = run(ctx, values, offsets, token, b1, b2, "gelu", 60, 30)
    hit = torch.from_numpy(token == token[7]).cuda()
    assert torch.isnan(O[hit]).all() and torch.equal(O[~hit], clean[~hit])

"""How exact evomoe_expert_ffn_mx8 is: bit for bit where nothing may round before the results do, the activation next to the borders of its
8-bit rounding, and both products apart on ordinary data.  act(H) is read where it lies in the workspace: [P_cap, F] elements, up to
a multiple of 256 bytes, then the scales."""
import numpy as np
import pytest
import torch
from scipy.special import erfc

import test_gpu_mx8_experts as ex
from oracle import block_oracle as blk
from paper_2112_14397_amd import binding as B
from test_mx8_tiles import tiles

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = B.Context()
    yield c
    c.close()


def run(ctx, x, W1, W2, offsets, token, b1, b2, act, T):
    """x, W1, W2: (elements, scales).  O, and act(H) as (elements, scales), all float64."""
    (E, F, d), P = W1[0].shape, len(token)
    shape = B.make_shape(T, d, E, F, "bf16", act, P)
    (xq, xs), (w1, s1), (w2, s2) = (ex.to_gpu(*v) for v in (x, W1, W2))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    O = torch.full((P, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.evomoe_workspace_bytes_mx8(shape),), 255, dtype=torch.uint8, device="cuda")
    B.evomoe_hint_pairs(ctx, P)
    B.evomoe_expert_ffn_mx8(ctx, shape, xq, xs, dev(token), dev(offsets), w1, s1, dev(b1), w2, s2, dev(b2), O, ws)
    B.evomoe_hint_pairs(ctx, 0)
    torch.cuda.synchronize()
    at = (P * F + 255) // 256 * 256
    Aq = ws[:P * F].view(torch.float8_e4m3fn).view(P, F).double().cpu().numpy()
    As = ws[at:at + P * (F // 32)].view(torch.float8_e8m0fnu).view(P, F // 32).double().cpu().numpy()
    return O.double().cpu().numpy(), Aq, As


def experts_of(rng, E, P):
    share = rng.random(E) ** 2 + 0.01
    expert = np.sort(rng.choice(E, P, p=share / share.sum()))
    return np.searchsorted(expert, np.arange(E + 1)).astype(np.int32)


@pytest.mark.parametrize("T,d,E,F,P,first,second", ex.CASES + ex.LARGE)
@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_sums_to_the_last_bit(ctx, T, d, E, F, P, first, second, act):
    """Whole multiples of 8 everywhere: H, act(H) (gelu of 8 is 8 in float32, of -8 it is 0 in 8 bits) and O before its rounding are
    exact in float32, and of eight neighbouring products none lies 13 bits below another.  In both products a term of 2^18 units comes
    with the first 32 k's and goes with the last, where there are more: whatever loses bits of a sum in between shows."""
    rng = np.random.default_rng(T + d + E + F + P)
    X = rng.integers(-2, 3, (T, d)) * (rng.random((T, d)) < 0.3) * 1.0
    W1 = rng.integers(-1, 2, (E, F, d)) * 1.0
    W2 = rng.integers(-1, 2, (E, d, F)) * 1.0
    b1, b2 = 8.0 * rng.integers(-9, 10, (E, F)), 8.0 * rng.integers(-9, 10, (E, d))
    xs, s1, s2 = np.full((T, d // 32), 8.0), np.ones((E, F, d // 32)), np.ones((E, d, F // 32))
    if d > 32:
        X[:, :32], X[:, -32:] = 0, 0
        X[:, 3], X[:, -6], xs[:, 0], xs[:, -1] = 1, 1, 8 * 2.0 ** 18, 8 * 2.0 ** 18
        W1[:, :, -6] = -W1[:, :, 3]
    if F > 32:
        W1[:, (5, F - 9), :] = 0
        b1[:, (5, F - 9)] = 256                                                     # act(H) = 32 units there
        W2[:, :, :32], W2[:, :, -32:] = 0, 0
        W2[:, :, 5], W2[:, :, F - 9], s2[:, :, 0], s2[:, :, -1] = 1, -1, 2.0 ** 13, 2.0 ** 13
    offsets, token = experts_of(rng, E, P), rng.integers(0, T, P).astype(np.int32)
    O, Aq, As = run(ctx, (X, xs), (W1, s1), (W2, s2), offsets, token, b1.astype(np.float32), b2.astype(np.float32), act, T)
    rows = np.arange(P) if P * F * d < 1 << 29 else ex.some_rows(offsets, rng)
    for e in range(E):
        r = rows[(rows >= offsets[e]) & (rows < offsets[e + 1])]
        if not len(r):
            continue
        H = blk.mx8_value(X[token[r]], xs[token[r]]) @ W1[e].T + b1[e]
        assert abs(H).max() < 8 * 448
        q, s = blk.mx8(np.maximum(H, 0))                  # (there is something positive in every group, so that gelu has the same scales)
        assert q.reshape(len(r), -1, 32).max(-1).min() > 0
        assert np.array_equal(Aq[r], q) and np.array_equal(As[r], s), e
        A = blk.mx8_value(q, s)
        want = A @ blk.mx8_value(W2[e], s2[e]).T + b2[e]
        assert np.array_equal(want.astype(np.float32), want)
        assert np.array_equal(O[r], torch.from_numpy(want.astype(np.float32)).to(torch.bfloat16).double().numpy()), e


def gelu(h):
    h = np.asarray(h, np.float64)
    return 0.5 * h * erfc(-h * np.sqrt(0.5))


# what the activation may be off by: 4.7e-7 of the fitted exponent, and half a float32 step of the result
def off(v):
    return 5e-7 + U * abs(v)


def where_gelu_is(v, lo, hi):
    up = gelu(hi) > gelu(lo)
    for _ in range(80):
        mid = (lo + hi) / 2
        if (gelu(mid) < v) == up:
            lo = mid
        else:
            hi = mid
    return (lo + hi) / 2


def borders():
    """Groups of 32 values h next to borders of the 8-bit rounding of gelu(h), each group with a first value that sets its scale; and
    what the groups become."""
    numbers = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()            # 0 .. 448
    hs, scales = [], []
    for power in range(-11, -5):
        s = 2.0 ** power
        top = 420 * s
        mids = (numbers[1:] + numbers[:-1]) / 2 * s
        mids = mids[(mids < 0.99 * top) & (np.diff(numbers) * s > 2.5e-6)]                       # (borders that lie apart)
        low = -0.7517915                                                              # where gelu is least
        places = [where_gelu_is(m, 0.0, 8.0) for m in mids]
        places += [where_gelu_is(-m, low, 0.0) for m in mids if m < 0.169] + [where_gelu_is(-m, -8.0, low) for m in mids if m < 0.169]
        here = []
        for h in places:
            v = gelu(h)
            slope = (gelu(h + 1e-6) - gelu(h - 1e-6)) / 2e-6
            for sign in (-1, 1):
                step = sign * 1.02 * off(v) / slope
                c = np.float32(h + step)
                if abs(step) < 0.05 and abs(gelu(c) - v) >= off(v):
                    here.append(c)
        first = np.float32(where_gelu_is(top, 0.0, 8.0))
        while len(here) % 31:
            here.append(np.float32(0))
        for i in range(0, len(here), 31):
            hs.append(np.concatenate([[first], here[i:i + 31]]))
            scales.append(s)
    return np.array(hs, np.float32), np.array(scales)


@pytest.mark.parametrize("T,d,E,F,P,tile", [(96, 64, 48, 96, 96, "32x32/4"), (300, 512, 4, 1152, 700, "64x128/4"),
                                            (700, 384, 2, 2176, 1300, "128x128/4"), (300, 1056, 5, 1184, 3000, "128x128/4"),
                                            (400, 384, 1, 8832, 4000, "256x256/8")])
def test_gelu_next_to_the_borders_of_its_rounding(ctx, T, d, E, F, P, tile):
    """x = 0, so that H is the bias."""
    assert tiles(B.make_shape(T, d, E, F, "bf16", "gelu", P), P)[0] == tile
    groups, scales = borders()
    n = E * (F // 32)
    at = np.arange(n) % len(groups)
    assert n >= len(groups) > 40
    b1 = groups[at].reshape(E, F)
    zeros = lambda *s: (np.zeros(s), np.ones((*s[:-1], s[-1] // 32)))
    offsets = np.linspace(0, P, E + 1).astype(np.int32)
    O, Aq, As = run(ctx, zeros(T, d), zeros(E, F, d), zeros(E, d, F), offsets, np.zeros(P, np.int32), b1, np.zeros((E, d), np.float32), "gelu", T)
    q, s = blk.mx8(gelu(b1))
    assert np.array_equal(s.reshape(-1), scales[at])
    expert = np.searchsorted(offsets, np.arange(P), side="right") - 1
    assert np.array_equal(As, s[expert])
    bad = Aq != q[expert]
    assert not bad.any(), (int(bad.sum()), b1[expert][bad][:4], Aq[bad][:4], q[expert][bad][:4])
    assert (O == 0).all()


@pytest.mark.parametrize("T,d,E,F,P", [(48, 768, 16, 256, 48), (60, 384, 5, 640, 77), (400, 768, 4, 256, 4000), (700, 384, 2, 1280, 1300),
                                       (300, 480, 3, 736, 3000)])
@pytest.mark.parametrize("act", ["gelu", "relu"])
def test_both_products_on_ordinary_data(ctx, T, d, E, F, P, act):
    """The cut of eight neighbouring products is the oracle's; beside it there are float32's roundings: for sixteen products one of the sum
    and two terms cut off at as much, and four for the waves' sums and the bias."""
    rng = np.random.default_rng(T + d + F)
    values, _, token, b1, b2 = ex.inputs(rng, T, d, E, F, P)
    offsets = experts_of(rng, E, P)
    O, Aq, As = run(ctx, values["x"], values["W1"], values["W2"], offsets, token, b1, b2, act, T)
    xq, xs = values["x"]
    rows = np.sort(rng.choice(P, 12, replace=False))
    for e in range(E):
        r = rows[(rows >= offsets[e]) & (rows < offsets[e + 1])]
        if not len(r):
            continue
        H, size = blk.eights(xq[token[r]], xs[token[r]], values["W1"][0][e], values["W1"][1][e])
        H, far = H + b1[e], (3 * d / 16 + 4) * U * (size + abs(b1[e]))
        A = np.maximum(H, 0) if act == "relu" else gelu(H)
        far = far if act == "relu" else 1.13 * far + off(A)                             # |gelu'| <= 1.13
        got = blk.mx8_value(Aq[r], As[r])
        # (act(H) is rounded with its group's scale, which is the same unless the largest of the group may cross a power of two)
        amax = abs(A).reshape(len(r), -1, 32).max(-1)
        slack = far.reshape(len(r), -1, 32).max(-1)
        sure = np.repeat(blk.mx8_scale(amax - slack) == blk.mx8_scale(amax + slack), 32, axis=1)
        assert sure.mean() > 0.9
        scale = np.repeat(blk.mx8_scale(amax), 32, axis=1)
        lo, hi = blk.e4m3((A - far) / scale) * scale, blk.e4m3((A + far) / scale) * scale
        assert ((lo <= got) & (got <= hi))[sure].all()
        want, size = blk.eights(Aq[r], As[r], values["W2"][0][e], values["W2"][1][e])
        want, far = want + b2[e], (3 * F / 16 + 4) * U * (size + abs(b2[e]))
        assert (abs(O[r] - want) <= far + 2.0 ** -8 * (abs(want) + far)).all()


@pytest.mark.parametrize("small,at,kept", [(8.0, 2, 8.0), (4.0, 2, 0.0), (12.0, 7, 8.0), (0.5, 8, 0.5), (0.5, 40, 0.5)])
def test_what_eight_neighbours_lose(ctx, small, at, kept):
    """2^16 - 2^16 + small: of the same eight k's, what is below 2^3 is cut off; of others nothing is."""
    T, d, F = 4, 64, 32
    X, W1 = np.zeros((T, d)), np.zeros((1, F, d))
    X[:, :2], W1[:, :, :2] = (256, -256), 256
    X[:, at], W1[:, :, at] = small, 1
    one = lambda *s: np.ones((*s[:-1], s[-1] // 32))
    z = np.zeros((1, F), np.float32), np.zeros((1, d), np.float32)
    _, Aq, As = run(ctx, (X, one(T, d)), (W1, one(1, F, d)), (np.zeros((1, d, F)), one(1, d, F)), np.array([0, T], np.int32),
                    np.arange(T, dtype=np.int32), *z, "relu", T)
    assert (blk.mx8_value(Aq, As) == kept).all()

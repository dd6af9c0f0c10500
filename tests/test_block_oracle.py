"""CPU-only pins of the block oracle: gradients against central differences and torch's float64 autograd, the 8-bit rounding against
torch's e4m3, the selection against torch.topk where there are no ties, and its limits."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk

OPTIONS = [blk.TopK(1), blk.TopK(3), blk.TopK(3, renormalise=False, scale=2.5), blk.TopK(2, "sigmoid"),
           blk.TopK(4, "sigmoid", 4, 2, 2, True, 2.5), blk.TopK(2, "softmax", 6, 3, 1, False), blk.TopK(12, "sigmoid")]


@pytest.mark.parametrize("o", OPTIONS)
@pytest.mark.parametrize("with_coef", [False, True])
def test_gradient_of_the_weights_against_differences(o, with_coef):
    rng = np.random.default_rng(5)
    z, dG = rng.standard_normal((7, 12)), rng.standard_normal((7, 12))
    coef = rng.standard_normal(12) if with_coef else None
    mask = blk.topk_select(z, rng.standard_normal(12) * 0.1, o)
    got, mag = blk.topk_bwd(z, mask, dG, o, coef)
    loss = lambda z: (blk.topk_weights(z, mask, o) * dG).sum() + (0 if coef is None else (blk.scores(z, o.score) * coef).sum())
    eps = 1e-5
    for t, e in ((0, 0), (3, 5), (6, 11), (2, int(np.argmax(mask[2])))):
        step = np.zeros_like(z)
        step[t, e] = eps
        # central differences: third derivatives (below 10 here) times eps^2 / 6, and 2^-52 of the loss over eps
        assert abs((loss(z + step) - loss(z - step)) / (2 * eps) - got[t, e]) < 1e-8 * (1 + mag[t, e])


def test_selection_without_ties_is_topk():
    rng = np.random.default_rng(6)
    z = rng.standard_normal((50, 17))
    mask = blk.topk_select(z, None, blk.TopK(5))
    want = np.zeros_like(mask)
    np.put_along_axis(want, torch.from_numpy(z).topk(5, 1).indices.numpy(), True, 1)
    assert (mask == want).all()


def test_selection_at_its_limits():
    inf, nan = np.inf, np.nan
    z = np.array([[1, 1, 1, 1], [-inf, 2, -inf, -inf], [-inf] * 4, [nan, 9, 0, 0], [0, 0, inf, 5]])
    assert (blk.topk_select(z, None, blk.TopK(2)) ==
            np.array([[1, 1, 0, 0], [0, 1, 0, 0], [0, 0, 0, 0], [1, 1, 0, 0], [0, 0, 1, 1]], bool)).all()
    # a group that has one expert left is worth that one; a bias of -inf takes an expert out
    o = blk.TopK(2, "sigmoid", 2, 1, 2)
    assert (blk.topk_select([[-inf, 0.5, 0, -1]], None, o) == [[False, False, True, True]]).all()
    assert (blk.topk_select([[-inf, 5, -inf, -1]], None, o) == [[False, True, False, False]]).all()
    assert (blk.topk_select([[3, 2, 1, 0]], [-inf, 0, 0, 0], blk.TopK(1, "sigmoid")) == [[False, True, False, False]]).all()
    assert blk.scores(np.full((1, 3), -inf), "softmax").tolist() == [[0, 0, 0]]


@pytest.mark.parametrize("with_dh", [False, True])
def test_norm_gradients_against_autograd(with_dh):
    rng = np.random.default_rng(7)
    h, dy, dh, gamma = rng.standard_normal((5, 24)), rng.standard_normal((5, 24)), rng.standard_normal((5, 24)), rng.standard_normal(24)
    (dx, dgamma), _ = blk.rmsnorm_bwd(dy, dh if with_dh else None, h, gamma, 1e-3)
    ht, gt = torch.tensor(h, requires_grad=True), torch.tensor(gamma, requires_grad=True)
    y = ht * torch.rsqrt(ht.square().mean(1, keepdim=True) + 1e-3) * gt
    (y * torch.tensor(dy)).sum().backward()
    np.testing.assert_allclose(dx, ht.grad.numpy() + (dh if with_dh else 0), atol=1e-12)
    np.testing.assert_allclose(dgamma, gt.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(blk.rmsnorm(h, gamma, 1e-3)[0], y.detach().numpy(), atol=1e-12)


def test_e4m3_is_torch_s():
    v = np.concatenate([np.linspace(-448, 448, 9001), np.linspace(-0.05, 0.05, 4001), [2.0 ** -10, 3 * 2.0 ** -10, 17, 19, 27]])
    v = v.astype(np.float32)
    assert np.array_equal(blk.e4m3(v), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())


def test_scales_keep_every_group_within_448_and_no_larger_than_needed():
    amax = np.float32(10.0) ** np.linspace(-37, 37, 999, dtype=np.float32)
    amax = np.concatenate([amax, np.float32([448, 448.0001, 447.9999, 1.75, 1.7500001, 2.0 ** 100, 3e38])]).astype(np.float64)
    s = blk.mx8_scale(amax)
    assert (amax / s <= 448).all() and ((amax / (s / 2) > 448) | (s == 2.0 ** -127)).all()
    assert blk.mx8_scale(np.array([0.0, 2.0 ** -140])).tolist() == [2.0 ** -127] * 2
    q, scale = blk.mx8(np.array([[np.inf, -np.nan, 3.0] + [1.0] * 29]))
    assert np.isnan(q[0, :2]).all() and scale[0, 0] == 2.0 ** -7 and q[0, 2] == 384

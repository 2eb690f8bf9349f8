"""The oracle's group normalization, top logits and distillation: gradients against differences of the forward functions, and what
their definitions say of simple inputs."""
import numpy as np
import pytest

from oracle import ops as orc


def _difference(f, v, step=1e-5):
    """Central differences of the scalar function f at v."""
    out = np.empty_like(v)
    for i in np.ndindex(*v.shape):
        hi, lo = v.copy(), v.copy()
        hi[i] += step
        lo[i] -= step
        out[i] = (f(hi) - f(lo)) / (2 * step)
    return out


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("use_res", [False, True])
def test_gn_gradients_against_differences(act, use_res):
    g = np.random.default_rng(5)
    n, c, h, w, groups, eps = 2, 6, 3, 2, 2, 1e-3
    x, res, dy = g.normal(size=(n, c, h, w)), g.normal(size=(n, c, h, w)), g.normal(size=(n, c, h, w))
    gamma, beta = 1 + 0.3 * g.normal(size=c), 0.3 * g.normal(size=c)
    r = res if use_res else None
    _, mean, invstd = orc.gn_fwd(x, groups, gamma, beta, eps, r, act)
    u = orc.gn_fwd(x, groups, gamma, beta, eps, r)[0]
    # differences stay on one side of the ReLU's corner: a step of 1e-5 in x, gamma, beta or the residual moves u by 1e-5 times at most
    # gamma*invstd, xhat or 1, none above 10
    assert np.abs(u).min() > 1e-4 and np.abs(gamma).max() * invstd.max() < 10
    dx, dres, dgamma, dbeta = orc.gn_bwd(x, dy, groups, gamma, beta, mean, invstd, r, act)

    def loss(x=x, gamma=gamma, beta=beta, r=r):
        return (orc.gn_fwd(x, groups, gamma, beta, eps, r, act)[0] * dy).sum()

    for got, f, at in ((dx, lambda v: loss(x=v), x), (dgamma, lambda v: loss(gamma=v), gamma), (dbeta, lambda v: loss(beta=v), beta),
                       (dres, (lambda v: loss(r=v)) if use_res else None, res)):
        if f is not None:
            np.testing.assert_allclose(got, _difference(f, at), rtol=1e-6, atol=1e-7)


def test_gn_with_one_group_per_image_and_one_per_channel():
    g = np.random.default_rng(6)
    x = g.normal(size=(3, 4, 5, 7)) + 3
    one, zero = np.ones(4), np.zeros(4)
    y, mean, invstd = orc.gn_fwd(x, 1, one, zero, 0.0)
    np.testing.assert_allclose(mean[:, 0], x.mean(axis=(1, 2, 3)))
    np.testing.assert_allclose(y.var(axis=(1, 2, 3)), 1.0)
    y, mean, invstd = orc.gn_fwd(x, 4, one, zero, 0.0)
    np.testing.assert_allclose(y, (x - x.mean((2, 3), keepdims=True)) / x.std((2, 3), keepdims=True))
    # one image of a batch: the statistics of batch normalization over it alone
    np.testing.assert_allclose(orc.gn_fwd(x[:1], 4, one, zero, 1e-5)[0], orc.bn_fwd(x[:1], one, zero, 1e-5)[0])


def test_topk_order():
    z = np.array([[1.0, 3.0, -0.0, 3.0, 0.0, -np.inf, np.nan, np.inf]])
    val, idx = orc.topk(z, 8)
    assert idx.tolist() == [[6, 7, 1, 3, 0, 2, 4, 5]]
    assert orc.topk(z[:, :6], 2)[0].tolist() == [[3.0, 3.0]]


@pytest.mark.parametrize("alpha,tau", [(0.0, 1.0), (0.4, 2.5), (1.0, 0.7)])
def test_distillation_gradient_against_differences(alpha, tau):
    g = np.random.default_rng(7)
    n, k, t = 5, 7, 4
    z, val = 2 * g.normal(size=(n, k)), g.normal(size=(n, t))
    idx = np.stack([g.permutation(k)[:t] for _ in range(n)])
    labels = np.array([1, -1, 0, 6, -1])
    idx[1, 2] = -1
    idx[2, 0] = idx[2, 3]
    val[3, 1] = -np.inf
    idx[4] = -1
    loss, grad = orc.distill_ce(z, labels, idx, val, alpha, tau, 0.3)
    np.testing.assert_allclose(grad, _difference(lambda v: orc.distill_ce(v, labels, idx, val, alpha, tau, 0.3)[0][0], z), rtol=1e-5, atol=1e-8)
    np.testing.assert_array_equal(grad[4], 0.0)


def test_distillation_against_softmax_ce_and_itself():
    g = np.random.default_rng(8)
    z, labels = g.normal(size=(6, 9)), g.integers(0, 9, 6)
    loss, grad = orc.distill_ce(z, labels, None, None, 0.0, 1.0, 1 / 6)
    ref, ref_grad = orc.softmax_ce(z, labels)
    np.testing.assert_allclose(loss, [ref, ref, 0.0])
    np.testing.assert_allclose(grad, ref_grad)
    # a teacher that keeps every logit and is the student: nothing to learn
    loss, grad = orc.distill_ce(z, None, np.tile(np.arange(9), (6, 1)), z, 1.0, 3.0, 1.0)
    np.testing.assert_allclose(loss, 0.0, atol=1e-12)
    np.testing.assert_allclose(grad, 0.0, atol=1e-12)

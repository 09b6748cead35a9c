"""The float64 definitions in oracle/operators_oracle.py, pinned by automatic differentiation and by differences."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as O


def test_layernorm_is_torch_layer_norm_in_64_bits():
    rng = np.random.default_rng(0)
    x, gain, shift = rng.normal(size=(3, 5, 17)), rng.normal(size=17), rng.normal(size=17)
    y, hat, mean, rstd = O.layernorm(x, gain, shift, 1e-5)
    want = torch.nn.functional.layer_norm(torch.from_numpy(x), (17,), torch.from_numpy(gain), torch.from_numpy(shift), 1e-5).numpy()
    assert np.abs(y - want).max() < 1e-13
    assert np.abs(hat.mean(-1)).max() < 1e-13 and np.abs((x - mean[..., None]) * rstd[..., None] - hat).max() == 0


def test_layernorm_backward_is_autograd_example_by_example():
    rng = np.random.default_rng(1)
    x, g, gain = rng.normal(size=(3, 5, 17)), rng.normal(size=(3, 5, 17)), rng.normal(size=17)
    _, _, mean, rstd = O.layernorm(x, gain, None, 1e-5)
    dx, gs, ss, sq = O.layernorm_backward(g, x, gain, mean, rstd)
    for i in range(3):
        tx, tg, tb = (torch.tensor(v, requires_grad=True) for v in (x[i], gain, np.zeros(17)))
        y = torch.nn.functional.layer_norm(tx, (17,), tg, tb, 1e-5)
        wx, wg, wb = torch.autograd.grad(y, (tx, tg, tb), torch.from_numpy(g[i]))
        assert np.abs(dx[i] - wx.numpy()).max() < 1e-12
        assert np.abs(gs[i] - wg.numpy()).max() < 1e-12 and np.abs(ss[i] - wb.numpy()).max() < 1e-12
        assert abs(sq[i] - (wg.square().sum() + wb.square().sum()).item()) < 1e-11


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_loss_and_gradient(smoothing):
    rng = np.random.default_rng(2)
    B, T, V, beta = 3, 4, 11, 0.7
    x = rng.normal(size=(B, 2 * T, V)) * 2
    t = rng.integers(0, V, size=(B, 2, T))
    t[0, 0, 2], t[1, 1, :], t[2, 0, 0] = -1, -5, V + 3
    ref = rng.normal(size=(B, 2)) - 8
    loss, logp, G = O.preference_loss(x, t, ref, beta, smoothing)
    tx = torch.tensor(x, requires_grad=True)
    tt = torch.from_numpy(np.where((t < 0) | (t >= V), -100, t)).view(B * 2 * T)
    token = -torch.nn.functional.cross_entropy(tx.view(-1, V), tt, ignore_index=-100, reduction="none")
    lp = token.view(B, 2, T).sum(-1)
    h = beta * ((lp[:, 0] - lp[:, 1]) - torch.from_numpy(ref[:, 0] - ref[:, 1]))
    ls = torch.nn.functional.logsigmoid
    want = -(1 - smoothing) * ls(h) - smoothing * ls(-h)
    assert np.abs(logp - lp.detach().numpy()).max() < 1e-12 and np.abs(loss - want.detach().numpy()).max() < 1e-12
    assert np.abs(G - torch.autograd.grad(want.sum(), tx)[0].numpy()).max() < 1e-13
    assert not G[1, T:].any() and not G[0, 2].any() and not G[2, 0].any()
    # differences along a random direction
    d, step = rng.normal(size=x.shape), 1e-6
    up, down = (O.preference_loss(x + s * d, t, ref, beta, smoothing)[0].sum() for s in (step, -step))
    assert abs((up - down) / (2 * step) - (G * d).sum()) < 1e-7


@pytest.mark.parametrize("shape", [(6, 6), (5, 12), (12, 5), (1, 9)])
def test_newton_schulz_acts_on_the_singular_values(shape):
    rng = np.random.default_rng(3)
    M = rng.normal(size=shape)
    coefs = [(3.4445, -4.7750, 2.0315)] * 5
    u, s, vt = np.linalg.svd(M, full_matrices=False)
    s = s / (np.linalg.norm(M) + 1e-7)
    for a, b, c in coefs:
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.abs(O.orthogonalize(M, coefs, 1e-7, 1.5) - 1.5 * (u * s) @ vt).max() < 1e-12


@pytest.mark.parametrize("smoothing", [0.0, 0.1, 1.0])
def test_preference_loss_of_answers_that_cannot_be(smoothing):
    """A target at -inf: h is infinite, and a term of weight 0 is not in the loss."""
    rng = np.random.default_rng(4)
    x, t = rng.normal(size=(2, 4, 5)), np.ones((2, 2, 2), dtype=int)
    x[0, 3, 1] = x[1, 0, 1] = -np.inf                # the other answer, the preferred one
    loss, logp, G = O.preference_loss(x, t, None, 0.5, smoothing)
    want = {0.0: [0.0, np.inf], 0.1: [np.inf, np.inf], 1.0: [np.inf, 0.0]}[smoothing]
    assert list(loss) == want
    assert logp[0, 1] == -np.inf and logp[1, 0] == -np.inf and np.isfinite(logp[0, 0]) and np.isfinite(logp[1, 1])
    soft = np.exp(x) / np.exp(x).sum(-1, keepdims=True)
    for i, slope in enumerate((0.5 * smoothing, -0.5 * (1 - smoothing))):        # beta (e s(h) - (1 - e) s(-h)) at either end
        for r in range(4):
            c = slope if r < 2 else -slope
            assert np.abs(G[i, r] - c * (np.eye(5)[1] - soft[i, r])).max() < 1e-15

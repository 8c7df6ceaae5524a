"""Pins of the oracle of the losses over a vocabulary: a library's own losses with reverse-mode differentiation, finite differences, and
cases that can be written down."""
import numpy as np
import pytest
import torch

from oracle import vocab_oracle as VO


def _case(M, D, V, K, tau, bias, seed=0):
    rng = np.random.default_rng(seed)
    params = rng.standard_normal(V * D + (V if bias else 0)) * 0.4
    X = rng.standard_normal((M, D))
    labels = rng.integers(0, V, M)
    labels[::3] = -100
    idx = rng.integers(0, V, (M, K))
    idx[1::4] = -1
    logits = 2 * rng.standard_normal((M, K))
    return params, X, labels, idx, logits, rng.standard_normal(M), rng.standard_normal(M)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_against_a_library_with_autodiff(bias, tau):
    M, D, V, K = 9, 5, 17, 4
    params, X, labels, idx, logits, dce, dkd = _case(M, D, V, K, tau, bias)
    got = VO.vocab_loss(params, X, V, bias, labels, idx, logits, tau, dce, dkd)
    p = torch.tensor(params, requires_grad=True)
    x = torch.tensor(X, requires_grad=True)
    z = torch.nn.functional.linear(x, p[:V * D].view(V, D), p[V * D:] if bias else None)
    ce = torch.nn.functional.cross_entropy(z, torch.tensor(labels), ignore_index=-100, reduction="none")
    target = torch.zeros(M, V, dtype=torch.float64)
    for r in range(M):
        on = idx[r] >= 0
        if on.any():
            target[r].index_add_(0, torch.tensor(idx[r][on]), torch.softmax(torch.tensor(logits[r][on]) / tau, 0))
    # the divergence counts entries one by one, so where an index repeats its p log p differs from that of the summed target by a constant
    kl = torch.nn.functional.kl_div(torch.log_softmax(z / tau, 1), target, reduction="none").sum(1) * tau * tau
    total = (ce * torch.tensor(dce)).sum() + (kl * torch.tensor(dkd)).sum()
    total.backward()
    np.testing.assert_allclose(got["loss_ce"], ce.detach().numpy(), atol=1e-12)
    single = [r for r in range(M) if len(set(idx[r])) == K]
    assert single
    np.testing.assert_allclose(got["loss_kd"][single], kl.detach().numpy()[single], atol=1e-12)
    np.testing.assert_allclose(got["dX"], x.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(got["dparams"], p.grad.numpy(), atol=1e-12)


def test_gradients_against_differences():
    M, D, V, K, tau = 4, 3, 7, 3, 2.0
    params, X, labels, idx, logits, dce, dkd = _case(M, D, V, K, tau, True, seed=3)
    idx[2] = [5, 5, 1]

    def value(p, x):
        o = VO.vocab_loss(p, x, V, True, labels, idx, logits, tau)
        return (o["loss_ce"] * dce).sum() + (o["loss_kd"] * dkd).sum()

    got = VO.vocab_loss(params, X, V, True, labels, idx, logits, tau, dce, dkd)
    h = 1e-6
    for i in range(0, params.size, 3):
        d = np.zeros_like(params)
        d[i] = h
        assert abs((value(params + d, X) - value(params - d, X)) / (2 * h) - got["dparams"][i]) < 1e-7
    for i in range(X.size):
        d = np.zeros_like(X)
        d.flat[i] = h
        assert abs((value(params, X + d) - value(params, X - d)) / (2 * h) - got["dX"].flat[i]) < 1e-7


def test_closed_forms():
    V, D = 6, 4
    X = np.ones((2, D))
    o = VO.vocab_loss(np.zeros(V * D), X, V, False, labels=np.array([2, -100]), dce=np.ones(2))
    assert np.allclose(o["loss_ce"], [np.log(V), 0.0]) and np.allclose(o["lse"], [np.log(V), 0.0])
    assert np.allclose(o["dparams"].reshape(V, D)[:, 0], 1 / V - (np.arange(V) == 2))
    # a student that equals a teacher known at every entry: no divergence, no gradient
    rng = np.random.default_rng(1)
    W = rng.standard_normal((V, D))
    z = X @ W.T
    idx = np.tile(np.arange(V), (2, 1))
    o = VO.vocab_loss(W.ravel(), X, V, False, teacher_idx=idx, teacher_logits=z, tau=3.0, dkd=np.ones(2))
    assert np.allclose(o["loss_kd"], 0) and np.allclose(o["dX"], 0) and np.allclose(o["dparams"], 0)
    # one entry alone is a label, times tau
    one = VO.vocab_loss(W.ravel(), X, V, False, teacher_idx=np.array([[4, -1], [7, 1]]), teacher_logits=np.array([[5.0, 9.0], [1.0, -np.inf]]),
                        tau=2.0, dkd=np.ones(2))
    ce = VO.vocab_loss(W.ravel() / 2.0, X, V, False, labels=np.array([4, -1]), dce=np.ones(2))
    assert np.allclose(one["loss_kd"], 4 * ce["loss_ce"]) and np.allclose(one["dX"], 4 * ce["dX"]) and one["lse_tau"][1] == 0

"""The oracle of a training step's head against torch's own operators on the CPU in fp64, values and autograd."""
import numpy as np
import pytest

from oracle import head_oracle as O

torch = pytest.importorskip("torch")
TOL = 1e-12                              # two fp64 computations of a few hundred operations on values of order 1


def _leaf(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).requires_grad_()


@pytest.mark.parametrize("n,H,eps", [(1, 1, 1e-5), (4, 7, 1e-5), (9, 40, 1e-3), (3, 150, 0.5)])
def test_layernorm(n, H, eps):
    rng = np.random.default_rng([n, H])
    x, gamma, beta, gy = rng.standard_normal((n, H)) + 2, rng.standard_normal(H), rng.standard_normal(H), rng.standard_normal((n, H))
    x_t, gamma_t, beta_t = _leaf(x), _leaf(gamma), _leaf(beta)
    y_t = torch.nn.functional.layer_norm(x_t, (H,), gamma_t, beta_t, eps)
    y_t.backward(torch.from_numpy(gy))
    y, mean, rstd = O.layernorm(x, gamma, beta, eps)
    assert np.abs(y - y_t.detach().numpy()).max() < TOL
    assert np.abs(mean - x.sum(1) / H).max() < TOL and np.abs(rstd ** -2 - x.var(1) - eps).max() < TOL
    for mine, leaf in zip(O.layernorm_backward(x, gamma, gy, eps), (x_t, gamma_t, beta_t)):
        # (a row of one value has rstd 300 and a gradient of 0)
        assert np.abs(mine - leaf.grad.numpy()).max() < TOL * 1e3


@pytest.mark.parametrize("n,H,C", [(1, 3, 1), (5, 4, 2), (30, 12, 9), (40, 20, 300)])
@pytest.mark.parametrize("bias", ["none", "random", "masked"])
def test_softmax_xent(n, H, C, bias):
    rng = np.random.default_rng([n, H, C])
    h, V, gloss = rng.standard_normal((n, H)), rng.standard_normal((C, H)), rng.random(n)
    label = rng.integers(-1, C, n)
    b = None if bias == "none" else rng.standard_normal(C)
    if bias == "masked":
        out = np.setdiff1d(np.arange(0, C - 1, 2), label)     # (the last class stays: torch makes rows without a label NaN where none does)
        b[out] = -np.inf
    h_t, V_t = _leaf(h), _leaf(V)
    b_t = None if b is None else _leaf(b)
    z = h_t @ V_t.t() + (0.0 if b is None else b_t)
    loss_t = torch.nn.functional.cross_entropy(z, torch.from_numpy(label), ignore_index=-1, reduction="none")
    (loss_t * torch.from_numpy(gloss)).sum().backward()
    loss, lse = O.softmax_xent(h, V, b, label)
    assert np.abs(loss - loss_t.detach().numpy()).max() < TOL
    assert np.abs(lse - np.where(label == -1, 0.0, torch.logsumexp(z, 1).detach().numpy())).max() < TOL
    dh, dV, db, g, p = O.softmax_xent_backward(h, V, b, label, gloss)
    assert np.abs(dh - h_t.grad.numpy()).max() < TOL and np.abs(dV - V_t.grad.numpy()).max() < TOL
    if b is not None:
        assert np.abs(db - b_t.grad.numpy()).max() < TOL
    used = label != -1
    assert np.abs(p[used] - torch.softmax(z, 1).detach().numpy()[used]).max(initial=0.0) < TOL and not p[~used].any()

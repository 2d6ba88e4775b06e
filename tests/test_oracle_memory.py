"""The oracles of the operators around a gated memory, against differences, closed forms and library calls in fp64."""
import numpy as np
import torch

from oracle import gated_recurrence as ogr, muon as om, rms_norm as orn


def _differences(loss, base, i, h=1e-6):
    up, down = [b.copy() for b in base], [b.copy() for b in base]
    ref = np.zeros_like(base[i])
    for k in np.ndindex(ref.shape):
        up[i][k] += h
        down[i][k] -= h
        ref[k] = (loss(*up) - loss(*down)) / (2 * h)
        up[i][k] = down[i][k] = base[i][k]
    return ref


def test_recurrence_gradients():
    r = np.random.default_rng(0).normal
    T, N, D = 7, 3, 2
    x, g, dh, s0, ds = r(size=(T, N, D)), r(size=(T, N, D)), r(size=(T, N, D)), r(size=(N, D)), r(size=(N, D))
    dones = (np.random.default_rng(1).random((T, N)) < 0.25).astype(np.uint8)
    lengths = np.array([7, 4, 0])

    def loss(x, g, s0):
        h, last, _ = ogr.forward(x, g, s0, dones, lengths)
        return (h * dh).sum() + (last * ds).sum()
    for i, got in enumerate(ogr.backward(x, g, dh, ds, s0, dones, lengths)):
        assert np.abs(got - _differences(loss, [x, g, s0], i)).max() < 1e-8


def test_recurrence_closed_form_and_episodes():
    """Equal gates: a geometric sum.  An episode that ends starts the next from zero."""
    T = 30
    x, g = np.ones((T, 1, 1)), np.full((T, 1, 1), 1.3)
    f = 1 / (1 + np.exp(-1.3))
    h, last, _ = ogr.forward(x, g)
    assert np.allclose(h[:, 0, 0], 1 - f ** np.arange(1, T + 1), atol=1e-14) and np.allclose(last, h[-1])
    dones = np.zeros((T, 1), np.uint8)
    dones[11] = 1
    h2, _, _ = ogr.forward(x, g, dones=dones)
    assert np.allclose(h2[:12], h[:12]) and np.allclose(h2[12:], h[:18])
    dones[-1] = 1
    assert not ogr.forward(x, g, dones=dones)[1].any()


def test_norm_gradients_and_library():
    r = np.random.default_rng(2).normal
    x, res, dy, dt, w = r(size=(4, 9)), r(size=(4, 9)), r(size=(4, 9)), r(size=(4, 9)), r(size=9)
    y, z, rstd = orn.forward(x, res, w, 1e-3)
    lib = torch.nn.functional.rms_norm(torch.as_tensor(x + res), (9,), torch.as_tensor(w), 1e-3).numpy()
    assert np.allclose(y, lib, atol=1e-13)

    def loss(x, w):
        y, z, _ = orn.forward(x, res, w, 1e-3)
        return (y * dy).sum() + (z * dt).sum()
    dx, dw = orn.backward(dy, z, w, rstd, dt)
    assert np.abs(dx - _differences(loss, [x, w], 0)).max() < 1e-7 and np.abs(dw - _differences(loss, [x, w], 1)).max() < 1e-7


def test_newton_schulz_acts_on_the_singular_values():
    g = np.random.default_rng(3)
    for shape in ((5, 9), (9, 5), (6, 6), (1, 4)):
        u = g.normal(size=shape)
        a, s, b = np.linalg.svd(u, full_matrices=False)
        s = s / np.linalg.norm(s)
        for _ in range(5):
            s = om.A * s + om.B * s ** 3 + om.C * s ** 5
        x = om.orthogonalize(u, 5)
        assert np.allclose(x, (a * s) @ b, atol=1e-12) and (s < 1.21).all()
    assert not om.orthogonalize(np.zeros((3, 4)), 5).any()


def test_muon_step_by_hand():
    w, grad, m = np.array([[2.0]]), np.array([[0.5]]), np.array([[1.0]])
    x = 1.0
    for _ in range(2):
        x = om.A * x + om.B * x ** 3 + om.C * x ** 5
    nw, nm, nx, u = om.step(w, grad, m, 0.1, 0.9, True, 0.5, 2, 3.0)
    assert np.isclose(nm[0, 0], 1.4) and np.isclose(u[0, 0], 0.5 + 0.9 * 1.4) and np.isclose(nx[0, 0], x) and np.isclose(nw[0, 0], 0.95 * 2 - 0.3 * x)


def test_steepest_bounds_what_a_step_does_to_a_small_change():
    g = np.random.default_rng(4)
    x = g.normal(size=(6, 8))
    x /= np.linalg.norm(x)

    def one(x):
        a = x @ x.T
        return om.A * x + (om.B * a + om.C * (a @ a)) @ x
    bound = om.steepest(np.linalg.svd(x, compute_uv=False))
    for _ in range(20):
        d = g.normal(size=x.shape) * 1e-6
        assert np.linalg.norm(one(x + d) - one(x)) <= bound * np.linalg.norm(d) * (1 + 1e-4)

"""The example memory (norm, projections, linear attention, norm): steps are the sequence, gradients are the formula's, training recalls."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import layer_norm as oln, linear_attention as ola
from sequence_util import U, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lm():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "linear_memory.py")
    spec = importlib.util.spec_from_file_location("linear_memory", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.rx.rslx_device_check()
    return m


def _oracle(memory, obs, dones, s0, d_answer):
    """Answers, states and gradients in 64 bits."""
    T, N, H, D = memory.T, memory.N, memory.H, memory.D
    p = {n: f64(w) for n, w in memory.params.items()}
    x = f64(obs).reshape(T * N, -1)
    h = x @ p["w_in"]
    z, m1, r1 = oln.forward(h, p["g1"], p["b1"])
    qkv = [a.reshape(T, N, H, D) for a in np.split(z @ p["w_qkv"], 3, 1)]
    args = (*qkv, f64(memory.log_decay), float(np.float32(memory.scale)))
    o, s = ola.forward(*args, s0=f64(s0), dones=dones.cpu().numpy())
    o = o.reshape(T * N, -1)
    y, m2, r2 = oln.forward(o, p["g2"], p["b2"])
    d = f64(d_answer).reshape(T * N, -1)
    g = dict(w_out=y.T @ d)
    do, g["g2"], g["b2"] = oln.backward(d @ p["w_out"].T, o, p["g2"], m2, r2)
    dqkv = ola.backward(*args, do=do.reshape(T, N, H, D), s0=f64(s0), dones=dones.cpu().numpy())[:3]
    dqkv = np.concatenate([a.reshape(T * N, -1) for a in dqkv], 1)
    g["w_qkv"] = z.T @ dqkv
    dx, g["g1"], g["b1"] = oln.backward(dqkv @ p["w_qkv"].T, h, p["g1"], m1, r1)
    g["w_in"] = x.T @ dx
    return (y @ p["w_out"]).reshape(T, N, -1), s, g


def _near(got, ref, roundings, name):
    """Within that many fp32 roundings of the result's size as a whole: sums of products lose a few each, their errors are of either sign."""
    assert np.linalg.norm(f64(got) - ref) <= roundings * U * np.linalg.norm(ref), name


def test_sequence_and_gradients(lm):
    T, N = 12, 6
    memory = lm.LinearMemory(T, N, 5, 4, heads=3, width=20, seed=3)
    g = torch.Generator("cuda").manual_seed(4)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    for name in ("g1", "g2", "b1", "b2"):
        memory.params[name] += 0.2 * normal(60)
    obs, s0, d = normal(T, N, 5), normal(N, 3, 20, 20), normal(T, N, 4)
    dones = (torch.rand(T, N, generator=g, device="cuda") < 0.1).to(torch.uint8)
    out, s = memory.forward(obs, dones, s0)
    grads = memory.backward(d)
    ref_out, ref_s, ref_g = _oracle(memory, obs, dones, s0, d)
    # norms divide by a row's spread, products of 60 and 72 terms follow each other: at most some thousand roundings in a row
    _near(out, ref_out, 4000, "answers")
    _near(s, ref_s, 4000, "states")
    assert set(grads) == set(memory.params)
    for name, grad in grads.items():
        _near(grad, ref_g[name], 8000, name)


def test_steps_are_the_sequence(lm):
    T, N = 9, 5
    memory = lm.LinearMemory(T, N, 5, 4, heads=2, width=16, seed=5)
    world = lm.Recall(N, end_p=0.3, seed=6)
    obs, _, dones = world.steps(T)
    out, s = memory.forward(obs, dones, memory.state)
    for t in range(T):
        y = memory.act(obs[t], dones[t - 1] if t else None)
        _near(y, f64(out[t]), 4000, t)
    memory.state[dones[-1].bool()] = 0
    _near(memory.state, f64(s), 4000, "states")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_recalls(lm, dtype):
    memory, world, losses = lm.train(T=24, N=64, iterations=150, dtype=dtype)
    # signs have a square of 1: answers of zero cost 1
    assert losses[0] > 0.9 and np.mean(losses[-10:]) < 0.5

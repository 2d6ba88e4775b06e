"""The example memory (norm, projections, gated recurrence, norm over the residual, Muon steps): gradients are the formula's, steps are the sequence, a training
iteration runs captured as it runs eagerly."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import gated_recurrence as ogr, muon as om, rms_norm as orn
from sequence_util import U, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gm():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_memory.py")
    spec = importlib.util.spec_from_file_location("gated_memory", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.rx.rslx_device_check()
    return m


def _oracle(memory, obs, dones, s0, d_answer):
    """Answers, states and gradients in 64 bits."""
    T, N, M = memory.T, memory.N, memory.M
    p = {n: f64(w) for n, w in memory.params.items()}
    x, rows = f64(obs).reshape(T * N, -1), T * N
    e = x @ p["w_in"]
    z, _, r1 = orn.forward(e, None, p["n1"])
    cg = (z @ p["w_cg"]).reshape(T, N, 2 * M)
    c, g = cg[..., :M], cg[..., M:] + f64(memory.bias)
    h, s, _ = ogr.forward(c, g, f64(s0), dones.cpu().numpy())
    y, total, r2 = orn.forward(h.reshape(rows, M) @ p["w_h"], e, p["n2"])
    d = f64(d_answer).reshape(rows, -1)
    G = dict(w_out=y.T @ d)
    d_sum, G["n2"] = orn.backward(d @ p["w_out"].T, total, p["n2"], r2)
    G["w_h"] = h.reshape(rows, M).T @ d_sum
    dc, dg, _ = ogr.backward(c, g, (d_sum @ p["w_h"].T).reshape(T, N, M), None, f64(s0), dones.cpu().numpy())
    dcg = np.concatenate([dc, dg], 2).reshape(rows, -1)
    G["w_cg"] = z.T @ dcg
    de, G["n1"] = orn.backward(dcg @ p["w_cg"].T, e, p["n1"], r1, d_sum)
    G["w_in"] = x.T @ de
    return (y @ p["w_out"]).reshape(T, N, -1), s, G


def _near(got, ref, roundings, name):
    """Within that many fp32 roundings of the result's size as a whole: sums of products lose a few each, their errors are of either sign."""
    assert np.linalg.norm(f64(got) - ref) <= roundings * U * np.linalg.norm(ref), name


def _inputs(memory, seed, d_in=5, d_out=4):
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    T, N, M = memory.T, memory.N, memory.M
    dones = (torch.rand(T, N, generator=g, device="cuda") < 0.1).to(torch.uint8)
    return normal(T, N, d_in), dones, normal(N, M), normal(T, N, d_out)


def test_sequence_and_gradients(gm):
    memory = gm.GatedMemory(14, 6, 5, 4, M=44, seed=3)
    for name in ("n1", "n2"):
        memory.params[name] += 0.2 * torch.randn(44, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    obs, dones, s0, d = _inputs(memory, 4)
    out, s = memory.forward(obs, dones, s0)
    grads = memory.backward(d)
    ref_out, ref_s, ref_g = _oracle(memory, obs, dones, s0, d)
    # products of 44 to 88 terms follow each other with two norms and a recurrence between them: at most some thousand roundings in a row
    _near(out, ref_out, 4000, "answers")
    _near(s, ref_s, 4000, "states")
    assert set(grads) == set(memory.params)
    for name, grad in grads.items():
        _near(grad, ref_g[name], 8000, name)


def test_steps_are_the_sequence(gm):
    T, N = 9, 5
    memory = gm.GatedMemory(T, N, 5, 4, M=32, seed=5)
    world = gm.Recall(N, end_p=0.3, seed=6)
    obs, _, dones = world.steps(T)
    out, s = memory.forward(obs, dones, memory.state)
    for t in range(T):
        _near(memory.act(obs[t], dones[t - 1] if t else None), f64(out[t]), 4000, t)
    memory.state[dones[-1].bool()] = 0
    _near(memory.state, f64(s), 4000, "states")


def test_the_matrices_take_muons_step(gm):
    memory = gm.GatedMemory(6, 8, 5, 4, M=40, seed=7)
    obs, dones, s0, d = _inputs(memory, 8)
    memory.forward(obs, dones, s0)
    memory.backward(d)
    before = {n: memory.params[n].clone() for n in memory.params}
    memory.step()
    cfg = memory.muon.cfg
    for n, (_, _, grad, _, _, scale) in zip(memory.muon_names, memory.muon.matrices):
        w, m, x, u = om.step(f64(before[n]), f64(grad), 0.0, cfg.lr, cfg.momentum, True, 0.0, 5, scale)
        _near(memory.muon.matrices[memory.muon_names.index(n)][4], m, 4, n)
        # (how far the update itself may be off is its own test's; here: this matrix's, and no other's)
        assert np.linalg.norm(f64(memory.params[n]) - w) <= 0.01 * np.linalg.norm(w - f64(before[n])), n
    for n in ("w_out", "n1", "n2"):
        assert not torch.equal(before[n], memory.params[n])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_runs(gm, dtype):
    memory, world, losses = gm.train(T=24, N=64, iterations=5, dtype=dtype)
    assert len(losses) == 5 and np.isfinite(losses).all()
    assert all(torch.isfinite(p).all() for p in memory.params.values())


def test_an_iteration_in_a_graph(gm):
    """Forward, backward and the Muon step captured together: replays change the weights as eager iterations do, bit for bit."""
    def fresh():
        memory = gm.GatedMemory(40, 7, 5, 4, M=36, dtype=torch.bfloat16, seed=9)
        return memory, _inputs(memory, 10)

    def iterate(memory, obs, dones, s0, d):
        memory.forward(obs, dones, s0)
        memory.backward(d)
        gm.rx.rslx_muon_step(memory.muon, memory.ws)
    eager, inputs = fresh()
    for _ in range(4):
        iterate(eager, *inputs)
    memory, inputs = fresh()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        iterate(memory, *inputs)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        iterate(memory, *inputs)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
    for n in memory.params:
        assert torch.equal(memory.params[n], eager.params[n]), n

"""A policy's memory of linear attention between two layer norms: trained over whole sequences, used step by step.

    z = norm(x W_in),  q, k, v = z W_qkv,  o = linear attention over the episode's steps,  y = norm(o) W_out

The task is recall: the first step of an episode shows a cue of signs, the later ones only noise, and every step has to answer with the cue.
`python examples/linear_memory.py` trains on sequences cut from running episodes (each starts from the state that the last one ended with), then
acts one step at a time and compares.  The projections are torch products; their gradients are written out below.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2509_10771_amd as rx  # noqa: E402

EPS = 1e-5


class LinearMemory:
    """T steps of N environments; `heads` heads of `width` keys and values each, inputs `d_in` wide, answers `d_out`."""

    def __init__(self, T, N, d_in, d_out, heads=4, width=32, dtype=torch.float32, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.N, self.H, self.D, self.dtype = T, N, heads, width, dtype
        M = heads * width
        dev = lambda x: x.float().cuda()  # noqa: E731
        matrix = lambda i, o: dev(torch.randn(i, o, generator=g) / math.sqrt(i))  # noqa: E731
        self.params = dict(w_in=matrix(d_in, M), w_qkv=matrix(M, 3 * M), w_out=matrix(M, d_out), g1=dev(torch.ones(M)), b1=dev(torch.zeros(M)),
                           g2=dev(torch.ones(M)), b2=dev(torch.zeros(M)))
        # memories of about 4 to 250 steps
        self.log_decay = torch.log1p(-torch.exp2(-torch.linspace(2, 8, heads, dtype=torch.float64))).float().cuda()
        self.scale = 1 / math.sqrt(width)
        self.state = torch.zeros(N, heads, width, width, device="cuda")
        # what is kept from call to call: descriptions, statistics, workspaces
        self.one = rx.LinearAttn(dtype, 1, N, heads, width, width, self.log_decay, self.scale)
        like = rx.LinearAttn(dtype, T, N, heads, width, width, self.log_decay, self.scale)
        self.ws = rx.workspace(max(rx.rslx_linear_attention_workspace_bytes(like), rx.rslx_linear_attention_backward_workspace_bytes(like),
                                   rx.rslx_layer_norm_backward_workspace_bytes(T * N, M)))

    def _split(self, qkv, T):
        return [x.unflatten(2, (self.H, self.D)) for x in qkv.view(T, self.N, -1).chunk(3, 2)]

    def _norm(self, x, weight, bias):
        y, mean, rstd = torch.empty_like(x), torch.empty(x.shape[0], device="cuda"), torch.empty(x.shape[0], device="cuda")
        rx.rslx_layer_norm(x, weight, bias, EPS, y, mean, rstd)
        return y, (x, mean, rstd)

    def _norm_backward(self, dy, kept, weight):
        x, mean, rstd = kept
        dx, dw, db = torch.empty_like(x), torch.empty_like(weight), torch.empty_like(weight)
        rx.rslx_layer_norm_backward(dy, x, weight, mean, rstd, dx, dw, db, self.ws)
        return dx, dw, db

    def act(self, obs, reset):
        """One step: obs [N, d_in], reset uint8 [N] (the environments whose last step ended an episode) or None."""
        p = {n: w.to(self.dtype) if w.dim() == 2 else w for n, w in self.params.items()}
        z, _ = self._norm(obs.to(self.dtype) @ p["w_in"], p["g1"], p["b1"])
        q, k, v = self._split(z @ p["w_qkv"], 1)
        o = torch.empty(1, self.N, self.H, self.D, dtype=self.dtype, device="cuda")
        rx.rslx_linear_attention_step(self.one, q, k, v, reset, self.state, self.state, o)
        y, _ = self._norm(o.view(self.N, -1), p["g2"], p["b2"])
        return y @ p["w_out"]

    def forward(self, obs, dones, s0):
        """A whole sequence: obs [T, N, d_in], dones uint8 [T, N], s0 the states before it.  Returns answers [T, N, d_out] and the states behind it."""
        p = {n: w.to(self.dtype) if w.dim() == 2 else w for n, w in self.params.items()}
        x = obs.to(self.dtype).reshape(self.T * self.N, -1)
        z, kept1 = self._norm(x @ p["w_in"], p["g1"], p["b1"])
        q, k, v = self._split(z @ p["w_qkv"], self.T)
        la = rx.LinearAttn(self.dtype, self.T, self.N, self.H, self.D, self.D, self.log_decay, self.scale, dones)
        o = torch.empty(self.T, self.N, self.H, self.D, dtype=self.dtype, device="cuda")
        s_last = torch.empty_like(self.state)
        rx.rslx_linear_attention(la, q, k, v, s0, o, s_last, self.ws)
        y, kept2 = self._norm(o.view(self.T * self.N, -1), p["g2"], p["b2"])
        self.kept = p, x, kept1, z, la, (q, k, v), s0, y, kept2
        return (y @ p["w_out"]).view(self.T, self.N, -1), s_last

    def backward(self, d_answer):
        """Gradients of every parameter, from that of forward()'s answers (the states' start and end are constants)."""
        p, x, kept1, z, la, (q, k, v), s0, y, kept2 = self.kept
        d = d_answer.to(self.dtype).reshape(self.T * self.N, -1)
        grads = dict(w_out=y.t() @ d)
        do, grads["g2"], grads["b2"] = self._norm_backward(d @ p["w_out"].t(), kept2, p["g2"])
        dqkv = torch.empty(self.T * self.N, p["w_qkv"].shape[1], dtype=self.dtype, device="cuda")
        rx.rslx_linear_attention_backward(la, q, k, v, s0, do.view(self.T, self.N, self.H, self.D), None, *self._split(dqkv, self.T), None, self.ws)
        grads["w_qkv"] = z.t() @ dqkv
        dx, grads["g1"], grads["b1"] = self._norm_backward(dqkv @ p["w_qkv"].t(), kept1, p["g1"])
        grads["w_in"] = x.t() @ dx
        return {n: g.float() for n, g in grads.items()}


class Recall:
    """Running episodes: cues of `width` signs, shown in an episode's first step; each step ends one with probability `end_p`."""

    def __init__(self, N, width=4, end_p=0.05, seed=0):
        self.N, self.width, self.end_p = N, width, end_p
        self.g = torch.Generator("cuda").manual_seed(seed)
        self.cue, self.first = self._cues(), torch.ones(N, dtype=torch.bool, device="cuda")

    def _cues(self):
        return torch.randint(0, 2, (self.N, self.width), generator=self.g, device="cuda").float() * 2 - 1

    def step(self):
        """Returns obs [N, width + 1], the answers [N, width] that are right, and whether the step ends its episode (uint8 [N])."""
        noise = 0.1 * torch.randn(self.N, self.width, generator=self.g, device="cuda")
        obs = torch.cat([torch.where(self.first[:, None], self.cue, noise), self.first[:, None].float()], 1)
        answer = self.cue
        done = torch.rand(self.N, generator=self.g, device="cuda") < self.end_p
        self.cue, self.first = torch.where(done[:, None], self._cues(), self.cue), done
        return obs, answer, done.to(torch.uint8)

    def steps(self, T):
        return [torch.stack(x) for x in zip(*(self.step() for _ in range(T)))]


def train(T=32, N=64, iterations=300, dtype=torch.float32, lr=3e-3, seed=0):
    """Returns the memory, its environments and the loss of every iteration."""
    world = Recall(N, seed=seed)
    memory = LinearMemory(T, N, world.width + 1, world.width, dtype=dtype, seed=seed)
    optimizer = torch.optim.Adam(list(memory.params.values()), lr=lr)
    losses = []
    for _ in range(iterations):
        obs, answers, dones = world.steps(T)
        out, state = memory.forward(obs, dones, memory.state)
        error = out.float() - answers
        for name, grad in memory.backward(2 * error / error.numel()).items():
            memory.params[name].grad = grad
        optimizer.step()
        memory.state = state
        losses.append((error ** 2).mean())
    return memory, world, torch.stack(losses).tolist()


def main():
    memory, world, losses = train()
    print("mean squared error: first iteration %.3f, last ten %.3f" % (losses[0], sum(losses[-10:]) / 10))
    right, reset = [], None                                    # the state is already that behind the last step, episode ends included
    for _ in range(100):
        obs, answer, done = world.step()
        right.append((memory.act(obs, reset).sign() == answer).float().mean())
        reset = done
    print("acting: %.1f %% of the signs recalled over 100 steps" % (100 * torch.stack(right).mean().item()))


if __name__ == "__main__":
    main()

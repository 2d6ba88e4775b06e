"""A policy's gated memory between two root-mean-square norms: trained over whole sequences with Muon steps, used step by step.

    e = x W_in,  z = norm(e),  [c, g] = z W_cg,  h = gated recurrence of candidates c and gates g over the episode's steps,
    y = norm(h W_h + e),  answers = y W_out

The task is the recall of examples/linear_memory.py: the first step of an episode shows a cue of signs, and every step has to answer with it.
`python examples/gated_memory.py` trains on sequences cut from running episodes (each starts from the state that the last one ended with), then acts one
step at a time.  The matrices take Muon steps, the norms' weights and the answers' matrix Adam's.  The projections are torch products; their gradients are
written out below.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2509_10771_amd as rx  # noqa: E402
from linear_memory import Recall  # noqa: E402

EPS = 1e-5


class GatedMemory:
    """T steps of N environments; M channels, inputs `d_in` wide, answers `d_out`."""

    def __init__(self, T, N, d_in, d_out, M=128, dtype=torch.float32, lr=0.02, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.N, self.M, self.dtype = T, N, M, dtype
        dev = lambda x: x.float().cuda()  # noqa: E731
        matrix = lambda i, o: dev(torch.randn(i, o, generator=g) / math.sqrt(i))  # noqa: E731
        self.params = dict(w_in=matrix(d_in, M), w_cg=matrix(M, 2 * M), w_h=matrix(M, M), w_out=matrix(M, d_out), n1=dev(torch.ones(M)), n2=dev(torch.ones(M)))
        # gates of about 4 to 250 steps to begin with
        self.bias = torch.log(torch.exp2(torch.linspace(2, 8, M)) - 1).cuda()
        self.state = torch.zeros(N, M, device="cuda")
        # what is kept from call to call: descriptions, gradients, momenta, workspaces
        self.one, like = rx.GatedRec(dtype, 1, N, M), rx.GatedRec(dtype, T, N, M)
        self.muon_names = ("w_in", "w_cg", "w_h")
        self.grads = {n: torch.zeros_like(p) for n, p in self.params.items()}
        momenta = {n: torch.zeros_like(self.params[n]) for n in self.muon_names}
        self.muon = rx.Muon([(self.params[n], self.params[n], self.grads[n], momenta[n], momenta[n], math.sqrt(max(1.0, self.params[n].shape[1] / self.params[n].shape[0])))
                             for n in self.muon_names], lr=lr)
        self.adam = torch.optim.Adam([self.params[n] for n in ("w_out", "n1", "n2")], lr=3e-3)
        self.ws = rx.workspace(max(rx.rslx_gated_recurrence_workspace_bytes(like), rx.rslx_gated_recurrence_backward_workspace_bytes(like),
                                   rx.rslx_rms_norm_backward_workspace_bytes(T * N, M), rx.rslx_muon_step_workspace_bytes(self.muon)))

    def _norm(self, x, residual, weight):
        y, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[0], device="cuda")
        rx.rslx_rms_norm(x, residual, weight, EPS, total, y, rstd)
        return y, (total, rstd)

    def _norm_backward(self, dy, kept, weight, dtotal, dweight):
        total, rstd = kept
        dx = torch.empty_like(total)
        rx.rslx_rms_norm_backward(dy, total, weight, rstd, dtotal, dx, dweight, self.ws)
        return dx

    def _typed(self):
        return {n: w.to(self.dtype) if w.dim() == 2 else w for n, w in self.params.items()}

    def _candidates_and_gates(self, z, p, T):
        cg = (z @ p["w_cg"]).view(T, self.N, 2 * self.M)
        cg[..., self.M:] += self.bias.to(self.dtype)
        return cg[..., :self.M], cg[..., self.M:]

    def act(self, obs, reset):
        """One step: obs [N, d_in], reset uint8 [N] (the environments whose last step ended an episode) or None."""
        p = self._typed()
        e = obs.to(self.dtype) @ p["w_in"]
        z, _ = self._norm(e, None, p["n1"])
        c, g = self._candidates_and_gates(z, p, 1)
        h = torch.empty(1, self.N, self.M, dtype=self.dtype, device="cuda")
        rx.rslx_gated_recurrence_step(self.one, c, g, reset, self.state, self.state, h)
        y, _ = self._norm(h[0] @ p["w_h"], e, p["n2"])
        return y @ p["w_out"]

    def forward(self, obs, dones, s0):
        """A whole sequence: obs [T, N, d_in], dones uint8 [T, N], s0 the states before it.  Returns answers [T, N, d_out] and the states behind it."""
        p, rows = self._typed(), self.T * self.N
        x = obs.to(self.dtype).reshape(rows, -1)
        e = x @ p["w_in"]
        z, kept1 = self._norm(e, None, p["n1"])
        c, g = self._candidates_and_gates(z, p, self.T)
        gr = rx.GatedRec(self.dtype, self.T, self.N, self.M, dones)
        h = torch.empty(self.T, self.N, self.M, dtype=self.dtype, device="cuda")
        s_last = torch.empty_like(self.state)
        rx.rslx_gated_recurrence(gr, c, g, s0, h, s_last, self.ws)
        y, kept2 = self._norm(h.view(rows, -1) @ p["w_h"], e, p["n2"])
        self.kept = p, x, kept1, z, gr, (c, g), s0, h, y, kept2
        return (y @ p["w_out"]).view(self.T, self.N, -1), s_last

    def backward(self, d_answer):
        """Gradients of every parameter, into self.grads, from that of forward()'s answers (the states' start and end are constants)."""
        p, x, kept1, z, gr, (c, g), s0, h, y, kept2 = self.kept
        rows, G = self.T * self.N, self.grads
        d = d_answer.to(self.dtype).reshape(rows, -1)
        G["w_out"].copy_(y.t() @ d)
        d_sum = self._norm_backward(d @ p["w_out"].t(), kept2, p["n2"], None, G["n2"])           # of h W_h and of e
        G["w_h"].copy_(h.view(rows, -1).t() @ d_sum)
        dh = (d_sum @ p["w_h"].t()).view(self.T, self.N, self.M)
        dcg = torch.empty(self.T, self.N, 2 * self.M, dtype=self.dtype, device="cuda")
        rx.rslx_gated_recurrence_backward(gr, c, g, s0, dh, None, dcg[..., :self.M], dcg[..., self.M:], None, self.ws)
        dcg = dcg.view(rows, -1)
        G["w_cg"].copy_(z.t() @ dcg)
        de = self._norm_backward(dcg @ p["w_cg"].t(), kept1, p["n1"], d_sum, G["n1"])
        G["w_in"].copy_(x.t() @ de)
        return G

    def step(self):
        """Muon's step of the matrices, Adam's of the others."""
        rx.rslx_muon_step(self.muon, self.ws)
        for n in ("w_out", "n1", "n2"):
            self.params[n].grad = self.grads[n]
        self.adam.step()


def train(T=32, N=64, iterations=200, dtype=torch.float32, seed=0):
    """Returns the memory, its environments and the loss of every iteration."""
    world = Recall(N, seed=seed)
    memory = GatedMemory(T, N, world.width + 1, world.width, dtype=dtype, seed=seed)
    losses = []
    for _ in range(iterations):
        obs, answers, dones = world.steps(T)
        out, state = memory.forward(obs, dones, memory.state)
        error = out.float() - answers
        memory.backward(2 * error / error.numel())
        memory.step()
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

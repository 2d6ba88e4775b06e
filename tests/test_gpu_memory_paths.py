"""Paths of the operators around a gated memory that sizes choose (test_memory_launches.py holds which sizes choose which): 16-bit and fp32 roll-outs past the
caches, the Muon step's products for several matrices, in tiles and pieces of each kind,
long sequences in pieces of 128 steps and in more than 128 pieces."""
import pytest
import torch

from oracle import muon as om
from sequence_util import U
from test_gpu_gated_recurrence import Case
from test_gpu_memory_large import _recurrence

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


@pytest.mark.parametrize("T,N,D,dtype", [(32, 12288, 256, torch.bfloat16), (32, 12288, 256, torch.float16), (24, 16384, 256, torch.bfloat16),
                                         (24, 8192, 256, torch.float32), (20, 4096, 512, torch.float32)])
def test_a_roll_out_past_the_caches_is_its_environments(rx, T, N, D, dtype):
    """Inputs and outputs of whole, aligned rows go past the caches in these calls, and through them in calls of a few environments: the bits are the same."""
    g = torch.Generator("cuda").manual_seed(T + N)
    xg, dh = torch.randn(T, N, 2 * D, generator=g, device="cuda").to(dtype), torch.randn(T, N, D, generator=g, device="cuda").to(dtype)
    s0 = torch.randn(N, D, generator=g, device="cuda")
    dones = (torch.rand(T, N, generator=g, device="cuda") < 0.02).to(torch.uint8)
    whole = _recurrence(rx, xg, dh, s0, dones)
    for n in (0, 5 * (N // 16) + 3, N - 64):
        part = slice(n, n + 64)
        few = _recurrence(rx, xg[:, part].contiguous(), dh[:, part].contiguous(), s0[part].contiguous(), dones[:, part].contiguous())
        for a, b, time_first in zip(whole, few, (1, 0, 1, 1, 0)):
            assert torch.equal(a[:, part] if time_first else a[part], b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_step_of_many_environments_is_theirs(rx, dtype):
    """A step's row of environments inside a longer buffer: the distance of steps is not used."""
    N, D = 16384, 256
    g = torch.Generator("cuda").manual_seed(9)
    xg = torch.randn(2, N, 2 * D, generator=g, device="cuda").to(dtype)[1:]
    s = torch.randn(N, D, generator=g, device="cuda")
    reset = (torch.rand(N, generator=g, device="cuda") < 0.1).to(torch.uint8)

    def step(xg, s, reset):
        gr = rx.GatedRec(dtype, 1, xg.shape[1], D)
        h, out = torch.empty(1, xg.shape[1], D, dtype=dtype, device="cuda"), torch.empty_like(s)
        rx.rslx_gated_recurrence_step(gr, xg[..., :D], xg[..., D:], reset, s, out, h)
        return h[0], out
    whole = step(xg, s, reset)
    for n in (0, 7777, N - 33):
        part = slice(n, n + 33)
        for a, b in zip(whole, step(xg[:, part].contiguous(), s[part].contiguous(), reset[part].contiguous())):
            assert torch.equal(a[part], b)


def _apart(x, y, ex, ey):
    """|x y| and the error of a product of held operands that are off by ex and ey, entry by entry: 3 K terms are summed in fp32, in whatever order, each addition off
    by a unit (2 u) at most; what the pairs of fp16 leave out is 4 u of a term, and an operand's rest is lost below 2^-37."""
    k = x.shape[1]
    size = x @ y
    off = ex @ (y + ey) + x @ ey + 1.01 * (6 * k + 16) * U * size
    return size, off + 2.0 ** -37 * (x.sum(1, keepdim=True) + y.sum(0, keepdim=True))


def _held(x, off):
    """The error of values that are held as two fp16 numbers after it."""
    return off + 2.0 ** -22 * (x + off) + 2.0 ** -37


def _two_steps(u):
    """X after two steps in fp64, shorter side first, and what each entry may be off by: first order and all higher ones, in absolute values."""
    t = lambda m: m.t().contiguous()  # noqa: E731
    x = u.double() / u.double().norm()
    x = t(x) if x.shape[0] > x.shape[1] else x
    off = _held(x.abs(), 4 * U * x.abs())
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(2):
        a = x @ t(x)
        ea = _apart(x.abs(), t(x).abs(), off, t(off))[1]
        ea = _held(a.abs(), ea)
        square = a @ a
        es = _apart(a.abs(), a.abs(), ea, ea)[1]
        b = om.A * eye + om.B * a + om.C * square
        eb = -om.B * ea + om.C * es + 8 * U * (om.A * eye - om.B * (a.abs() + ea) + om.C * (square.abs() + es))
        off = _apart(b.abs(), x.abs(), _held(b.abs(), eb), off)[1]
        x = b @ x
        off = _held(x.abs(), off)
    return x, off + 4 * U * x.abs()


@pytest.mark.parametrize("shapes", [
    [(1536, 1536), (1530, 1700)],                              # two matrices in three pieces each
    [(1900, 3000), (1600, 2000)],                              # in two
    [(2600, 2600), (2600, 2700)],                              # in one
    [(40, 70), (2000, 4200), (12, 2000), (4200, 40)],          # one in three pieces among others in tiles of 32 x 32
    [(300, 9000), (2700, 2600), (2600, 2600)] + [(480, 500)] * 8,        # two in one piece each, the others in tiles of 64 x 64
    [(100, 130), (1, 1), (333, 777)], [(1000, 1024)] * 3,      # no pieces: tiles of 32 x 32, of 64 x 64
    [(30, 100), (2040, 4090), (300, 200)],                     # a product with X in large tiles beside others in tiles of 32 x 32
    [(2048, 2000), (1900, 600), (2000, 2048)],                 # two beside one in tiles of 64 x 64
], ids=lambda s: "%dx%dx%d" % (len(s), *s[0]))
def test_products_of_several_matrices(rx, shapes):
    """Two steps, every entry within a bound of its own: what belongs to another block, piece or matrix is seen wherever it is."""
    g = torch.Generator("cuda").manual_seed(len(shapes))
    us = [torch.randn(s, generator=g, device="cuda") for s in shapes]
    outs = [torch.full_like(u, float("nan")) for u in us]
    mu = rx.Muon([(None, o, u, None, None, 1.0) for u, o in zip(us, outs)], -1.0, nesterov=False, steps=2)
    rx.rslx_muon_step(mu, rx.workspace(rx.rslx_muon_step_workspace_bytes(mu)))
    for i, (u, o) in enumerate(zip(us, outs)):
        ref, bound = _two_steps(u)
        got = o.double().t() if o.shape[0] > o.shape[1] else o.double()
        rms = ref.square().mean().sqrt().item()
        assert bound.max().item() < 0.3 * rms, (i, u.shape, bound.max().item(), rms)
        off = (got - ref).abs()
        worst = (off / bound).max().item()
        assert torch.isfinite(off).all() and worst <= 1, (i, u.shape, worst)


@pytest.mark.parametrize("T,N,D,dtype,layout,ragged", [
    (4096, 4, 1024, "bf16", "side", False), (2500, 6, 896, "fp32", "dense", True), (3001, 5, 1280, "fp16", "side", True),      # gradients in pieces of 128 steps
    (9000, 2, 64, "fp32", "side", False), (12345, 1, 40, "bf16", "odd", True), (20000, 3, 20, "fp16", "batch_first", True)],   # more than 128 pieces to join
    ids=lambda x: str(x))
def test_long_sequences(rx, T, N, D, dtype, layout, ragged):
    c = Case(T, T, N, D, dtype, done_p=0.0005, ragged=ragged, layout=layout)
    if ragged and N > 2:
        c.lengths[2] = T - 1
    c.check_forward(*c.forward(rx))
    c.check_backward(*c.backward(rx))

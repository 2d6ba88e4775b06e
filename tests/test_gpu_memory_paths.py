"""Paths of the operators around a gated memory that sizes choose (test_memory_launches.py holds which sizes choose which): 16-bit and fp32 roll-outs past the
caches."""
import pytest
import torch

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

"""Rows of linear attention so far apart that a chunk of them has no 32-bit offsets (64 MiB and more from step to step), and sizes at which
registers once came back stale."""
import numpy as np
import pytest
import torch

from oracle import linear_attention as ola
from sequence_util import TYPES, U, Attention, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


class Far(Attention):
    backwards = False

    def place(self, x):
        T, N, H, D = x.shape
        far = (1 << 26) // x.element_size() + 48
        memory = torch.full(((T - 1) * far + N * H * D,), float("nan"), dtype=x.dtype, device="cuda")
        view = memory.as_strided((T, N, H, D), (far, H * D, D, 1))
        view.copy_(x)
        return view


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,N,H,Dk,Dv", [(45, 4, 2, 16, 24), (33, 2, 1, 33, 70), (17, 3, 1, 128, 128)])
def test_far_rows(rx, T, N, H, Dk, Dv, dtype):
    c = Far(T + Dk, T, N, H, Dk, Dv, dtype, done_p=0.1, ragged=True)
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_far_rows_in_pieces(rx, dtype):
    c = Far(7, 130, 2, 1, 20, 40, dtype, done_p=0.02, ragged=True)
    c.on_gpu(rx)
    assert rx.rslx_linear_attention_workspace_bytes(c.la) > 256
    c.check_forward(*c.run_forward(rx))
    c.check_backward(*c.run_backward(rx))


@pytest.mark.parametrize("name", ["q", "k", "v", "do"])
def test_far_rows_that_are_not_finite(rx, name):
    c = Far(9, 40, 2, 2, 12, 20, "fp32", done_p=0.05)
    getattr(c, name)[17, 0, 1, 2] = float("inf")
    c.dones[21, 0] = 1
    more = dict(do=f64(c.do), ds_last=f64(c.ds_last))
    ref = ola.forward(*c.args(), **c.kw()) + ola.backward(*c.args(), **c.kw(), **more)
    for what, r, x in zip(("o", "s_last", "dq", "dk", "dv", "ds0"), ref, c.run_forward(rx) + c.run_backward(rx)):
        x, fine = f64(x), np.isfinite(r)
        assert np.array_equal(np.isfinite(x), fine), what
        # sizes of sums of finite terms: within a few hundred roundings of the largest
        assert np.abs(x[fine] - r[fine]).max() <= c.roundings * U * 40 * max(1.0, np.abs(r[fine]).max()), what


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [17, 18, 31, 33, 47, 64])
def test_gradients_with_episode_ends_at_the_limit_of_registers(rx, T, dtype):
    """Wrong once: registers stored where a branch of some lanes ended, and taken back by all."""
    c = Attention(T * 137 + 40, T, 3, 2, 33, 40, dtype, done_p=0.1, ragged=True)
    c.check_backward(*c.run_backward(rx))

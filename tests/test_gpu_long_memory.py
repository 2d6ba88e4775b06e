"""States that live through many chunks and pieces: what a state is multiplied by must not err the same way every time, nor may what is
added to it.

Few wavefronts are walked in pieces, so cases that are about one walk have more than 1024 sequences.  U = 2^-24 is half a step of fp32.
"""
import numpy as np
import pytest
import torch

from sequence_util import TYPES, U, f64, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


def _last_state(rx, dtype, q, k, v, log_decay, s0=None):
    """The state behind the last step; q, k, v [T, N, H, .] on the GPU."""
    (T, N, H, Dk), Dv = k.shape, v.shape[-1]
    la = rx.LinearAttn(dtype, T, N, H, Dk, Dv, log_decay.cuda(), 1.0)
    o, s = torch.empty(T, N, H, Dv, dtype=dtype, device="cuda"), torch.full((N, H, Dk, Dv), float("nan"), device="cuda")
    need = rx.rslx_linear_attention_workspace_bytes(la)
    rx.rslx_linear_attention(la, q, k, v, s0, o, s, rx.workspace(need))
    return s, need > 256


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_young_state_is_decayed_as_often_as_it_is_old(rx, dtype):
    """One 1 at the last place of chunk c of eight: behind the last chunk it is worth l^(16 (7 - c)) (32 in 16 bits).

    The 1 itself is exact.  Every chunk multiplies it by a neighbour of the chunk's decay, so that the product of any number of them is
    off by one step of fp32 (2 U of a number just above a power of two) at most, and rounds once."""
    chunk, H, N = (16 if dtype == "fp32" else 32), 40, 32
    # chunk decays just above one half: there a step of fp32 is largest beside the number
    log_decay = typed(np.log(0.5 + 0.03 * np.arange(1, H + 1) / H) / chunk, torch.float32)
    T, age = 8 * chunk, 7 - np.arange(N) % 8
    x = torch.zeros(T, N, H, 1, dtype=TYPES[dtype])
    for n in range(N):
        x[chunk * (8 - age[n]) - 1, n] = 1
    x = x.cuda()
    s, pieces = _last_state(rx, TYPES[dtype], x, x, x, log_decay)
    assert not pieces
    ref = np.exp(f64(log_decay)[None] * chunk * age[:, None])
    off = np.abs(f64(s)[:, :, 0, 0] / ref - 1)
    bound = 1.01 * U * (2 + age) * (age > 0)
    assert (off <= bound[:, None]).all(), [(int(a), float(off[age == a].max() / U)) for a in range(8)]


def _long_sum(rx, dtype, T=20000, N=1030, D=64):
    """What the elements of a state are off by, in units of their root mean square, behind T steps of a memory that hardly forgets, in one
    walk."""
    g = np.random.default_rng(5)
    k, v = (typed(g.normal(size=(T, 1, 1, D)), TYPES[dtype]) for _ in range(2))
    log_decay = typed(np.array([-1e-5]), torch.float32)
    one = lambda x: x.cuda().expand(T, N, 1, D)  # noqa: E731
    s, pieces = _last_state(rx, TYPES[dtype], one(k), one(k), one(v), log_decay)
    assert not pieces
    assert torch.equal(s, s[:1].expand_as(s))
    w = np.exp(f64(log_decay) * np.arange(T - 1, -1, -1))
    ref = (f64(k)[:, 0, 0] * w[:, None]).T @ f64(v)[:, 0, 0]
    return (f64(s[0, 0]) - ref) / np.sqrt((ref ** 2).mean())


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_long_sum_is_not_cut_off_in_one_direction(rx, dtype):
    """At most one rounding a step, each at most U of the state and independent of the others: sqrt(T) U of the state's norm in all, and the
    mean over its 4096 elements 64 times less (times 5: five standard deviations)."""
    off = _long_sum(rx, dtype)
    assert np.sqrt((off ** 2).mean()) <= np.sqrt(20000) * U
    assert abs(off.mean()) <= 5 * np.sqrt(20000) * U / 64


@pytest.mark.parametrize("dtype", list(TYPES))
def test_the_mean_of_a_long_sum_is_noise(rx, dtype):
    """Beside what its elements are off by, whatever that is: within five standard errors."""
    off = _long_sum(rx, dtype)
    assert abs(off.mean()) <= 5 * off.std() / 64, off.mean() / (off.std() / 64)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_state_through_many_pieces(rx, dtype):
    """A start state alone through one long sequence, which is walked in pieces of 96 steps (at least 64: one rounding each), and the
    last piece's chunks (at most eight, two steps of fp32 for their decays).  Roundings are independent: the root of their number."""
    T, D = 38400, 64
    tries = np.float32(-np.linspace(1e-5, 2e-4, 20001))
    f = np.exp(96 * tries.astype(np.float64))
    # pieces' decays that lie in the middle between two floats
    worst = tries[np.argsort(np.abs(f.astype(np.float32).astype(np.float64) - f) / f)[-4:]]
    zero = torch.zeros(T, 1, 1, D, dtype=TYPES[dtype], device="cuda")
    s0 = typed(np.random.default_rng(6).normal(size=(1, 1, D, D)), torch.float32)
    for ld in worst:
        log_decay = typed(np.array([ld]), torch.float32)
        s, pieces = _last_state(rx, TYPES[dtype], zero, zero, zero, log_decay, s0.cuda())
        assert pieces
        ref = f64(s0) * np.exp(T * f64(log_decay)[0])
        off = np.linalg.norm(f64(s) - ref) / np.linalg.norm(ref)
        assert off <= (np.sqrt(T / 64) + 4 + 8) * U, off / U


@pytest.mark.parametrize("name", ["k", "v", "do"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [200, 231, 290])
def test_what_is_not_finite_behind_an_odd_or_even_chunk(rx, name, dtype, T):
    """The state's sign turns with every chunk; positions taken one by one start with its own.  In pieces, a wavefront for a tile."""
    import test_gpu_linear_attention as attention
    attention.test_what_is_not_finite_in_16_bits(rx, name, dtype, T, 40, 64)

"""The largest counts of heads: everything that the checks admit can be launched."""
import pytest
import torch

import paper_2509_10771_amd as rx

MOST_HEADS = 1 << 24


def _attn(dtype, N, H, Dk, Dv):
    la = rx.LinearAttn(dtype, 1, N, H, Dk, Dv, torch.zeros(H), 1.0)
    view = lambda at, width: rx.binding._CSeqView(at, 0, H * width, width)  # noqa: E731
    return la, view


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that stand for the GPU's")
@pytest.mark.parametrize("dtype,Dk,Dv", [(torch.float32, 1, 1), (torch.float32, 64, 64), (torch.float32, 128, 8), (torch.bfloat16, 128, 128),
                                         (torch.float16, 33, 100)])
def test_gradients_of_the_most_heads_reach_the_launch(dtype, Dk, Dv):
    la, view = _attn(dtype, MOST_HEADS // 4, 4, Dk, Dv)
    far = lambda i, width: view(1 << 40 | i << 36, width)  # noqa: E731
    a = [far(i, w) for i, w in enumerate((Dk, Dk, Dv, Dv, Dk, Dk, Dv))]
    code = rx.lib.rslx_linear_attention_backward(la.c, a[0], a[1], a[2], None, a[3], None, a[4], a[5], a[6], None, None, 0, None)
    assert code == 4 and b"no ROCm-capable device" in rx.lib.rslx_last_error(), rx.lib.rslx_last_error()


@pytest.mark.gpu
def test_gradients_of_the_most_heads():
    """Three walks a head are more workgroups than a launch takes."""
    N, H = MOST_HEADS // 4, 4
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v, do = (torch.randn(1, N, H, 1, generator=g, device="cuda") for _ in range(4))
    s0 = torch.randn(N, H, 1, 1, generator=g, device="cuda")
    decay = torch.tensor([-0.1, -0.2, -0.3, -3.0], device="cuda")
    la = rx.LinearAttn(torch.float32, 1, N, H, 1, 1, decay, 0.5)
    dq, dk, dv, ds0 = (torch.full_like(x, float("nan")) for x in (q, k, v, s0))
    rx.rslx_linear_attention_backward(la, q, k, v, s0, do, None, dq, dk, dv, ds0, None)
    state = lambda x: x.double()[0, ..., None]  # noqa: E731
    l = decay.double().exp()[:, None, None]
    S = l * s0 + state(k) * state(v)
    dS = 0.5 * state(q) * state(do)
    mag = (l * s0).abs() + (state(k) * state(v)).abs()
    # a product of three factors and the decay, the scale and a sum of two: at most 12 roundings
    for got, ref, size in ((dq, 0.5 * S * state(do), 0.5 * mag * state(do).abs()), (dk, dS * state(v), (dS * state(v)).abs()),
                           (dv, dS * state(k), (dS * state(k)).abs()), (ds0, l * dS, (l * dS).abs())):
        assert ((got.reshape(N, H, 1, 1).double() - ref).abs() <= 12 * 2.0 ** -24 * size).all()


@pytest.mark.gpu
def test_heads_whose_rows_a_workgroup_shares():
    """Keys and values above 64 in 16 bits: a workgroup a head, more of them than a launch takes.  The inputs are one row for all."""
    N, D = MOST_HEADS - 3, 72
    g = torch.Generator("cuda").manual_seed(2)
    q, k, v = (torch.randn(1, 1, 1, D, generator=g, device="cuda").bfloat16() for _ in range(3))
    la = rx.LinearAttn(torch.bfloat16, 1, N, 1, D, D, torch.zeros(1, device="cuda"), 1.0)
    o = torch.full((1, N, 1, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    rx.rslx_linear_attention(la, *(x.expand(1, N, 1, D) for x in (q, k, v)), None, o, None, None)
    ref = (q.double() * k.double()).sum() * v.double()
    size = (q.double() * k.double()).abs().sum() * v.double().abs()
    # the output's rounding; a score of 72 products, in two bf16 parts
    assert ((o[:, :1].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -16 + 80 * 2.0 ** -24) * size).all()
    assert torch.equal(o, o[:, :1].expand_as(o))


@pytest.mark.parametrize("name", ["T", "N", "H", "Dk", "Dv"])
def test_sizes_of_more_than_32_bits(name):
    sizes = dict(T=3, N=2, H=2, Dk=4, Dv=8)
    sizes[name] += 1 << 32
    with pytest.raises(rx.RslxError, match=name + " = .* more than 32 bits"):
        rx.LinearAttn(torch.float32, log_decay=torch.zeros(1).expand(sizes["H"]), **sizes)


def test_columns_of_more_than_32_bits():
    x = torch.empty(2, (1 << 32) + 8, device="meta")           # (no memory behind it)
    r = torch.zeros(2)
    with pytest.raises(rx.RslxError, match="columns are taken"):
        rx.rslx_layer_norm(x, None, None, 1e-5, x, None, None)
    with pytest.raises(rx.RslxError, match="columns are taken"):
        rx.rslx_layer_norm_backward(x, x, None, r, r, x, None, None, None)
    with pytest.raises(rx.RslxError, match="more than 32 bits"):
        rx.rslx_layer_norm_backward_workspace_bytes(2, (1 << 32) + 8)

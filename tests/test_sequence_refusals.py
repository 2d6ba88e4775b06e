"""Arguments that the sequence operators refuse, on the host, before anything is launched."""
import pytest
import torch

import paper_2509_10771_amd as rx


def _attn(T=3, N=2, H=2, Dk=4, Dv=8, dtype=torch.float32, **kw):
    return rx.LinearAttn(dtype, T, N, H, Dk, Dv, torch.zeros(H), 0.5, **kw)


def _forward(la, **kw):
    z = lambda d: torch.zeros(la.T, la.N, la.H, d, dtype=la.dtype)  # noqa: E731
    a = dict(q=z(la.Dk), k=z(la.Dk), v=z(la.Dv), s0=None, o=z(la.Dv), s_last=None, ws=None)
    a.update(kw)
    rx.rslx_linear_attention(la, *(a[n] for n in ("q", "k", "v", "s0", "o", "s_last", "ws")))


def test_attention_shapes_and_types():
    with pytest.raises(rx.RslxError, match="head widths"):
        _forward(_attn(Dk=129))
    with pytest.raises(rx.RslxError, match="head widths"):
        _forward(_attn(Dv=0))
    with pytest.raises(rx.RslxError, match="head widths"):
        rx.rslx_linear_attention_workspace_bytes(_attn(Dk=200))
    with pytest.raises(rx.RslxError, match="not one of"):
        _attn(dtype=torch.float64)
    with pytest.raises(rx.RslxError, match="q is"):
        _forward(_attn(), q=torch.zeros(3, 2, 2, 5))
    with pytest.raises(rx.RslxError, match="v is"):
        _forward(_attn(), v=torch.zeros(3, 2, 2, 8, dtype=torch.bfloat16))
    with pytest.raises(rx.RslxError, match="side by side"):
        _forward(_attn(), k=torch.zeros(3, 2, 4, 2).transpose(2, 3))
    with pytest.raises(rx.RslxError, match="log_decay"):
        rx.LinearAttn(torch.float32, 3, 2, 2, 4, 4, torch.zeros(3))
    with pytest.raises(rx.RslxError, match="dones"):
        _attn(dones=torch.zeros(3, 2))
    with pytest.raises(rx.RslxError, match="lengths"):
        _attn(lengths=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(rx.RslxError, match="s0 has"):
        _forward(_attn(), s0=torch.zeros(2, 2, 4, 4))


def test_attention_pointers():
    la = _attn()
    la.c.log_decay = None
    with pytest.raises(rx.RslxError, match="null log_decay"):
        _forward(la)
    la = _attn()
    la.c.dtype = 7
    with pytest.raises(rx.RslxError, match="unknown dtype"):
        _forward(la)
    la = _attn()
    la.c.T = -1
    assert rx.lib.rslx_linear_attention_workspace_bytes(la.c) == 0 and b"T = -1" in rx.lib.rslx_last_error()
    assert rx.lib.rslx_linear_attention_workspace_bytes(None) == 0
    la = _attn()
    v = la.view("v", torch.zeros(3, 2, 2, 8), 8)
    assert rx.lib.rslx_linear_attention(la.c, None, v, v, None, v, None, None, 0, None) == 1
    assert b"null q" in rx.lib.rslx_last_error()


def test_attention_outputs_that_overlap():
    la = _attn()
    with pytest.raises(rx.RslxError, match="rows of o overlap"):
        _forward(la, o=torch.zeros(3, 2, 1, 8).expand(3, 2, 2, 8))
    s = torch.zeros(64 * 2 + 4)
    with pytest.raises(rx.RslxError, match="s0 and s_last overlap"):
        _forward(la, s0=s[:128], s_last=s[4:132])
    with pytest.raises(rx.RslxError, match="16-byte aligned"):
        _forward(la, s0=s[1:129])
    z = lambda d: torch.zeros(3, 2, 2, d)  # noqa: E731
    with pytest.raises(rx.RslxError, match="ds0 overlaps"):
        rx.rslx_linear_attention_backward(la, z(4), z(4), z(8), None, z(8), s[:128], z(4), z(4), z(8), s[:128], None)
    with pytest.raises(rx.RslxError, match="rows of dk overlap"):
        rx.rslx_linear_attention_backward(la, z(4), z(4), z(8), None, z(8), None, z(4), torch.zeros(1, 2, 2, 4).expand(3, 2, 2, 4), z(8), None, None)


def test_attention_workspace():
    la = _attn(T=2000, N=1, H=1)
    need = rx.rslx_linear_attention_workspace_bytes(la)
    assert need > 256 and rx.rslx_linear_attention_backward_workspace_bytes(la) > need
    with pytest.raises(rx.RslxError, match=r"workspace 1024 < \d+ bytes"):
        _forward(la, ws=torch.zeros(1024, dtype=torch.uint8))
    with pytest.raises(rx.RslxError, match=r"workspace 0 < \d+ bytes"):
        _forward(la)
    assert rx.rslx_linear_attention_workspace_bytes(_attn(T=0)) == 256
    _forward(_attn(N=0))                                       # nothing to do
    _forward(_attn(H=0))


def test_step():
    la = _attn(T=1)
    z = lambda d: torch.zeros(1, 2, 2, d)  # noqa: E731
    with pytest.raises(rx.RslxError, match="null s_out"):
        rx.rslx_linear_attention_step(la, z(4), z(4), z(8), None, None, None, z(8))
    with pytest.raises(rx.RslxError, match="reset has"):
        rx.rslx_linear_attention_step(la, z(4), z(4), z(8), torch.zeros(2), None, torch.zeros(2, 2, 4, 8), z(8))
    s = torch.zeros(132)
    with pytest.raises(rx.RslxError, match="s_in and s_out overlap"):
        rx.rslx_linear_attention_step(la, z(4), z(4), z(8), None, s[:128], s[4:], z(8))
    with pytest.raises(rx.RslxError, match="T = 1"):
        y = lambda d: torch.zeros(3, 2, 2, d)  # noqa: E731
        rx.rslx_linear_attention_step(_attn(), y(4), y(4), y(8), None, None, s[:128], y(8))


def test_layer_norm():
    x = torch.zeros(4, 8)
    with pytest.raises(rx.RslxError, match="columns are taken"):
        rx.rslx_layer_norm(torch.zeros(2, 16385), None, None, 1e-5, torch.zeros(2, 16385), None, None)
    with pytest.raises(rx.RslxError, match="y is"):
        rx.rslx_layer_norm(x, None, None, 1e-5, x.bfloat16(), None, None)
    with pytest.raises(rx.RslxError, match="weight has"):
        rx.rslx_layer_norm(x, torch.ones(4), None, 1e-5, x, None, None)
    with pytest.raises(rx.RslxError, match="weight has"):
        rx.rslx_layer_norm(x, torch.ones(8).double(), None, 1e-5, x, None, None)
    with pytest.raises(rx.RslxError, match="side by side"):
        rx.rslx_layer_norm(torch.zeros(8, 4).t(), None, None, 1e-5, x, None, None)
    with pytest.raises(rx.RslxError, match="rows of y overlap"):
        rx.rslx_layer_norm(x, None, None, 1e-5, torch.zeros(8).expand(4, 8), None, None)
    with pytest.raises(rx.RslxError, match="16-byte aligned"):
        rx.rslx_layer_norm(x, torch.ones(9)[1:], None, 1e-5, x, None, None)
    rx.rslx_layer_norm(torch.zeros(0, 8), None, None, 1e-5, torch.zeros(0, 8), None, None)    # no rows
    r, c = torch.zeros(4), torch.zeros(8)
    with pytest.raises(rx.RslxError, match="null dy, x, mean or rstd"):
        rx.rslx_layer_norm_backward(x, x, None, None, r, x, c, c, None)
    with pytest.raises(rx.RslxError, match="workspace 0 <"):
        rx.rslx_layer_norm_backward(x, x, None, r, r, x, c, None, None)
    with pytest.raises(rx.RslxError, match="rows of 0"):
        rx.rslx_layer_norm_backward_workspace_bytes(4, 0)
    assert rx.lib.rslx_layer_norm(5, None, 8, 4, 8, None, None, 1e-5, None, 8, None, None, None) == 1
    assert rx.lib.rslx_layer_norm(0, None, 8, -4, 8, None, None, 1e-5, None, 8, None, None, None) == 2

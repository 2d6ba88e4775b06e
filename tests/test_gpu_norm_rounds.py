"""Layer norm where a workgroup goes round the rows: the next row's loads run ahead, the sums' LDS is used again, and a row may be written in
place while the next one is on its way.  A forward launch goes round above 2048 sets of rows (a set is up to 16 rows of a wavefront's lanes, or
one row of a workgroup), a backward launch from four sets a workgroup on.

A column's gradient is, for these sizes, a lane's sum of at most eight rows, then of at most 16 sets of lanes, 16 workgroups' sums a lane and
two levels of eight: 56 roundings and the products' own, within the 80 that the bound counts.
"""
import pytest
import torch

from sequence_util import check, f64
from test_gpu_layer_norm import _backward_bounds, _case, _forward_bounds

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -17


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


# every number of lanes a row has: parts of a wavefront, a wavefront, workgroups of 256 to 1024; rows of whole loads and rows that start anywhere
@pytest.mark.parametrize("rows,cols,dtype", [(40000, 64, "fp32"), (33333, 61, "bf16"), (18000, 128, "fp16"), (9001, 240, "fp32"), (8300, 500, "fp32"),
                                             (2100, 1100, "fp32"), (2100, 1101, "fp16"), (2085, 2048, "bf16"), (2070, 4100, "fp32"), (2060, 4099, "fp16"),
                                             (2055, 9000, "bf16"), (1100, 9001, "fp32"), (1030, 12001, "fp16"), (1040, 16384, "fp32")])
def test_rounds(rx, rows, cols, dtype):
    x, dy, w, b = _case(rows + cols, rows, cols, dtype)
    gx, gd, gw, gb = x.cuda(), dy.cuda(), w.cuda(), b.cuda()
    y, mean, rstd = torch.empty_like(gx), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    rx.rslx_layer_norm(gx, gw, gb, EPS, y, mean, rstd)
    ref, bound = _forward_bounds(x, f64(w), f64(b), EPS, x.dtype)
    for name, got, r, t in zip(("y", "mean", "rstd"), (y, mean, rstd), ref, bound):
        check(name, got, r, t)
    z = gx.clone()
    rx.rslx_layer_norm(z, gw, gb, EPS, z, None, None)
    assert torch.equal(y, z)
    dx, dw, db = torch.empty_like(gx), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = rx.workspace(rx.rslx_layer_norm_backward_workspace_bytes(rows, cols))
    rx.rslx_layer_norm_backward(gd, gx, gw, mean, rstd, dx, dw, db, ws)
    ref, bound = _backward_bounds(dy, x, f64(w), mean, rstd, x.dtype)
    for name, got, r, t in zip(("dx", "dweight", "dbias"), (dx, dw, db), ref, bound):
        check(name, got, r, t)
    for which in range(2):
        d, xx, dw2, db2 = gd.clone(), gx.clone(), torch.empty_like(dw), torch.empty_like(db)
        rx.rslx_layer_norm_backward(d, xx, gw, mean, rstd, (d, xx)[which], dw2, db2, ws)
        assert torch.equal((d, xx)[which], dx) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_columns_side_by_side(rx):
    """Input and output are columns of one buffer."""
    x, dy, w, b = _case(3, 9000, 72, "bf16")
    both = torch.full((9000, 144), float("nan"), dtype=x.dtype, device="cuda")
    both[:, :72] = x.cuda()
    rx.rslx_layer_norm(both[:, :72], w.cuda(), b.cuda(), EPS, both[:, 72:], None, None)
    ref, bound = _forward_bounds(x, f64(w), f64(b), EPS, x.dtype)
    check("y", both[:, 72:], ref[0], bound[0])
    assert torch.equal(both[:, :72].cpu(), x)

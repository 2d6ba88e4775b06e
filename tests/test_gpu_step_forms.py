"""One step of linear attention on both sides of the size from which a head is a wavefront's (1024 heads, 2048 of keys above 64) instead of a
workgroup's; counts of heads that leave wavefronts of the last workgroup without one."""
import numpy as np
import pytest
import torch

from oracle import linear_attention as ola
from sequence_util import TYPES, U, Attention, check, f64, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rx():
    import paper_2509_10771_amd as m
    m.rslx_device_check()
    return m


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,H,Dk,Dv", [(341, 3, 20, 36), (1024, 1, 64, 64), (205, 5, 20, 36), (343, 3, 64, 33), (1027, 1, 1, 1), (411, 5, 33, 128),
                                       (682, 3, 100, 65), (683, 3, 100, 65), (1025, 2, 128, 128), (514, 4, 65, 2), (4096, 4, 8, 12)])
def test_forms_of_the_step(rx, N, H, Dk, Dv, dtype):
    for reset_p, has_state, layout in ((0.3, True, "dense"), (0.0, True, "odd"), (0.5, False, "batch_first")):
        c = Attention(N * 7 + Dk, 1, N, H, Dk, Dv, dtype, done_p=reset_p, layout=layout)
        reset, c.dones = c.dones, None
        g, la = c.on_gpu(rx)
        o, s = c.empty(Dv), c.state()
        gpu_reset = None if reset is None else reset.cuda()
        rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], gpu_reset, g["s0"] if has_state else None, s, o)
        args = (f64(c.q)[0], f64(c.k)[0], f64(c.v)[0], f64(c.log_decay), c.scale)
        kw = dict(s_in=f64(c.s0) if has_state else None, reset=None if reset is None else reset[0].numpy())
        ro, rs = ola.step(*args, **kw)
        mo, ms = ola.step(*(np.abs(x) if isinstance(x, np.ndarray) and x.ndim == 3 else x for x in args),
                          **dict(kw, s_in=None if not has_state else np.abs(kw["s_in"])))
        # the decay's two roundings, its product, the outer product's sum; then q's scaling, a product and a sum of Dk
        check("o", o[0], ro, rounding(c.dtype, ro) + (Dk + 12) * U * mo)
        check("s_out", s, rs, 6 * U * ms)
        if has_state:                                          # in place, the same bits
            s2, o2 = g["s0"].clone(), c.empty(Dv)
            rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], gpu_reset, s2, s2, o2)
            assert torch.equal(s, s2) and torch.equal(o, o2)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("N,H,Dk,Dv", [(33, 3, 64, 64), (700, 3, 64, 64), (40, 4, 100, 36), (900, 3, 100, 36), (3, 2, 128, 128)])
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_output_in_place(rx, name, N, H, Dk, Dv, dtype):
    """o where q, k or v lies (the first values of wider rows): the same bits, and nothing beside them."""
    c = Attention(N + Dk, 1, N, H, Dk, Dv, dtype)
    g, la = c.on_gpu(rx)
    want, s = c.empty(Dv), c.state()
    rx.rslx_linear_attention_step(la, g["q"], g["k"], g["v"], None, g["s0"], s, want)
    x = {n: g[n].clone() for n in "qkv"}
    s2 = c.state()
    rx.rslx_linear_attention_step(la, x["q"], x["k"], x["v"], None, g["s0"], s2, x[name][..., :Dv])
    assert torch.equal(x[name][..., :Dv], want) and torch.equal(s, s2)
    assert torch.equal(x[name][..., Dv:], g[name][..., Dv:])
    assert all(torch.equal(x[n], g[n]) for n in "qkv" if n != name)

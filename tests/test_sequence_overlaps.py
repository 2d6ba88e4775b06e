"""Outputs of the sequence operators that share memory with themselves or with inputs are refused on the host, before anything is
launched; layouts that interleave without sharing any are not."""
import pytest
import torch

import paper_2509_10771_amd as rx


def _refused(call, match):
    with pytest.raises(rx.RslxError, match=match):
        call()


def _taken(call):
    """The arguments are taken: without a GPU the launch fails, and nothing else."""
    if torch.cuda.is_available():
        pytest.skip("host tensors are not for a GPU")
    with pytest.raises(rx.RslxError) as e:
        call()
    assert "overlap" not in str(e.value) and "launch" in str(e.value), str(e.value)


def _rows(buf, start, ld, rows, cols):
    return torch.as_strided(buf, (rows, cols), (ld, 1), start)


# start and distance of y's rows beside x's (40 rows of 8, 16 apart): every one shares values with another row of x, or with its own from
# another place
@pytest.mark.parametrize("start,ld", [(0, 8), (0, 24), (0, 32), (0, 20), (16, 16), (1, 16), (4, 20), (-7, 16), (8, 24), (15, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_with_rows_that_overlap(start, ld, dtype):
    buf = torch.zeros(4096, dtype=dtype)
    x, y = _rows(buf, 64, 16, 40, 8), _rows(buf, 64 + start, ld, 40, 8)
    _refused(lambda: rx.rslx_layer_norm(x, None, None, 1e-5, y, None, None), "x and y overlap")
    r, other = torch.zeros(40), torch.zeros(40, 8, dtype=dtype)
    _refused(lambda: rx.rslx_layer_norm_backward(x, other, None, r, r, y, None, None, None), "dx and dy overlap")
    _refused(lambda: rx.rslx_layer_norm_backward(other, x, None, r, r, y, None, None, None), "dx and x overlap")


# the same matrix, columns beside it, rows between its own, buffers of their own
@pytest.mark.parametrize("start,ld", [(0, 16), (8, 16), (8, 32), (8, 48), (-8, 16), (640, 16), (2000, 9)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_with_rows_that_do_not(start, ld, dtype):
    buf = torch.zeros(4096, dtype=dtype)
    x, y = _rows(buf, 64, 16, 40, 8), _rows(buf, 64 + start, ld, 40, 8)
    _taken(lambda: rx.rslx_layer_norm(x, None, None, 1e-5, y, None, None))
    r = torch.zeros(40)
    _taken(lambda: rx.rslx_layer_norm_backward(x, x, None, r, r, y, None, None, None))


def test_norm_of_one_row_in_place_at_any_distance():
    buf = torch.zeros(64)
    _taken(lambda: rx.rslx_layer_norm(_rows(buf, 0, 16, 1, 8), None, None, 1e-5, _rows(buf, 0, 24, 1, 8), None, None))
    _refused(lambda: rx.rslx_layer_norm(_rows(buf, 0, 16, 1, 8), None, None, 1e-5, _rows(buf, 4, 24, 1, 8), None, None), "x and y overlap")


def test_norm_in_place_of_a_row_for_all():
    """x one row read for all of y's: y is written where it lies."""
    buf = torch.zeros(400)
    _refused(lambda: rx.rslx_layer_norm(buf[:8].expand(40, 8), None, None, 1e-5, _rows(buf, 0, 8, 40, 8), None, None), "x and y overlap")
    _taken(lambda: rx.rslx_layer_norm(buf[:8].expand(40, 8), None, None, 1e-5, _rows(buf, 8, 8, 40, 8), None, None))


def test_norm_against_a_count_of_bytes():
    """Any two matrices of one buffer: refused where a byte is in both, and they are not the same rows."""
    import random
    rng, buf, refused = random.Random(1), torch.zeros(4096), 0
    for _ in range(600):
        rows, cols = rng.randint(1, 9), rng.randint(1, 6)
        ld = [rng.choice([0, cols, cols + 1, 2 * cols, 3 * cols + 1, -cols, -2 * cols, rng.randint(-20, 20)]) for _ in range(2)]
        if abs(ld[1]) < cols and rows > 1:
            continue
        at = [1000, 1000 + rng.choice([0, cols, rng.randint(-40, 40)])]
        used = [{at[i] + r * ld[i] + c for r in range(rows) for c in range(cols)} for i in range(2)]
        same = at[0] == at[1] and (rows == 1 or ld[0] == ld[1])
        code = rx.lib.rslx_layer_norm(0, buf.data_ptr() + 4 * at[0], ld[0], rows, cols, None, None, 1e-5, buf.data_ptr() + 4 * at[1], ld[1], None, None,
                                      None) if not torch.cuda.is_available() else pytest.skip("host tensors are not for a GPU")
        want = bool(used[0] & used[1]) and not same
        assert (code == 1) == want, (rows, cols, ld, at, code)
        refused += want
    assert refused > 100


def _attn(T, N, H, width, dtype=torch.float32):
    return rx.LinearAttn(dtype, T, N, H, width, width, torch.zeros(H), 1.0)


def _view(data, strides):
    v = _attn(1, 1, 1, 1).view("x", torch.zeros(1, 1, 1, 1), 1)
    v.data, v.step, v.seq, v.head = data, *strides
    return v


def _output(la, buf, at, strides):
    """Status of a forward call whose o lies at `at` with these strides; inputs elsewhere, one row for all."""
    if torch.cuda.is_available():
        pytest.skip("host tensors are not for a GPU")
    x = torch.zeros(la.Dk)
    same = _view(x.data_ptr(), (0, 0, 0))
    return rx.lib.rslx_linear_attention(la.c, same, same, same, None, _view(buf.data_ptr() + 4 * at, strides), None, None, 0, None)


@pytest.mark.parametrize("strides", [(8, 8, 64), (64, 8, 8), (32, 8, 32), (0, 8, 24), (24, 8, 12), (-8, 8, 64), (24, 8, -24), (1, 24, 300), (30, 15, 8)])
def test_attention_output_that_overlaps_itself(strides):
    la, buf = _attn(3, 3, 4, 8), torch.zeros(4096)
    assert _output(la, buf, 2000, strides) == 2 and b"rows of o overlap" in rx.lib.rslx_last_error()


# dense in every order, backwards, and two distances that fall between each other's multiples
@pytest.mark.parametrize("strides", [(96, 32, 8), (8, 24, 72), (32, 96, 8), (-96, -32, -8), (24, 16, 100), (100, 24, 300)])
def test_attention_output_that_does_not(strides):
    la, buf = _attn(2, 2, 4, 8) if strides[0] == 24 else _attn(3, 3, 4, 8), torch.zeros(4096)
    assert _output(la, buf, 2000, strides) == 4                # no GPU to launch on


def test_attention_output_against_a_count_of_bytes():
    import random
    rng, buf, refused = random.Random(2), torch.zeros(1 << 14), 0
    for _ in range(600):
        T, N, H, width = rng.randint(1, 5), rng.randint(1, 5), rng.randint(1, 5), rng.randint(1, 4)
        order = rng.sample(range(3), 3)
        strides, step = [0] * 3, width
        for i in order:
            strides[i] = rng.choice([1, 1, 1, -1]) * (step if rng.random() < 0.6 else rng.randint(0, 3 * step))
            step = max(1, abs(strides[i])) * (T, N, H)[i]
        rows = [t * strides[0] + n * strides[1] + h * strides[2] for t in range(T) for n in range(N) for h in range(H)]
        want = len({r + i for r in rows for i in range(width)}) < len(rows) * width
        la = _attn(T, N, H, width)
        assert (_output(la, buf, 8192, strides) == 2) == want, (T, N, H, width, strides)
        refused += want
    assert 100 < refused < 500


def _forward(at, T=3, N=2, H=4, D=8):
    """A forward call whose tensors lie at these places of one buffer, the others apart."""
    la, buf, z = _attn(T, N, H, D), torch.zeros(1 << 14), lambda: torch.zeros(T, N, H, D)  # noqa: E731
    dense = lambda x: torch.as_strided(buf, (T, N, H, D), (N * H * D, H * D, D, 1), x)  # noqa: E731
    state = lambda x: None if x is None else buf[x:x + N * H * D * D]  # noqa: E731
    a = {n: dense(at[n]) if n in at else z() for n in "qkvo"}
    return lambda: rx.rslx_linear_attention(la, a["q"], a["k"], a["v"], state(at.get("s0")), a["o"], state(at.get("s_last")), None)


@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("apart", [0, 8, -64, 191, 100])
def test_attention_output_over_an_input(name, apart):
    _refused(_forward({name: 4000, "o": 4000 + apart}), "o overlaps " + name)


def test_attention_states_over_rows():
    _refused(_forward(dict(q=4100, s_last=4000)), "s_last overlaps q")
    _refused(_forward(dict(o=4500, s_last=4000)), "o overlaps s_last")
    _refused(_forward(dict(o=4500, s0=4000)), "o overlaps s0")
    _taken(_forward(dict(q=4000, k=4000, v=4000, o=4192, s0=4384, s_last=4384)))      # (a state has 512 values)
    _taken(_forward(dict(q=4192, k=4180, v=4100, o=4512, s0=4000)))      # inputs may overlap each other


def test_attention_output_between_the_rows_of_an_input():
    la, buf = _attn(5, 2, 3, 8), torch.zeros(4096)
    side = buf[:5 * 2 * 4 * 24].view(5, 2, 96)                 # q, k, v and o of a step side by side
    q, k, v, o = (x.unflatten(2, (3, 8)) for x in side.chunk(4, 2))
    _taken(lambda: rx.rslx_linear_attention(la, q, k, v, None, o, None, None))
    _refused(lambda: rx.rslx_linear_attention(la, q, k, v, None, k, None, None), "o overlaps k")
    back = buf[:5 * 2 * 4 * 24].view(2, 5, 96).transpose(0, 1)[..., 72:].unflatten(2, (3, 8))      # the same memory, sequences first
    _refused(lambda: rx.rslx_linear_attention(la, q, k, back, None, o, None, None), "o overlaps v")


def _backward(at, T=3, N=2, H=4, D=8):
    la, buf, z = _attn(T, N, H, D), torch.zeros(1 << 14), lambda: torch.zeros(T, N, H, D)  # noqa: E731
    dense = lambda x: torch.as_strided(buf, (T, N, H, D), (N * H * D, H * D, D, 1), x)  # noqa: E731
    state = lambda x: None if x is None else buf[x:x + N * H * D * D]  # noqa: E731
    a = {n: dense(at[n]) if n in at else z() for n in ("q", "k", "v", "do", "dq", "dk", "dv")}
    s = {n: state(at.get(n)) for n in ("s0", "ds_last", "ds0")}
    return lambda: rx.rslx_linear_attention_backward(la, a["q"], a["k"], a["v"], s["s0"], a["do"], s["ds_last"], a["dq"], a["dk"], a["dv"], s["ds0"], None)


@pytest.mark.parametrize("out", ["dq", "dk", "dv"])
@pytest.mark.parametrize("other", ["q", "k", "v", "do", "s0", "ds_last", "ds0", "dq", "dk", "dv"])
def test_gradients_over_other_tensors(out, other):
    if out != other:
        _refused(_backward({out: 4040, other: 4000}), "overlaps")
        _taken(_backward({out: 5000, other: 4000}))


def _step(o, N=3, H=4, D=8, s_in=None, s_out=None, **inputs):
    la, z = _attn(1, N, H, D), lambda: torch.zeros(1, N, H, D)  # noqa: E731
    a = {n: inputs.get(n, z()) for n in "qkv"}
    s = torch.zeros(N, H, D, D) if s_out is None else s_out
    return lambda: rx.rslx_linear_attention_step(la, a["q"], a["k"], a["v"], None, s if s_in is None else s_in, s, o)


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_step_in_place_and_over_other_rows(name):
    buf = torch.zeros(4096)
    rows = lambda at, strides: torch.as_strided(buf, (1, 3, 4, 8), (0, *strides, 1), at)  # noqa: E731
    o = rows(2000, (32, 8))
    _taken(_step(o, **{name: o}))
    _taken(_step(o, **{name: rows(2096, (32, 8))}))
    _refused(_step(o, **{name: rows(2008, (32, 8))}), "o overlaps " + name)
    _refused(_step(o, **{name: rows(2000, (0, 8))}), "o overlaps " + name)
    _refused(_step(o, **{name: rows(2000, (8, 24))}), "o overlaps " + name)


def test_step_over_states():
    buf, o = torch.zeros(4096), torch.zeros(1, 3, 4, 8)
    state = buf[:768]
    _refused(_step(buf[400:496].view(1, 3, 4, 8), s_out=state), "s_out overlaps o")
    _refused(_step(o, s_out=state, k=buf[400:496].view(1, 3, 4, 8)), "s_out overlaps k")
    _refused(_step(buf[400:496].view(1, 3, 4, 8), s_in=state), "o overlaps s_in")
    _taken(_step(buf[768:864].view(1, 3, 4, 8), s_out=state))


def test_step_in_place_of_wider_rows():
    """Rows of q that reach into the next head's row of o."""
    buf, la, s = torch.zeros(4096), rx.LinearAttn(torch.float32, 1, 3, 4, 16, 8, torch.zeros(4), 1.0), torch.zeros(3, 4, 16, 8)
    rows = lambda width, head: torch.as_strided(buf, (1, 3, 4, width), (0, 4 * head, head, 1), 0)  # noqa: E731
    k, v = torch.zeros(1, 3, 4, 16), torch.zeros(1, 3, 4, 8)
    _taken(lambda: rx.rslx_linear_attention_step(la, rows(16, 16), k, v, None, s, s, rows(8, 16)))
    _refused(lambda: rx.rslx_linear_attention_step(la, rows(16, 8), k, v, None, s, s, rows(8, 8)), "o overlaps q")

"""The oracles of linear attention and layer norm: closed forms, and gradients against central differences."""
import numpy as np
import pytest

from oracle import layer_norm as ln, linear_attention as la


def _case(seed, T=6, N=3, H=2, Dk=3, Dv=4, done_p=0.3):
    g = np.random.default_rng(seed)
    r = lambda *s: g.normal(size=s)  # noqa: E731
    return dict(q=r(T, N, H, Dk), k=r(T, N, H, Dk), v=r(T, N, H, Dv), log_decay=np.array([-0.05, -0.7])[:H], scale=0.6,
                s0=r(N, H, Dk, Dv), dones=(g.random((T, N)) < done_p).astype(np.uint8), lengths=np.array([T, 0, T - 2], np.int32)[:N])


def test_sums_over_pairs():
    c = _case(1)
    o, s = la.forward(**c)
    T, N, H, _ = c["q"].shape
    for n in range(N):
        for h in range(H):
            for t in range(T):
                want = np.zeros(c["v"].shape[-1])
                if t < c["lengths"][n]:
                    for j in range(t + 1):
                        if not c["dones"][j:t, n].any():
                            want += np.exp(c["log_decay"][h] * (t - j)) * (c["q"][t, n, h] @ c["k"][j, n, h]) * c["v"][j, n, h]
                    if not c["dones"][:t, n].any():
                        want += np.exp(c["log_decay"][h] * (t + 1)) * (c["q"][t, n, h] @ c["s0"][n, h])
                assert np.allclose(o[t, n, h], c["scale"] * want, atol=1e-12)
    assert np.array_equal(s[1], c["s0"][1])                  # no step: the state it started from


def test_two_calls_are_one():
    c = _case(2)
    c["lengths"] = None
    o, s = la.forward(**c)
    cut = lambda a, b: {x: (c[x][a:b] if x in ("q", "k", "v", "dones") else c[x]) for x in c}  # noqa: E731
    o1, s1 = la.forward(**cut(0, 4))
    o2, s2 = la.forward(**dict(cut(4, 6), s0=s1))
    assert np.allclose(np.concatenate([o1, o2]), o, atol=1e-13) and np.allclose(s2, s, atol=1e-13)


def test_steps_are_the_sequence():
    c = _case(3)
    c["lengths"] = None
    o, s = la.forward(**c)
    S = c["s0"]
    for t in range(len(c["q"])):
        reset = None if t == 0 else c["dones"][t - 1]
        ot, S = la.step(c["q"][t], c["k"][t], c["v"][t], c["log_decay"], c["scale"], S, reset)
        assert np.allclose(ot, o[t], atol=1e-13)


@pytest.mark.parametrize("seed", [4, 5])
def test_attention_gradients_are_differences(seed):
    c = _case(seed, T=5)
    g = np.random.default_rng(seed + 100)
    do, ds = g.normal(size=c["v"].shape), g.normal(size=c["s0"].shape)

    def loss(**kw):
        o, s = la.forward(**dict(c, **kw))
        return (o * do).sum() + (s * ds).sum()

    got = dict(zip(("q", "k", "v", "s0"), la.backward(do=do, ds_last=ds, **c)))
    eps = 1e-6
    for name, grad in got.items():
        assert grad.shape == c[name].shape
        for i in [tuple(g.integers(0, m) for m in grad.shape) for _ in range(25)]:
            up, down = c[name].copy(), c[name].copy()
            up[i] += eps
            down[i] -= eps
            want = (loss(**{name: up}) - loss(**{name: down})) / (2 * eps)
            assert abs(want - grad[i]) < 1e-7 * max(1.0, abs(want)), (name, i)


def test_what_is_not_finite_stays_in_its_episode():
    c = _case(6, done_p=0.0)
    c["lengths"] = None
    c["dones"][3, 0] = 1
    c["v"][2, 0, 0, 1] = np.inf
    o, _ = la.forward(**c)
    assert np.isfinite(o[:2]).all() and np.isfinite(o[4:]).all() and np.isfinite(o[:, 1:]).all() and np.isfinite(o[:, 0, 1]).all()
    assert not np.isfinite(o[2:4, 0, 0, 1]).any() and np.isfinite(o[2:4, 0, 0, [0, 2, 3]]).all()


def test_layer_norm_gradients_are_differences():
    g = np.random.default_rng(7)
    x, w, b, dy = g.normal(2, 1, (4, 9)), g.normal(size=9), g.normal(size=9), g.normal(size=(4, 9))
    y, m, r = ln.forward(x, w, b)
    assert np.allclose(((y - b) / w).mean(1), 0, atol=1e-12) and np.allclose(((y - b) / w).var(1), 1, atol=1e-4)
    dx, dw, db = ln.backward(dy, x, w, m, r)
    loss = lambda x=x, w=w, b=b: (ln.forward(x, w, b)[0] * dy).sum()  # noqa: E731
    eps = 1e-6
    for name, at, grad in (("x", x, dx), ("w", w, dw), ("b", b, db)):
        for i in np.ndindex(*at.shape):
            up, down = at.copy(), at.copy()
            up[i] += eps
            down[i] -= eps
            assert abs((loss(**{name: up}) - loss(**{name: down})) / (2 * eps) - grad[i]) < 1e-7

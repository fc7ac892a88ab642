"""The oracle of the inner step's operators against differences, closed forms and brute force (CPU only)."""
import numpy as np
import pytest

from oracle import inner as O


def _difference(f, x, weight, eps=1e-6):
    """Gradient of sum(weight * f(x)) by central differences."""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + eps
        hi = (weight * f()).sum()
        x[i] = keep - eps
        lo = (weight * f()).sum()
        x[i] = keep
        g[i] = (hi - lo) / (2 * eps)
    return g


@pytest.mark.parametrize("lens,hq,hk,d", [((4, 1, 0, 3), 4, 2, 3), ((5,), 1, 1, 2), ((2, 3), 3, 1, 4)])
def test_attention_gradient_against_differences(lens, hq, hk, d):
    rng = np.random.default_rng(0)
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    q, k, v, do = (rng.normal(size=(T, h, d)) for h in (hq, hk, hk, hq))
    g, _ = O.attention_grad(q, k, v, do, cu, 0.7)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        np.testing.assert_allclose(g[name], _difference(lambda: O.attention(q, k, v, cu, 0.7)[0], t, do), rtol=1e-6, atol=1e-8)


def test_attention_closed_forms():
    rng = np.random.default_rng(1)
    cu = [0, 1, 4]
    q, k, v = rng.normal(size=(4, 2, 3)), rng.normal(size=(4, 1, 3)), rng.normal(size=(4, 1, 3))
    o, lse, _ = O.attention(q, k, v, cu, 0.5)
    for first in (0, 1):      # the first token of a sequence attends to itself alone
        np.testing.assert_allclose(o[first], np.broadcast_to(v[first], (2, 3)))
        np.testing.assert_allclose(lse[:, first], 0.5 * (q[first] @ k[first, 0]))
    o0, lse0, _ = O.attention(0 * q, k, v, cu, 0.5)      # equal scores: the running mean
    np.testing.assert_allclose(o0[3, 0], v[1:4, 0].mean(0))
    np.testing.assert_allclose(lse0[:, 3], np.log(3.0))


@pytest.mark.parametrize("gate_kind", [None, "channel", "element"])
@pytest.mark.parametrize("post", [True, False])
def test_block_norm_gradient_against_differences(gate_kind, post):
    rng = np.random.default_rng(2)
    K, R, H, eps, s = 2, 3, 5, 1e-3, 0.4
    x, y = rng.normal(size=(K * R, H)), rng.normal(size=(K * R, H))
    wa, wb = (rng.normal(size=(K, H)) if post else None), rng.normal(size=(K, H))
    gate = None if gate_kind is None else rng.normal(size=(K, H) if gate_kind == "channel" else (K * R, H))
    dn, dres = rng.normal(size=x.shape), rng.normal(size=x.shape)
    xn, _ = O.block_norm(x, y, gate, gate_kind, wa, wb, K, eps, s)
    g, _ = O.block_norm_grad(dn, dres, xn, y, gate, gate_kind, wa, wb, K, eps, s)
    both = np.stack([dres, dn])
    f = lambda: np.stack(O.block_norm(x, y, gate, gate_kind, wa, wb, K, eps, s))  # noqa: E731
    for name, t in (("dx", x), ("dy", y), ("dgate", gate), ("dw_post", wa), ("dw_pre", wb)):
        if t is not None:
            np.testing.assert_allclose(g[name], _difference(f, t, both), rtol=2e-6, atol=1e-7, err_msg=name)
        else:
            assert name not in g


def test_swiglu_gradient_against_differences():
    rng = np.random.default_rng(3)
    g, u, dh = rng.normal(0, 3, size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    dg, du = O.swiglu_grad(dh, g, u)
    np.testing.assert_allclose(dg, _difference(lambda: O.swiglu(g, u), g, dh), rtol=1e-6, atol=1e-8)
    np.testing.assert_allclose(du, _difference(lambda: O.swiglu(g, u), u, dh), rtol=1e-6, atol=1e-8)


def test_save8_by_hand():
    x = np.zeros((2, 40))
    x[0, :4] = [1.0, -0.5, 0.0078125, 0.3]           # largest 1.0: step 2^-6
    x[0, 32:34] = [-127.0, 126.4]                    # largest 127: step 1
    x[1, 32] = np.inf
    q, e = O.save8(x)
    assert e.tolist() == [[127 - 6, 127], [1, 255]]
    assert q[0, :4].tolist() == [64, -32, 0, 19]     # 0.0078125 * 64 = 0.5 rounds to even
    assert q[0, 32:34].tolist() == [-127, 126]
    back = O.load8(q, e)
    assert back[0, :3].tolist() == [1.0, -0.5, 0.0] and np.isnan(back[1, 32:]).all() and (back[1, :32] == 0).all()


def test_save8_error_bound():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(50, 64)).astype(np.float32) * np.exp(rng.normal(0, 8, size=(50, 1))).astype(np.float32)
    back = O.load8(*O.save8(x))
    top = np.repeat(np.abs(x).reshape(50, 2, 32).max(2), 32, axis=1)
    assert (np.abs(back - x) <= top / 64 * (1 + 1e-12)).all()                 # a step is at most 1/64 of the largest magnitude
    assert np.mean(np.abs(back - x) <= top / 128 * (1 + 1e-12)) > 0.99        # and only a value above 127 steps is more than half a step off

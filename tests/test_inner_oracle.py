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


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot,normed", [(6, 6, True), (7, 4, True), (8, 4, False)])
def test_head_rope_gradient_against_differences(d, rot, normed, interleaved):
    rng = np.random.default_rng(2)
    T, K = 4, 2
    x, dy, w = rng.normal(size=(T, 3, d)), rng.normal(size=(T, 3, d)), 1 + 0.3 * rng.normal(size=(K, d))
    angle = rng.normal(size=(T, rot // 2))
    f = lambda: O.head_rope(x, w if normed else None, np.cos(angle), np.sin(angle), K, interleaved, 1e-3)[0]  # noqa: E731
    dx, dw, _, _ = O.head_rope_grad(dy, x, w if normed else None, np.cos(angle), np.sin(angle), K, interleaved, 1e-3)
    np.testing.assert_allclose(dx, _difference(f, x, dy), rtol=1e-6, atol=1e-8)
    if normed:
        np.testing.assert_allclose(dw, _difference(f, w, dy), rtol=1e-6, atol=1e-8)


def test_head_rope_closed_forms():
    """A quarter turn; lengths are kept; the norm's heads have root mean square 1."""
    x = np.arange(1.0, 7.0).reshape(1, 1, 6)
    quarter = (np.zeros((1, 2)), np.ones((1, 2)))
    np.testing.assert_array_equal(O.head_rope(x, None, *quarter, 1, False, 0.0)[0].ravel(), [-3, -4, 1, 2, 5, 6])
    np.testing.assert_array_equal(O.head_rope(x, None, *quarter, 1, True, 0.0)[0].ravel(), [-2, 1, -4, 3, 5, 6])
    angle = np.array([[0.3, 1.1, 2.0]])
    y, _ = O.head_rope(x, np.ones((1, 6)), np.cos(angle), np.sin(angle), 1, False, 0.0)
    assert abs((y ** 2).mean() - 1.0) < 1e-12


def test_embed_gradient_is_the_transpose():
    rng = np.random.default_rng(3)
    tokens, table, dout = rng.integers(-2, 9, (2, 20)), rng.normal(size=(2, 7, 3)), rng.normal(size=(40, 3))
    out = O.embed(tokens, table, 0.5)
    assert np.isnan(out[(tokens >= 7).ravel()]).all() and (out[(tokens < 0).ravel()] == 0).all()
    inside = (tokens < 7).ravel()
    g, _, n = O.embed_grad(tokens, dout, 7, 0.5)
    np.testing.assert_allclose((out[inside] * dout[inside]).sum(), (g * table).sum())
    assert n.sum() == ((tokens >= 0) & (tokens < 7)).sum()


def test_philox_known_answers():
    """The published test vectors of Philox4x32 with seven and ten rounds: all zeros, all ones, digits of pi."""
    zeros, ones, pi = [0] * 6, [0xFFFFFFFF] * 6, [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344, 0xA4093822, 0x299F31D0]
    for rounds, words, want in ((7, zeros, "5f6fb709 0d893f64 4f121f81 4f730a48"), (10, zeros, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
                                (10, ones, "408f276d 41c83b0e a20bc7c6 6d5451fd"), (10, pi, "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert [int(w) for w in O.philox4x32(words[:4], words[4:], rounds)] == [int(w, 16) for w in want.split()]


def test_dropout_mask_rate_and_words():
    keeps = O.dropout_keeps(300, 203, 0.25, 7, 1 << 40)
    assert abs(keeps.mean() - 0.75) < 5 * (0.25 * 0.75 / keeps.size) ** 0.5
    word = O.philox4x32((50, 9, 0, 1 << 8), (7, 0), 7)[2]
    assert keeps[9, 202] == (word >= 2 ** 30)

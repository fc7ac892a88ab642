"""Head norms with rotation, embeddings and dropout on the GPU against the float64 oracle, and their manners (streams, graphs, strides,
untouched memory).

Tolerances as in test_gpu_inner_ops: u, the unit roundoff of the activations' type, for a result that is rounded once from fp32, and a multiple of
2^-24 of the sum of the terms' magnitudes for the fp32 arithmetic before it.
"""
import numpy as np
import pytest

from oracle import inner as O
from tests.test_gpu_inner_ops import F32, TINY, U, _dt, _layout, _near, _np, _randn, _torch, _untouched

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------- head norms and rotation
def _tables(N, rot, seed=0, pad=0):
    """cos and sin of N positions, as a user makes them; with `pad` columns of another tensor behind every row."""
    torch = _torch()
    angle = (torch.arange(N, dtype=torch.float64) + seed)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    out = []
    for t in (angle.cos(), angle.sin()):
        full = torch.full((N, rot // 2 + pad), 9.0, device="cuda")
        full[:, :rot // 2] = t.float().cuda()
        out.append(full[:, :rot // 2])
    return out


def _rope_case(K, rows, hq, hk, d, rot, inter, norm, dtype, layout="plain", positions="i64", N=50, pad=0, eps=1e-5, seed=0):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T = K * rows
    u, tiny = U[dtype], TINY[dtype]
    if positions == "none":
        N = T
    cos, sin = _tables(N, rot, pad=pad)
    gen = torch.Generator().manual_seed(seed)
    pos = None if positions == "none" else torch.randint(N, (T,), generator=gen).to({"i64": torch.int64, "i32": torch.int32}[positions]).cuda()
    at = np.arange(T) if pos is None else pos.cpu().numpy()
    theta = torch.full((K, 2 * d + 5), 5.0, device="cuda")            # the weights are column ranges of a matrix
    theta[:, :2 * d] = 1.0 + _randn((K, 2 * d), "f32", seed + 1, 0.2)
    grads = torch.full_like(theta, 5.0)
    w = {"q": theta[:, :d] if "q" in norm else None, "k": theta[:, d:2 * d] if "k" in norm else None}
    dw = {"q": grads[:, :d] if "q" in norm else None, "k": grads[:, d:2 * d] if "k" in norm else None}
    h = {"q": hq, "k": hk}
    x, y, dy, dx = {}, {}, {}, {}
    for i, n in enumerate("qk"):
        if h[n] == 0:
            x[n] = y[n] = dy[n] = dx[n] = (None, None)
            continue
        x[n] = _layout(T, h[n], d, dtype, layout, fill=_randn((T, h[n], d), dtype, seed + 2 + i, 1.5))
        dy[n] = _layout(T, h[n], d, dtype, layout, fill=_randn((T, h[n], d), dtype, seed + 4 + i))
        y[n], dx[n] = _layout(T, h[n], d, dtype, layout), _layout(T, h[n], d, dtype, layout)

    def forward(q_out, k_out, q=x["q"][0], k=x["k"][0]):
        fgd.fgd_qk_rope_forward(q, k, w["q"], w["k"], cos, sin, pos, q_out, k_out, eps, inter)

    def backward(dq, dk, dq_out=dy["q"][0], dk_out=dy["k"][0]):
        fgd.fgd_qk_rope_backward(dq_out, dk_out, x["q"][0] if "q" in norm else None, x["k"][0] if "k" in norm else None, w["q"], w["k"], cos, sin, pos,
                                 dq, dk, dw["q"], dw["k"], eps, inter)

    forward(y["q"][0], y["k"][0])
    backward(dx["q"][0], dx["k"][0])
    fp = F32 * (d / 2 + 16)                            # the sum of d squares, a reciprocal root of 2^-22, a few products
    for n in "qk":
        if h[n] == 0:
            continue
        ref, mag = O.head_rope(_np(x[n][0]), _np(w[n]), _np(cos)[at], _np(sin)[at], K, inter, eps)
        _near(y[n][0], ref, u * np.abs(ref) + fp * mag + tiny, n + "_out")
        ref, ref_w, mag, mag_w = O.head_rope_grad(_np(dy[n][0]), _np(x[n][0]), _np(w[n]), _np(cos)[at], _np(sin)[at], K, inter, eps)
        _near(dx[n][0], ref, u * np.abs(ref) + 4 * fp * mag + tiny, "d" + n)
        if ref_w is not None:
            _near(dw[n], ref_w, (fp + F32 * rows * h[n]) * mag_w, "dw_" + n)
        if layout != "plain":
            _untouched(*y[n], n + "_out")
            _untouched(*dx[n], "d" + n)
    assert bool((grads[:, 2 * d:] == 5.0).all()), "columns beside the gradients were written"
    keep = {n: (y[n][0].clone(), dx[n][0].clone(), dw[n].clone() if dw[n] is not None else None) for n in "qk" if h[n]}
    backward(dx["q"][0], dx["k"][0])
    for n in keep:
        assert torch.equal(dx[n][0], keep[n][1]) and (dw[n] is None or torch.equal(dw[n], keep[n][2])), f"gradients of {n} differ from run to run"
    forward(x["q"][0], x["k"][0])                      # in place
    backward(dy["q"][0], dy["k"][0]) if not norm else None
    for n in keep:
        assert torch.equal(x[n][0], keep[n][0]), f"{n} in place"
        assert norm or torch.equal(dy[n][0], keep[n][1]), f"d{n} in place"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("norm", ["qk", ""])
@pytest.mark.parametrize("K,rows,hq,hk,d,rot,inter", [
    (1, 1, 1, 1, 64, 64, False), (1, 1, 4, 2, 128, 128, True), (2, 37, 4, 2, 64, 64, False), (1, 131, 6, 2, 80, 48, True), (3, 5, 5, 1, 96, 96, False),
    (1, 66, 3, 3, 72, 72, False), (8, 9, 16, 4, 128, 128, False), (1, 20, 8, 8, 32, 16, False), (1, 19, 2, 1, 256, 256, True), (1, 23, 7, 1, 192, 64, False),
    (2, 11, 2, 2, 2, 2, False), (1, 17, 3, 1, 65, 64, True), (1, 9, 2, 1, 255, 128, False), (1, 13, 1, 1, 7, 4, False), (1, 8, 2, 1, 12, 6, True),
    (1, 300, 20, 1, 16, 16, False), (2, 2, 3, 2, 250, 250, True), (4, 300, 6, 3, 112, 112, False)])
def test_rope(K, rows, hq, hk, d, rot, inter, norm, dtype):
    _rope_case(K, rows, hq, hk, d, rot, inter, norm, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["fused", "head_major", "odd"])
@pytest.mark.parametrize("inter", [False, True])
def test_rope_layouts(layout, inter, dtype):
    _rope_case(2, 21, 4, 2, 64, 32, inter, "qk", dtype, layout)


@pytest.mark.parametrize("norm,hk", [("q", 2), ("k", 2), ("q", 0), ("", 0)])
@pytest.mark.parametrize("positions", ["none", "i32"])
def test_rope_parts(norm, hk, positions):
    _rope_case(2, 30, 4, hk, 64, 64, False, norm, "bf16", positions=positions)


@pytest.mark.parametrize("layout", ["plain", "fused", "head_major", "odd"])
@pytest.mark.parametrize("K,rows,hq,hk,d,rot,inter,norm,dtype", [
    (2, 37, 4, 2, 64, 64, False, "qk", "bf16"), (1, 9001, 6, 2, 128, 128, False, "qk", "bf16"), (1, 5003, 6, 2, 80, 48, True, "qk", "f32"), (3, 3001, 6, 2, 40, 40, False, "qk", "f16"),
    (1, 301, 3, 1, 66, 66, False, "qk", "bf16"), (1, 1, 16, 4, 128, 128, True, "qk", "f32"), (2, 700, 4, 4, 72, 72, True, "q", "bf16"), (2, 700, 4, 4, 255, 128, False, "k", "f16")])
def test_rope_gradients_in_place_of_what_they_come_from(K, rows, hq, hk, d, rot, inter, norm, dtype, layout):
    """dq may be dq_out and dk dk_out with weights, too: the same bits as beside one another."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T = K * rows
    cos, sin = _tables(300, rot)
    pos = (torch.arange(T, device="cuda") * 7 + 3) % 300
    w = {n: 1.0 + _randn((K, d), "f32", i, 0.2) if n in norm else None for i, n in enumerate("qk")}
    x, dy, dx = ({n: _layout(T, h, d, dtype, layout, fill=_randn((T, h, d), dtype, seed + h)) for n, h in (("q", hq), ("k", hk))} for seed in (10, 50, 90))

    def run(dq, dk):
        dw = {n: None if w[n] is None else torch.empty_like(w[n]) for n in "qk"}
        fgd.fgd_qk_rope_backward(dy["q"][0], dy["k"][0], x["q"][0], x["k"][0], w["q"], w["k"], cos, sin, pos, dq, dk, dw["q"], dw["k"], 1e-5, inter)
        return [t for t in dw.values() if t is not None]

    apart = run(dx["q"][0], dx["k"][0])
    inside = run(dy["q"][0], dy["k"][0])
    assert all(torch.equal(a, b) for a, b in zip(apart, inside))
    for n in "qk":
        assert torch.equal(dx[n][0], dy[n][0]), "d" + n
        if layout != "plain":
            _untouched(*dy[n], "d" + n)


@pytest.mark.parametrize("pad", [1, 4])
def test_rope_table_strides(pad):
    _rope_case(1, 40, 4, 2, 128, 128, False, "qk", "bf16", pad=pad)


@pytest.mark.parametrize("norm", ["qk", ""])
def test_rope_many_tokens(norm):
    """More tokens than one walk of the grid."""
    _rope_case(2, 9001, 3, 1, 64, 64, False, norm, "bf16", N=4000)


@pytest.mark.parametrize("K,rows,hq,hk,d,rot,inter,norm,dtype", [
    (2, 6001, 2, 1, 72, 72, False, "qk", "bf16"), (1, 12002, 2, 1, 72, 40, True, "q", "f16"), (1, 12001, 2, 1, 72, 72, True, "", "bf16"), (3, 3001, 6, 2, 40, 40, False, "qk", "bf16"),
    (1, 30001, 2, 2, 24, 16, True, "qk", "f16"), (1, 9000, 16, 4, 80, 80, False, "qk", "bf16"), (2, 4501, 4, 4, 96, 96, True, "qk", "bf16"), (1, 5003, 6, 2, 80, 48, True, "qk", "f32"),
    (5, 1001, 6, 0, 80, 80, False, "q", "f32"), (1, 9001, 4, 4, 96, 48, False, "k", "f16")])
def test_rope_many_tokens_of_heads_of_any_number_of_lanes(K, rows, hq, hk, d, rot, inter, norm, dtype):
    """As many lanes to a head as it has chunks, three to six heads to a warp: taken where there are more tokens than the GPU's warps."""
    _rope_case(K, rows, hq, hk, d, rot, inter, norm, dtype, "fused" if K == 1 else "plain", N=300)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rotation_alone_is_the_plain_one_to_the_bit(dtype):
    """Without weights: the results and gradients of the rotation written out in fp32."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, d = 333, 64
    q, k, gq, gk = (_randn((T, h, d), dtype, i) for i, h in enumerate((4, 2, 4, 2)))
    cos, sin = _tables(T, d)
    c, s = cos[:, None], sin[:, None]

    def plain(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat((a * c - b * s, b * c + a * s), -1).to(x.dtype)

    got, want = [torch.empty_like(t) for t in (q, k)], [plain(t) for t in (q, k)]
    fgd.fgd_qk_rope_forward(q, k, None, None, cos, sin, None, *got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for t, g in ((q, gq), (k, gk)):
        t.requires_grad_(True)
        plain(t).backward(g)
    fgd.fgd_qk_rope_backward(gq, gk, None, None, None, None, cos, sin, None, *got, None, None)
    assert torch.equal(got[0], q.grad) and torch.equal(got[1], k.grad)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 10)])
def test_rope_positions_outside_the_tables(dtype, d):
    """Their tokens become NaN, all channels of them, nothing else does; without weights the gradients likewise."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, N = 40, 16
    rot = d // 4 * 2
    q, k = _randn((T, 3, d), dtype, 0), _randn((T, 1, d), dtype, 1)
    cos, sin = _tables(N, rot)
    pos = torch.arange(T, device="cuda") % N
    bad = {3: -1, 17: N, 18: 2 ** 40, 39: -2 ** 62}
    for t, p in bad.items():
        pos[t] = p
    inside = torch.tensor([t not in bad for t in range(T)]).cuda()
    w = 1.0 + _randn((1, d), "f32", 2, 0.1)
    for wq in (w, None):
        yq, yk = torch.empty_like(q), torch.empty_like(k)
        fgd.fgd_qk_rope_forward(q, k, wq, wq, cos, sin, pos, yq, yk)
        good_q, good_k = torch.empty_like(q), torch.empty_like(k)
        fgd.fgd_qk_rope_forward(q, k, wq, wq, cos, sin, torch.where(inside, pos, 0), good_q, good_k)
        for y, g in ((yq, good_q), (yk, good_k)):
            assert bool(y[~inside].isnan().all()) and torch.equal(y[inside], g[inside])
        dq, dk, dw = torch.empty_like(q), torch.empty_like(k), [None if wq is None else torch.zeros_like(w) for _ in range(2)]
        fgd.fgd_qk_rope_backward(yq.nan_to_num(0.5), yk.nan_to_num(0.5), q, k, wq, wq, cos, sin, pos, dq, dk, *dw)
        assert bool(dq[~inside].isnan().all()) and not bool(dq[inside].isnan().any())
        assert wq is None or all(bool(t.isnan().all()) for t in dw)


def test_rope_channels_that_pass_do_not_see_each_other():
    """An infinity in one of the channels beyond the rotation stays where it is."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q = _randn((5, 2, 64), "bf16", 0)
    q[2, 1, 40], q[3, 0, 63] = float("inf"), float("nan")
    cos, sin = _tables(5, 32)
    y = torch.empty_like(q)
    fgd.fgd_qk_rope_forward(q, None, None, None, cos, sin, None, y, None)
    assert torch.equal(y[..., 32:].nan_to_num(7.0, posinf=9.0), q[..., 32:].nan_to_num(7.0, posinf=9.0)) and bool(y[..., :32].isfinite().all())


def test_rope_no_tokens():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q, k, w, dw = _randn((0, 2, 64), "bf16", 0), _randn((0, 1, 64), "bf16", 0), torch.ones((2, 64), device="cuda"), [torch.full((2, 64), 5.0, device="cuda") for _ in range(2)]
    cos, sin = _tables(3, 64)
    fgd.fgd_qk_rope_forward(q, k, w, w, cos, sin, None, torch.empty_like(q), torch.empty_like(k))
    fgd.fgd_qk_rope_backward(q, k, q, k, w, w, cos, sin, None, torch.empty_like(q), torch.empty_like(k), *dw)
    assert all(bool((t == 0).all()) for t in dw)


def test_rope_gradient_against_differences():
    """Directional derivatives of the kernel's own forward pass, in fp32."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, K, d = 12, 2, 24
    q, k, w = _randn((T, 3, d), "f32", 0), _randn((T, 2, d), "f32", 1), 1.0 + _randn((K, 2 * d), "f32", 2, 0.2)
    gq, gk = _randn((T, 3, d), "f32", 3), _randn((T, 2, d), "f32", 4)
    cos, sin = _tables(T, 16)

    def loss(q, k, w):
        yq, yk = torch.empty_like(q), torch.empty_like(k)
        fgd.fgd_qk_rope_forward(q, k, w[:, :d], w[:, d:], cos, sin, None, yq, yk)
        return float((yq.double() * gq).sum() + (yk.double() * gk).sum())

    dq, dk, dw = torch.empty_like(q), torch.empty_like(k), torch.empty_like(w)
    fgd.fgd_qk_rope_backward(gq, gk, q, k, w[:, :d], w[:, d:], cos, sin, None, dq, dk, dw[:, :d], dw[:, d:])
    h = 2.0 ** -6
    for i, (t, g) in enumerate(((q, dq), (k, dk), (w, dw))):
        v = _randn(tuple(t.shape), "f32", 9)
        v = v / v.norm()
        at = [q, k, w]
        diff = []
        for s in (h, -h):
            moved = list(at)
            moved[i] = t + s * v
            diff.append(loss(*moved))
        got, want = (diff[0] - diff[1]) / (2 * h), float((g.double() * v).sum())
        # the third derivative along a unit step (below 8 |g|), and fp32's 2^-22 of the terms' magnitudes over the step
        bound = float(gq.norm() + gk.norm()) * (8 * h * h + 2.0 ** -22 * 8 / h)
        assert abs(got - want) <= bound, f"argument {i}: {got} against {want} (bound {bound})"


def test_rope_refuses_a_small_workspace():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q, w = _randn((8, 2, 64), "bf16", 0), torch.ones((1, 64), device="cuda")
    cos, sin = _tables(8, 64)
    small = torch.empty(fgd.fgd_qk_rope_workspace(1, 64) - 4, dtype=torch.uint8, device="cuda")
    with pytest.raises(fgd.FgdError) as e:
        fgd.fgd_qk_rope_backward(q, None, q, None, w, None, cos, sin, None, torch.empty_like(q), None, torch.empty_like(w), None, workspace=small)
    assert e.value.status == fgd.FGD_ERR_INVALID_ARG


# ------------------------------------------------------------------------------- embeddings
def _embed_case(tokens, V, W, dtype, scale=0.7, layout="plain", token_type="i64", seed=0):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    tokens = np.asarray(tokens, dtype=np.int64)
    K, rows = tokens.shape
    u, tiny = U[dtype], TINY[dtype]
    tt = {"i64": torch.int64, "i32": torch.int32}[token_type]
    tok = torch.full((K, rows + 3), 2 ** 30, dtype=tt, device="cuda")
    tok[:, :rows] = torch.from_numpy(tokens).to(tt).cuda()
    tok = tok[:, :rows]
    lead, trail = {"plain": (0, 0), "columns": (32, 64), "odd": (3, 2)}[layout]
    theta = torch.full((K, lead + V * W + trail), -777.0, device="cuda")          # the table is a column range of the parameter matrix
    table = theta[:, lead:lead + V * W].unflatten(1, (V, W))
    table.copy_(_randn((K, V, W), "f32", seed))
    pad = {"plain": 0, "columns": 16, "odd": 1}[layout]
    out_buf = torch.full((K * rows, W + pad), -777.0, dtype=_dt(dtype), device="cuda")
    out = out_buf[:, :W]
    fgd.fgd_embed_forward(tok, table, out, scale)
    ref = O.embed(tokens, _np(table), scale)
    assert np.array_equal(np.isnan(ref), np.isnan(_np(out)))
    _near(torch.nan_to_num(out), np.nan_to_num(ref), (u + 3 * F32) * np.abs(np.nan_to_num(ref)) + tiny, "out")
    assert bool((out_buf[:, W:] == -777.0).all())

    dout = torch.full((K * rows, W + pad), float("nan"), dtype=_dt(dtype), device="cuda")[:, :W]
    dout.copy_(_randn((K * rows, W), dtype, seed + 1))
    grads = torch.full_like(theta, -777.0)
    dtable = grads[:, lead:lead + V * W].unflatten(1, (V, W))
    fgd.fgd_embed_backward(tok, dout, dtable, scale)
    g, m, n = O.embed_grad(tokens, _np(dout), V, scale)
    _near(dtable, g, F32 * (n[:, :, None] + 4) * m, "dtable")
    assert bool((grads[:, :lead] == -777.0).all()) and bool((grads[:, lead + V * W:] == -777.0).all()), "columns beside the gradient were written"
    again = torch.full((K, V, W), float("nan"), device="cuda")
    fgd.fgd_embed_backward(tok, dout, again, scale)
    assert torch.equal(again, dtable), "the gradient differs from run to run"


def _text(K, rows, V, seed=0):
    """Tokens with a few common ones."""
    rng = np.random.default_rng(seed)
    return np.minimum(((V + 1.0) ** rng.random((K, rows))).astype(np.int64) - 1, V - 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("K,rows,V,W", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 63, 7, 64), (1, 64, 64, 40), (3, 65, 33, 136), (1, 129, 1000, 257), (8, 17, 300, 256), (1, 33, 257, 1001),
                                        (2, 500, 1023, 24), (2, 512, 40, 520), (2, 513, 1023, 24), (2, 600, 1024, 24), (3, 1024, 11, 300), (1, 1500, 3000, 2048), (1, 4096, 100, 16), (1, 4097, 2000, 48), (2, 9000, 5000, 32), (1, 16384, 900, 8), (1, 16385, 900, 8), (1, 70000, 300, 8), (1, 140000, 70000, 8)])
def test_embed(K, rows, V, W, dtype):
    _embed_case(_text(K, rows, V), V, W, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["columns", "odd"])
@pytest.mark.parametrize("token_type", ["i64", "i32"])
def test_embed_layouts(layout, token_type, dtype):
    _embed_case(_text(3, 150, 90), 90, 72, dtype, layout=layout, token_type=token_type)


@pytest.mark.parametrize("what", ["one", "all_padding", "every_one_once", "backwards", "outside", "two_long_runs", "runs_end_at_chunks", "pad_inside"])
@pytest.mark.parametrize("rows", [400, 640, 6000])
def test_embed_orders(what, rows):
    """Orders of tokens that a cut into chunks of 64 has to stand."""
    V = 7000
    t = {"one": np.full(rows, 77), "all_padding": np.full(rows, -1), "every_one_once": np.arange(rows), "backwards": np.arange(rows)[::-1] + 5,
         "outside": np.where(np.arange(rows) % 3 == 0, V + np.arange(rows), np.where(np.arange(rows) % 3 == 1, -1 - np.arange(rows), 9)),
         "two_long_runs": np.where(np.arange(rows) < rows // 3, V - 1, 0), "runs_end_at_chunks": np.arange(rows) // 64 * 3,
         "pad_inside": np.where(np.arange(rows) % 7 < 3, -5, np.arange(rows) % 11)}[what]
    _embed_case(np.stack([t, _text(1, rows, V, 3)[0]]), V, 24, "bf16", scale=-1.5)


def test_embed_long_vocabulary():
    """Three passes of the sort."""
    rng = np.random.default_rng(0)
    V = 2 ** 20 + 3
    tokens = rng.integers(0, V, (1, 5000))
    tokens[0, :3] = 0, V - 1, V - 1
    _embed_case(tokens, V, 4, "f32")


def test_embed_offsets_beyond_32_bits():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    V, W = 2 ** 21, 2056                       # 4.3e9 elements
    table = torch.zeros((1, V, W), device="cuda")
    tokens = torch.tensor([[0, V - 1, V - 2, V - 1, V // 2 + 1, 12345]], device="cuda")
    for i, t in enumerate(tokens[0].tolist()):
        table[0, t] = 1.0 + t % 97
    out = torch.empty((6, W), dtype=torch.bfloat16, device="cuda")
    fgd.fgd_embed_forward(tokens, table, out)
    assert torch.equal(out[:, 0].float().cpu(), torch.tensor([1.0 + t % 97 for t in tokens[0].tolist()]).bfloat16().float()) and bool((out == out[:, :1]).all())
    table.fill_(7.0)
    dout = torch.arange(1, 7, device="cuda")[:, None].expand(6, W).bfloat16().contiguous()
    fgd.fgd_embed_backward(tokens, dout, table, 2.0)
    want = {0: 2.0, V - 1: 12.0, V - 2: 6.0, V // 2 + 1: 10.0, 12345: 12.0}
    for t, v in want.items():
        assert bool((table[0, t] == v).all()), t
        table[0, t] = 0.0
    assert not bool(table.any()), "rows of absent tokens"


@pytest.mark.parametrize("V,W", [(50, 24), (20000, 24), (20000, 7)])
def test_embed_no_tokens(V, W):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    d = torch.full((2, V, W), 5.0, device="cuda")
    none = torch.empty((2, 0), dtype=torch.int64, device="cuda")
    fgd.fgd_embed_backward(none, torch.empty((0, W), dtype=torch.bfloat16, device="cuda"), d)
    assert not bool(d.any())
    fgd.fgd_embed_forward(none, d, torch.empty((0, W), dtype=torch.bfloat16, device="cuda"))


def test_embed_one_table_for_all_workers():
    """A table expanded over the workers may be read; the gradients need a place each."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    table, tokens = _randn((1, 30, 40), "f32", 0), torch.arange(60, device="cuda").view(3, 20) % 30
    out = torch.empty((60, 40), dtype=torch.bfloat16, device="cuda")
    fgd.fgd_embed_forward(tokens, table.expand(3, -1, -1), out)
    assert torch.equal(out, table[0, tokens.flatten()].bfloat16())
    with pytest.raises(fgd.FgdError) as e:
        fgd.fgd_embed_backward(tokens, out, table.expand(3, -1, -1))
    assert e.value.status == fgd.FGD_ERR_INVALID_ARG


def test_embed_non_finite_gradients_stay_in_their_rows():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    tokens = torch.arange(200, device="cuda")[None] % 50
    tokens[0, 77] = -1
    dout = _randn((200, 40), "bf16", 0)
    dout[33, 5], dout[77] = float("inf"), float("nan")      # the second is padding's
    d = torch.empty((1, 60, 40), device="cuda")
    fgd.fgd_embed_backward(tokens, dout, d)
    bad = ~d.isfinite()
    assert bad.sum() == 1 and bool(bad[0, 33, 5])


def test_embed_gradient_is_the_transpose_of_the_lookup():
    """<dout, lookup(table)> = <gradient, table> for small whole numbers, exactly."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    gen = torch.Generator().manual_seed(0)
    K, rows, V, W = 3, 700, 90, 64
    tokens = torch.randint(-2, V, (K, rows), generator=gen).cuda()
    table = torch.randint(-8, 9, (K, V, W), generator=gen).float().cuda()
    dout = torch.randint(-8, 9, (K * rows, W), generator=gen).bfloat16().cuda()
    out, d = torch.empty_like(dout), torch.empty_like(table)
    fgd.fgd_embed_forward(tokens, table, out, 2.0)
    fgd.fgd_embed_backward(tokens, dout, d, 2.0)
    assert float((out.double() * dout.double()).sum()) == float((d.double() * table.double()).sum())


# ------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,W,ld,lead", [(1, 1, 1, 0), (3, 7, 7, 0), (40, 777, 777, 0), (5, 64, 64, 0), (33, 1024, 1040, 16), (9, 130, 131, 1), (17, 4097, 4097, 3), (2, 16, 1000, 5),
                                         (300, 4, 4, 0), (1000, 33, 36, 2), (6, 2500, 2501, 1), (4, 5001, 5005, 2), (9, 2049, 2049, 0), (5, 8195, 8203, 7)])
def test_dropout(R, W, ld, lead, dtype):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    p, seed, offset = 0.3, 0x9E3779B97F4A7C15, 2 ** 33 + 7
    buf = torch.full((lead + R * ld,), -777.0, dtype=_dt(dtype), device="cuda")
    x = buf[lead:].view(R, ld)[:, :W]
    x.copy_(_randn((R, W), dtype, 0))
    keeps = O.dropout_keeps(R, W, p, seed, offset)
    out_buf = torch.full_like(buf, -777.0)
    out = out_buf[lead:].view(R, ld)[:, :W]
    fgd.fgd_dropout(x, out, p, seed, offset)
    ref = np.where(keeps, _np(x) / (1 - p), 0.0)
    _near(out, ref, (U[dtype] + 3 * F32) * np.abs(ref) + TINY[dtype], "out")
    assert np.array_equal(_np(out) != 0, keeps & (_np(x) != 0))
    rest = out_buf.clone()
    rest[lead:].view(R, ld)[:, :W] = -777.0
    assert bool((rest == -777.0).all()), "memory outside the tensor was written"
    keep = out.clone()
    fgd.fgd_dropout(x, x, p, seed, offset)                    # in place
    assert torch.equal(x, keep)
    rest = buf.clone()
    rest[lead:].view(R, ld)[:, :W] = -777.0
    assert bool((rest == -777.0).all())


def test_dropout_mask_does_not_depend_on_the_layout():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    ones = torch.ones((700, 520), device="cuda")
    masks = []
    for dt, W, ld in ((torch.bfloat16, 520, 520), (torch.float16, 520, 521), (torch.float32, 520, 520), (torch.float32, 517, 523)):
        x = torch.ones((700, ld), dtype=dt, device="cuda")[:, :W]
        out = torch.empty_like(x)
        fgd.fgd_dropout(x, out, 0.5, 5, 9)
        masks.append(out != 0)
    assert all(torch.equal(masks[0][:, :517], m[:, :517]) for m in masks)
    out = torch.empty_like(ones)
    for seed, offset in ((6, 9), (5, 10), (5 + 2 ** 32, 9), (5, 9 + 2 ** 32)):      # every word of seed and offset counts
        fgd.fgd_dropout(ones, out, 0.5, seed, offset)
        same = float(((out != 0) == masks[2]).double().mean())
        assert abs(same - 0.5) < 5 * 0.5 / (700 * 520) ** 0.5


# Widths whose rows, with what the first 16-byte chunk has before them, are whole numbers of 32 chunks, and their neighbours.
ENDS = [("f32", W) for W in (1148, 1149, 1150, 1151, 1152, 1279, 4095)] + [(t, W) for t in ("bf16", "f16") for W in (2296, 2297, 2298, 2299, 2301, 2302, 2303, 2304, 4095)]


@pytest.mark.parametrize("dtype,W", ENDS)
def test_dropout_rows_that_end_with_a_warps_last_chunk(dtype, W):
    """Long rows that start anywhere in a 16-byte chunk, x and out alike: the last columns have verdicts of their own."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    R, seed, offset = 19, 0x1234567812345678, 2 ** 40 + 3
    for lead in (0, 1, 3):
        for ld in (W, W + 1):
            x, out = (torch.empty((lead + R * ld,), dtype=_dt(dtype), device="cuda")[lead:].view(R, ld)[:, :W] for _ in range(2))
            x.copy_(_randn((R, W), dtype, lead))
            fgd.fgd_dropout(x, out, 0.0, seed, offset)
            assert torch.equal(out, x), (lead, ld, "nothing is dropped where p is 0")
            keeps = O.dropout_keeps(R, W, 0.4, seed, offset)
            fgd.fgd_dropout(x, out, 0.4, seed, offset)
            ref = np.where(keeps, _np(x) / 0.6, 0.0)
            _near(out, ref, (U[dtype] + 3 * F32) * np.abs(ref) + TINY[dtype], f"out {lead} {ld}")
            assert np.array_equal(_np(out) != 0, keeps & (_np(x) != 0)), (lead, ld)


@pytest.mark.parametrize("dtype,W", ENDS)
def test_dropout_mask_of_long_rows_does_not_depend_on_the_layout(dtype, W):
    """Rows on the 16-byte boundaries (with columns behind them), rows that start anywhere in a chunk, and x and out at different places of one."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    R, wide = 19, -(-W // 8) * 8
    masks = []
    for width, ld, lead_x, lead_out in ((wide, wide, 0, 0), (W, W, 0, 0), (W, W, 1, 1), (W, W + 2, 3, 3), (W, W, 0, 1), (W, W + 1, 3, 2)):
        x = torch.ones((lead_x + R * ld,), dtype=_dt(dtype), device="cuda")[lead_x:].view(R, ld)[:, :width]
        out = torch.empty((lead_out + R * ld,), dtype=_dt(dtype), device="cuda")[lead_out:].view(R, ld)[:, :width]
        fgd.fgd_dropout(x, out, 0.5, 5, 9)
        masks.append(out[:, :W] != 0)
    assert all(torch.equal(masks[0], m) for m in masks)


@pytest.mark.parametrize("p", [0.0, 1e-3, 0.1, 0.5, 0.9, 1.0 - 2.0 ** -33])
def test_dropout_rate(p):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    R, W = 2000, 1000
    x, out = torch.ones((R, W), device="cuda"), torch.empty((R, W), device="cuda")
    fgd.fgd_dropout(x, out, p, 3)
    kept = float((out != 0).double().mean())
    assert abs(kept - (1 - p)) <= 6 * (p * (1 - p) / (R * W)) ** 0.5 + 2.0 ** -31
    if p == 0.0:
        assert torch.equal(out, x)


def test_dropout_drops_what_is_not_finite():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x = torch.full((64, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[::2] = float("inf")
    out = torch.empty_like(x)
    fgd.fgd_dropout(x, out, 0.5, 1)
    keeps = O.dropout_keeps(64, 64, 0.5, 1, 0)
    got = _np(out)
    assert (got[~keeps] == 0).all() and not np.isfinite(got[keeps]).any()


def test_dropout_far_rows():
    """Rows more than 2^32 elements apart."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    ld = 2 ** 31 + 24
    buf = torch.zeros((2 * ld + 1000,), dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 1000), (ld, 1))
    x.fill_(1.0)
    fgd.fgd_dropout(x, x, 0.5, 11, 4)
    assert np.array_equal(_np(x) != 0, O.dropout_keeps(3, 1000, 0.5, 11, 4))


def test_dropout_counter_in_a_graph():
    """A captured call takes its counter's value at every replay."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x, out = torch.ones((50, 96), device="cuda"), torch.empty((50, 96), device="cuda")
    counter = torch.zeros((), dtype=torch.int64, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fgd.fgd_dropout(x, out, 0.4, 21, 100, counter)
        counter.add_(3)
    for step in range(3):
        g.replay()
        assert np.array_equal(_np(out) != 0, O.dropout_keeps(50, 96, 0.4, 21, 100 + 3 * step))
    counter.fill_(-100)      # the sum wraps in 64 bits
    fgd.fgd_dropout(x, out, 0.4, 21, 50, counter)
    assert np.array_equal(_np(out) != 0, O.dropout_keeps(50, 96, 0.4, 21, 2 ** 64 - 50))


# ------------------------------------------------------------------------------- what the bindings do before the kernels
def test_bindings_give_the_kernels_the_same_either_way(monkeypatch):
    """The checks of the usual call, written out, and the checks one by one pass the same arguments: the same bits, strides and all."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    K, rows, V, W, hq, hk, d = 2, 21, 30, 48, 3, 1, 40
    T = K * rows
    theta = 1.0 + _randn((K, V * W + 2 * d + 3), "f32", 0, 0.2)
    table, w_q, w_k = theta[:, :V * W].view(K, V, W), theta[:, V * W:V * W + d], theta[:, V * W + d:V * W + 2 * d]
    tokens = torch.from_numpy(_text(K, rows + 4, V)).cuda()[:, :rows]
    cos, sin = _tables(40, 24, pad=3)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) % 40
    (q, _), (k, _), (gq, _), (gk, _) = (_layout(T, h, d, "bf16", "fused", fill=_randn((T, h, d), "bf16", 3 + i)) for i, h in enumerate((hq, hk, hq, hk)))

    def run(counter=None):
        grads = torch.zeros_like(theta)
        e, dtable = torch.zeros((T, W + 8), device="cuda", dtype=torch.bfloat16)[:, :W], grads[:, :V * W].view(K, V, W)
        yq, yk, dq, dk, dr = (torch.zeros_like(t) for t in (q, k, q, k, e))
        fgd.fgd_embed_forward(tokens, table, e, 0.5)
        fgd.fgd_embed_backward(tokens, e, dtable, 0.5)
        fgd.fgd_dropout(e, dr, 0.3, 5, 6, counter)
        fgd.fgd_qk_rope_forward(q, k, w_q, w_k, cos, sin, pos, yq, yk, 1e-4, True)
        fgd.fgd_qk_rope_backward(gq, gk, q, k, w_q, w_k, cos, sin, pos, dq, dk, grads[:, V * W:V * W + d], grads[:, V * W + d:V * W + 2 * d], 1e-4, True)
        return e.clone(), grads, yq, yk, dq, dk, dr

    first = run()
    monkeypatch.setattr(fgd, "_rope_usual", lambda *a: None)
    monkeypatch.setattr(fgd, "_embed_usual", lambda *a: None)
    assert all(torch.equal(a, b) and bool(a.any()) for a, b in zip(first, run(torch.zeros((), dtype=torch.int64, device="cuda"))))


def test_bindings_refuse_on_the_gpu():
    """What no kernel may get, one argument of a good call changed at a time: an error, and the outputs as they were."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    K, rows, V, W, h, d = 2, 4, 9, 16, 2, 32
    T, f32 = K * rows, torch.float32
    cos, sin = _tables(20, d)
    full = lambda *shape, dtype=torch.bfloat16: torch.full(shape, 3.0, device="cuda", dtype=dtype)      # noqa: E731
    pos, w = torch.zeros(T, dtype=torch.int64, device="cuda"), full(K, d, dtype=f32)
    tokens, table = torch.zeros((K, rows), dtype=torch.int64, device="cuda"), full(K, V, W, dtype=f32)
    forward = dict(q=full(T, h, d), k=full(T, h, d), w_q=w, w_k=w, cos=cos, sin=sin, positions=pos, q_out=full(T, h, d), k_out=full(T, h, d))
    backward = dict(dq_out=full(T, h, d), dk_out=full(T, h, d), q=full(T, h, d), k=full(T, h, d), w_q=w, w_k=w, cos=cos, sin=sin, positions=pos,
                    dq=full(T, h, d), dk=full(T, h, d), dw_q=full(K, d, dtype=f32), dw_k=full(K, d, dtype=f32))
    x = full(T, W)
    wrong = lambda t: (t.cpu(), t[:-1], t.to(torch.float64), t.unsqueeze(0))      # noqa: E731

    def refused(call, good, extra):
        kept = {n: t.clone() for n, t in good.items()}
        for name, t in [(n, t) for n in good for t in wrong(good[n])] + extra:
            with pytest.raises((TypeError, ValueError, fgd.FgdError)):
                call(**{**good, name: t})
                raise AssertionError(f"{name} {tuple(t.shape)} {t.dtype} {t.device} was taken")
        assert all(torch.equal(good[n], t) for n, t in kept.items())

    narrow = torch.empty((T, h, 2 * d), device="cuda", dtype=torch.bfloat16)[:, :, ::2]
    refused(fgd.fgd_qk_rope_forward, forward, [
        ("q", narrow), ("k", full(T, h, d - 1)), ("k_out", full(T, h + 1, d)), ("q_out", full(1, h, d).expand(T, h, d)), ("q_out", forward["k"]), ("k_out", forward["q_out"]),
        ("q_out", forward["q"][:, :1].expand(T, h, d)), ("w_q", full(K + 1, d, dtype=f32)), ("w_k", full(K, d + 1, dtype=f32)), ("positions", pos.to(torch.int16)),
        ("positions", torch.zeros(2 * T, dtype=torch.int64, device="cuda")[::2]), ("cos", cos[:, :-1]), ("sin", sin.t().contiguous().t())])
    refused(fgd.fgd_qk_rope_backward, backward, [
        ("q", narrow), ("dk_out", full(T, h, d - 1)), ("dq", full(1, h, d).expand(T, h, d)), ("dq", backward["q"]), ("dw_q", w), ("dw_k", backward["dw_q"]),
        ("dw_q", full(1, d, dtype=f32).expand(K, d)), ("dw_q", full(K, 2 * d, dtype=f32)[:, ::2]), ("dw_k", full(K + 1, d, dtype=f32)), ("positions", pos[:-1])])
    for call, good in ((fgd.fgd_embed_forward, dict(tokens=tokens, table=table, out=x)), (fgd.fgd_embed_backward, dict(tokens=tokens, dout=x, dtable=table))):
        refused(call, good, [("tokens", tokens.to(torch.int16)), (list(good)[1 + ("out" not in good)], full(K, V, 2 * W, dtype=f32)[:, :, ::2])])
    refused(fgd.fgd_embed_forward, dict(tokens=tokens, table=table, out=x), [("out", full(1, W).expand(T, W)), ("out", full(T, 2 * W)[:, ::2])])
    refused(fgd.fgd_embed_backward, dict(tokens=tokens, dout=x, dtable=table), [("dtable", full(1, V, W, dtype=f32).expand(K, V, W)), ("dout", full(T, 2 * W)[:, ::2])])
    refused(lambda x, out: fgd.fgd_dropout(x, out, 0.5, 0), dict(x=x, out=full(T, W)), [("out", full(1, W).expand(T, W)), ("x", full(T, 2 * W)[:, ::2]), ("out", x.t()), ("out", full(T, W + 1))])


# ------------------------------------------------------------------------------- streams and graphs
def test_inputs_written_right_before():
    """The kernels start before the one in front of them has ended; what it writes is what they read, the counter too."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, h, d, K, rows, V, W = 20000, 8, 64, 1, 8192, 5000, 512
    given = [_randn((T, h, d), "f32", 0), 1.0 + _randn((1, d), "f32", 1, 0.1), torch.arange(T, device="cuda") % 300, _tables(300, d)[0], _randn((K, V, W), "f32", 2),
             torch.from_numpy(_text(K, rows, V)).cuda(), torch.full((), 3, dtype=torch.int64, device="cuda")]
    sin = _tables(300, d)[1]

    def run(fresh):
        q, w, pos, cos, table, tokens, counter = given
        if fresh:      # each input is written by the kernel in front of the call
            q, w, pos, cos, table, tokens, counter = (torch.zeros_like(t) for t in given)
            for to, t in zip((w, pos, cos, q), (given[1], given[2], given[3], given[0])):
                to.copy_(t)
        qo, ko, e, dtable, dropped = torch.empty_like(q), torch.empty_like(q), torch.empty((K * rows, W), device="cuda"), torch.empty_like(given[4]), torch.empty((K * rows, W), device="cuda")
        fgd.fgd_qk_rope_forward(q, q, w, w, cos, sin, pos, qo, ko)
        if fresh:
            table.copy_(given[4])
            tokens.copy_(given[5])
        fgd.fgd_embed_forward(tokens, table, e)
        fgd.fgd_embed_backward(tokens, e, dtable)
        if fresh:
            counter.copy_(given[6])
        fgd.fgd_dropout(e, dropped, 0.3, 1, 2, counter)
        torch.cuda.synchronize()
        return qo, ko, e, dtable, dropped

    want = run(False)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(want, run(True)))


@pytest.mark.parametrize("rows", [900, 5000, 17000])
@pytest.mark.parametrize("given", [False, True])
def test_on_streams_and_in_graphs(given, rows):
    """All three, forward and backward, on another stream and captured twice, with workspaces of the caller and without."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    K, V, W, hq, hk, d = 2, 500, 384, 4, 2, 64
    T = K * rows
    tokens = torch.from_numpy(_text(K, rows, V)).cuda()
    table = _randn((K, V, W), "f32", 0)
    dout, q, k, gq, gk = _randn((T, W), "bf16", 1), *(_randn((T, h, d), "bf16", 2 + i) for i, h in enumerate((hq, hk, hq, hk)))
    w = 1.0 + _randn((K, d), "f32", 9, 0.1)
    cos, sin = _tables(rows, d)
    pos = torch.arange(T, device="cuda") % rows
    outs = [torch.empty_like(t) for t in (dout, table, q, k, q, k, w, w, dout)]
    room = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (fgd.fgd_embed_workspace(K, rows, V, W), fgd.fgd_qk_rope_workspace(K, d))] if given else [None, None]

    def body(stream=None):
        e, dtab, yq, yk, dq, dk, dwq, dwk, dr = outs
        fgd.fgd_embed_forward(tokens, table, e, 2.0, stream=stream)
        fgd.fgd_dropout(e, dr, 0.2, 1, 2, stream=stream)
        fgd.fgd_qk_rope_forward(q, k, w, w, cos, sin, pos, yq, yk, stream=stream)
        fgd.fgd_qk_rope_backward(gq, gk, q, k, w, w, cos, sin, pos, dq, dk, dwq, dwk, workspace=room[1], stream=stream)
        fgd.fgd_embed_backward(tokens, dout, dtab, 2.0, workspace=room[0], stream=stream)

    body()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]

    def cleared():
        for t in outs:
            t.fill_(-1)
        torch.cuda.synchronize()

    def check(what):
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), what

    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        cleared()
        body(stream)
        check("on a stream")
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            body()
    for g in (*graphs, graphs[0]):
        cleared()
        g.replay()
        check("replayed")
    keep = [t.clone() for t in (tokens, dout)]      # a replay reads what the inputs hold then
    tokens.copy_(tokens.flip(1))
    dout.copy_(dout.view(K, rows, W).flip(1).reshape(T, W))
    cleared()
    graphs[1].replay()
    torch.cuda.synchronize()
    g, m, n = O.embed_grad(tokens.cpu().numpy(), _np(dout), V, 2.0)
    _near(outs[1], g, F32 * (n[:, :, None] + 4) * m, "dtable")
    tokens.copy_(keep[0])
    dout.copy_(keep[1])

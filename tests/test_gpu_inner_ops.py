"""The inner step's operators on the GPU against the float64 oracle, their refusals, and their manners (streams, graphs,
strides, untouched memory).

Tolerances.  u is the unit roundoff of the activations' type.  A result that is rounded once from fp32 is off by u |r|;
where a product's left factor (P, dS) is rounded too, every term of the sum is off by u more; fp32 arithmetic adds a
multiple of 2^-24 of the sum of the terms' magnitudes, which the oracle returns.
"""
import numpy as np
import pytest

from oracle import inner as O

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25, "f32": 0.0}          # half the smallest step of the type
F32 = 2.0 ** -24


def _torch():
    import torch
    return torch


def _dt(name):
    torch = _torch()
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def _np(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _randn(shape, dtype, seed, std=1.0):
    torch = _torch()
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * std).to(_dt(dtype)).cuda()


def _near(got, ref, bound, what):
    got = _np(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == ref.shape, f"{what}: shape {got.shape}, not {ref.shape}"
    err = np.abs(got - ref)
    bad = ~(err <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, err / np.maximum(bound, 1e-300), 0)), err.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} values out of bounds; worst at {i}: got {got[i]!r}, want {ref[i]!r}, bound {bound[i]:.3e}")


# ------------------------------------------------------------------------------- attention
def _layout(T, heads, d, dtype, layout, seed=None, fill=None):
    """A [T, heads, d] tensor in one of several layouts, inside a larger buffer of sentinels; -> (view, buffer)."""
    torch = _torch()
    dt = _dt(dtype)
    if layout == "fused":          # the middle heads of a wider projection
        buf = torch.full((T + 2, heads + 3, d), -777.0, dtype=dt, device="cuda")
        view = buf[1:T + 1, 2:heads + 2]
    elif layout == "head_major":
        buf = torch.full((heads, T + 3, d), -777.0, dtype=dt, device="cuda")
        view = buf[:, 1:T + 1].permute(1, 0, 2)
    elif layout == "odd":          # base and strides off the 16-byte grid
        buf = torch.full((T, heads, d + 1), -777.0, dtype=dt, device="cuda")
        view = buf[:, :, 1:]
    else:
        buf = torch.full((T, heads, d), -777.0, dtype=dt, device="cuda")
        view = buf
    if fill is not None:
        view.copy_(fill)
    elif seed is not None:
        view.copy_(_randn((T, heads, d), dtype, seed))
    return view, buf


def _untouched(view, buf, what):
    torch = _torch()
    keep = buf.clone()
    # everything but the view still holds the sentinel
    view_in_keep = keep.as_strided(view.shape, view.stride(), view.storage_offset())
    view_in_keep.fill_(-777.0)
    assert bool((keep == -777.0).all()), f"{what}: memory outside the tensor was written"


def _attn_case(lens, hq, hk, d, dtype, layout="plain", scale=None, backward=True, seed=0, std=1.0):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    T = int(cu[-1])
    scale = d ** -0.5 if scale is None else scale
    (q, _), (k, _), (v, _) = (_layout(T, h, d, dtype, layout, fill=_randn((T, h, d), dtype, seed + i, std)) for i, h in enumerate((hq, hk, hk)))
    o, o_buf = _layout(T, hq, d, dtype, layout)
    lse = torch.full((hq, T), -777.0, device="cuda")
    plan = fgd.AttnPlan(cu)
    fgd.fgd_attn_forward(plan, q, k, v, o, lse, scale)
    ref_o, ref_lse, mag = O.attention(_np(q), _np(k), _np(v), cu, scale)
    u = U[dtype]
    # fp32: scores of d products, exp of a number of that size, a sum over the keys
    qk = np.abs(scale) * np.sqrt((_np(q) ** 2).sum(2).max(initial=0) * (_np(k) ** 2).sum(2).max(initial=0))
    fp = F32 * (16 + d / 4 + 8 * qk)
    _near(o, ref_o, u * np.abs(ref_o) + (1.01 * u + fp) * mag + TINY[dtype], "o")
    _near(lse, ref_lse, fp + 4 * F32 * np.abs(ref_lse), "lse")
    _untouched(o, o_buf, "o")
    if backward:
        do, _ = _layout(T, hq, d, dtype, layout, fill=_randn((T, hq, d), dtype, seed + 9))
        outs = {n: _layout(T, h, d, dtype, layout) for n, h in (("dq", hq), ("dk", hk), ("dv", hk))}
        delta = torch.full((hq, T), -777.0, device="cuda")
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, outs["dq"][0], outs["dk"][0], outs["dv"][0], scale)
        g, m = O.attention_grad(_np(q), _np(k), _np(v), _np(do), cu, scale)
        for n, (t, buf) in outs.items():
            # P or dS rounded, o (inside delta) rounded, the result rounded; dS = P (dP - delta) in fp32
            _near(t, g[n], u * np.abs(g[n]) + (2.02 * u + 4 * fp) * m[n] + TINY[dtype] * (1 if dtype == "f32" else 2 + T), n)
            _untouched(t, buf, n)
        again = {n: torch.empty_like(t) for n, (t, _) in outs.items()}
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, again["dq"], again["dk"], again["dv"], scale)
        for n in again:
            assert torch.equal(again[n], outs[n][0]), f"{n} differs from run to run"
    fgd.fgd_attn_status(plan)


ATTN_SHAPES = [
    ((1,), 1, 1, 64), ((0, 1, 0, 2, 0), 2, 1, 64), ((127,), 2, 2, 64), ((128,), 4, 2, 128), ((129,), 3, 1, 128),
    ((31, 97, 256, 1, 0, 385), 4, 2, 64), ((200, 56), 6, 2, 80), ((300, 140), 8, 1, 128), ((257, 3), 5, 5, 72),
    ((64, 64, 64, 65), 2, 2, 8), ((513,), 2, 1, 96), ((130, 260), 6, 2, 112), ((383,), 7, 7, 32), ((640, 1, 255), 4, 4, 128), ((77,) * 5, 4, 1, 40),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lens,hq,hk,d", ATTN_SHAPES)
def test_attention(lens, hq, hk, d, dtype):
    _attn_case(lens, hq, hk, d, dtype)


@pytest.mark.parametrize("lens,hq,hk,d,dtype", [
    ((1,), 1, 1, 1, "f32"), ((70, 0, 33, 1), 4, 2, 64, "f32"), ((129, 31), 2, 1, 128, "f32"), ((50, 20), 3, 3, 200, "bf16"), ((40,), 2, 1, 256, "f16"),
    ((33, 90), 2, 2, 5, "bf16"), ((150,), 4, 1, 33, "f16"),
])
def test_attention_element_wise(lens, hq, hk, d, dtype):
    _attn_case(lens, hq, hk, d, dtype)


@pytest.mark.parametrize("layout", ["fused", "head_major", "odd"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attention_layouts(layout, dtype):
    _attn_case((130, 1, 70), 4, 2, 64, dtype, layout=layout)
    if dtype != "f32":
        _attn_case((200, 3), 2, 2, 128, dtype, layout=layout)


def test_attention_scales():
    _attn_case((150, 10), 2, 1, 64, "bf16", scale=0.0)
    _attn_case((150, 10), 2, 1, 64, "bf16", scale=-0.2)
    _attn_case((150, 140), 2, 1, 64, "f16", scale=0.5, std=2.0, seed=4)     # sharp rows: the running maximum moves a lot


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (64, "f32")])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_attention_other_sequences_do_not_leak(d, dtype, bad):
    """Infinities and NaN in one sequence leave every other sequence's results as they were, bit for bit."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    lens, hq, hk = (100, 60, 170, 30), 4, 2
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    plan = fgd.AttnPlan(cu)
    clean = [_randn((T, h, d), dtype, i) for i, h in enumerate((hq, hk, hk, hq))]
    spoilt = [t.clone() for t in clean]
    value = float(bad)
    for t in spoilt:
        t[100:160] = value
        t[330:] = value
    res = []
    for q, k, v, do in (clean, spoilt):
        o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
        fgd.fgd_attn_forward(plan, q, k, v, o, lse)
        delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv)
        res.append((o, lse.T, dq, dk, dv))
    good = torch.ones(T, dtype=torch.bool)
    good[100:160] = False
    good[330:] = False
    for name, a, b in zip(("o", "lse", "dq", "dk", "dv"), *res):
        assert torch.equal(a[good.cuda()], b[good.cuda()]), f"{name} of a clean sequence changed"


@pytest.mark.parametrize("d", [64, 128])
def test_attention_neighbours_do_not_change_rounding(d):
    """Large values in the next sequence, which shares a tile of rows, leave this one's results as they were, bit for bit."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    hq, hk = 4, 2
    plan = fgd.AttnPlan([0, 650, 760])
    q, k, v = (_randn((760, h, d), "bf16", i) for i, h in enumerate((hq, hk, hk)))
    res = []
    for factor in (1.0, 64.0):
        q2 = q.clone()
        q2[650:] *= factor
        o, lse = torch.empty_like(q), torch.empty((hq, 760), device="cuda")
        fgd.fgd_attn_forward(plan, q2, k, v, o, lse)
        res.append((o[:650], lse[:, :650]))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_attention_later_keys_do_not_leak():
    """A NaN key or query of a later token never reaches an earlier token's output."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    for d, dtype in ((64, "bf16"), (128, "bf16"), (64, "f32")):
        q, k, v = (_randn((300, h, d), dtype, i) for i, h in enumerate((4, 2, 2)))
        plan = fgd.AttnPlan([0, 300])
        o1, o2, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((4, 300), device="cuda")
        fgd.fgd_attn_forward(plan, q, k, v, o1, lse)
        k[150:] = float("nan")
        q[150:] = float("inf")
        fgd.fgd_attn_forward(plan, q, k, v, o2, lse)
        assert torch.equal(o1[:150], o2[:150])


def test_attention_gradient_against_differences():
    """Directional differences of the forward kernel itself, in fp32."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    cu, hq, hk, d = [0, 20, 53], 4, 2, 16
    plan = fgd.AttnPlan(cu)
    q, k, v, do = (_randn((53, h, d), "f32", i) for i, h in enumerate((hq, hk, hk, hq)))

    def loss(q, k, v):
        o, lse = torch.empty_like(q), torch.empty((hq, 53), device="cuda")
        fgd.fgd_attn_forward(plan, q, k, v, o, lse)
        return float((o.double() * do.double()).sum()), o, lse

    _, o, lse = loss(q, k, v)
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv)
    for i, g in enumerate((dq, dk, dv)):
        step = _randn(g.shape, "f32", 20 + i)
        eps = 2.0 ** -8
        args_hi, args_lo = [q, k, v], [q, k, v]
        args_hi[i], args_lo[i] = args_hi[i] + eps * step, args_lo[i] - eps * step
        num = (loss(*args_hi)[0] - loss(*args_lo)[0]) / (2 * eps)
        want = float((g.double() * step.double()).sum())
        # truncation eps^2 of a third derivative of order 10^2, rounding 2^-24 10^2 / eps
        assert abs(num - want) <= 1e-2 * max(1.0, abs(want)) ** 0.5 + 2e-3 * abs(want)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_long(d):
    """2100 tokens: many key blocks per row.  Reference in fp64 on the GPU by plain products."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    lens, hq, hk, dtype = (1900, 200), 4, 2, "bf16"
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    q, k, v, do = (_randn((T, h, d), dtype, i) for i, h in enumerate((hq, hk, hk, hq)))
    q[5] *= 8      # a few sharp rows
    q[1500] *= 8
    plan = fgd.AttnPlan(cu)
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse)
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv)
    fgd.fgd_attn_status(plan)
    g, m = O.attention_grad(_np(q), _np(k), _np(v), _np(do), cu, d ** -0.5)
    u = U[dtype]
    for n, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        _near(t, g[n], u * np.abs(g[n]) + 2.1 * u * m[n], n)
    ro = np.zeros((T, hq, d))
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq):
            s = torch.where(torch.tril(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda")), (q[a:b, h].double() @ k[a:b, h // 2].double().T) * d ** -0.5, -float("inf"))
            p = torch.softmax(s, 1)
            ro[a:b, h] = _np(p @ v[a:b, h // 2].double())
            np.testing.assert_allclose(_np(lse[h, a:b]), _np(torch.logsumexp(s, 1)), rtol=1e-6, atol=2e-5)
    rel = np.linalg.norm(_np(o) - ro) / np.linalg.norm(ro)
    assert rel <= u, f"relative error {rel:.2e}"


def test_attention_stream_and_graph():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q, k, v, do = (_randn((200, h, 64), "bf16", i) for i, h in enumerate((4, 2, 2, 4)))
    plan = fgd.AttnPlan([0, 150, 200])
    o, lse = torch.empty_like(q), torch.empty((4, 200), device="cuda")
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def body(stream=None):
        fgd.fgd_attn_forward(plan, q, k, v, o, lse, stream=stream)
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv, stream=stream)

    body()
    torch.cuda.synchronize()
    want = [t.clone() for t in (o, lse, dq, dk, dv)]
    for t in (o, lse, dq, dk, dv):
        t.fill_(-1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    body(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (o, lse, dq, dk, dv)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        body()
    for t in (o, lse, dq, dk, dv):
        t.fill_(-1)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (o, lse, dq, dk, dv)))


@pytest.mark.parametrize("d", [64, 128])
def test_attention_wait_runs_out_and_plan_recovers(d):
    """A load that never comes: the kernels record a timeout, give everything back and return; the plan then works as a new one does."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    cu, T, hq, hk = [0, 700, 900], 900, 4, 2
    q, k, v, do = (_randn((T, h, d), "bf16", i) for i, h in enumerate((hq, hk, hk, hq)))

    def run(plan):
        o, lse = torch.zeros_like(q), torch.zeros((hq, T), device="cuda")
        delta, dq, dk, dv = torch.zeros_like(lse), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        fgd.fgd_attn_forward(plan, q, k, v, o, lse)
        torch.cuda.synchronize()
        return o, lse, (delta, dq, dk, dv)

    def back(plan, o, lse, outs):
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, *outs)
        torch.cuda.synchronize()

    def timed_out(plan):
        with pytest.raises(fgd.FgdError) as e:
            fgd.fgd_attn_status(plan)
        assert e.value.status == fgd.FGD_ERR_TIMEOUT
        fgd.fgd_attn_status(plan)                                         # reported once

    fresh = fgd.AttnPlan(cu)
    want = run(fresh)
    back(fresh, want[0], want[1], want[2])
    fgd.fgd_attn_status(fresh)
    for skip in (1, 2):                                                   # a middle tile; in the forward pass a K and a V tile
        plan = fgd.AttnPlan(cu)
        fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SPIN_LIMIT, 4096)
        fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SKIP_TILE, skip)
        run(plan)
        timed_out(plan)
        back(plan, want[0], want[1], tuple(torch.zeros_like(t) for t in want[2]))
        timed_out(plan)
        fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SPIN_LIMIT, 0)
        fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SKIP_TILE, -1)
        got = run(plan)
        back(plan, got[0], got[1], got[2])
        fgd.fgd_attn_status(plan)
        for a, b in zip(want[:2] + want[2], got[:2] + got[2]):
            assert torch.equal(a, b)
    for key, value in ((fgd.FGD_DEBUG_SKIP_TILE, -2), (fgd.FGD_DEBUG_SPIN_LIMIT, -1), (99, 0)):
        with pytest.raises(fgd.FgdError):
            fgd.fgd_attn_debug_set(fresh, key, value)


def test_attention_refusals():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    for cu in ([1, 2], [0, 3, 2]):
        with pytest.raises(fgd.FgdError) as e:
            fgd.AttnPlan(cu)
        assert e.value.status == fgd.FGD_ERR_INVALID_ARG
    plan = fgd.AttnPlan([0, 10])
    mk = lambda h, d=64, dt="bf16", T=10: _randn((T, h, d), dt, 0)  # noqa: E731
    q, k, v, lse = mk(4), mk(2), mk(2), torch.empty((4, 10), device="cuda")
    o = torch.empty_like(q)

    def refused(status, *args, **kw):
        with pytest.raises(fgd.FgdError) as e:
            fgd.fgd_attn_forward(plan, *args, **kw)
        assert e.value.status == status, e.value

    refused(fgd.FGD_ERR_INVALID_ARG, mk(3), k, v, torch.empty_like(mk(3)), torch.empty((3, 10), device="cuda"))      # 3 heads over 2
    refused(fgd.FGD_ERR_UNSUPPORTED, mk(4, 264), mk(2, 264), mk(2, 264), torch.empty_like(mk(4, 264)), lse)          # width above 256
    refused(fgd.FGD_ERR_ALIAS, q, k, v, q, lse)
    refused(fgd.FGD_ERR_INVALID_ARG, q, k, v, o, lse, float("nan"))
    refused(fgd.FGD_ERR_INVALID_ARG, q, k, v, torch.empty((1, 4, 64), dtype=q.dtype, device="cuda").expand(10, 4, 64), lse)   # an output's rows overlap
    for args, err in (((q.cpu(), k, v, o, lse), (TypeError, ValueError)), ((q, k.half(), v, o, lse), TypeError), ((q, k[:9], v, o, lse), ValueError),
                      ((q.double(), k, v, o, lse), TypeError), ((q, k, v, o, lse.double()), TypeError), ((q, k, v, o, lse[:2]), ValueError)):
        with pytest.raises(err):
            fgd.fgd_attn_forward(plan, *args)
    with pytest.raises(ValueError):
        fgd.fgd_attn_forward(fgd.AttnPlan([0, 11]), q, k, v, o, lse)
    do, delta, dk, dv = torch.empty_like(q), torch.empty_like(lse), torch.empty_like(k), torch.empty_like(v)
    with pytest.raises(fgd.FgdError) as e:
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, do, dk, dv)
    assert e.value.status == fgd.FGD_ERR_ALIAS
    empty = fgd.AttnPlan([0, 0, 0])      # no tokens at all: nothing to do
    z = lambda h: torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    fgd.fgd_attn_forward(empty, z(4), z(2), z(2), z(4), torch.empty((4, 0), device="cuda"))
    fgd.fgd_attn_backward(empty, z(4), z(2), z(2), z(4), z(4), torch.empty((4, 0), device="cuda"), torch.empty((4, 0), device="cuda"), z(4), z(2), z(2))


# ------------------------------------------------------------------------------- block norm
def _matrix(T, H, dtype, layout, seed=None, std=1.0):
    torch = _torch()
    pad = {"plain": 0, "padded": 8, "odd": 1}[layout]
    buf = torch.full((T, H + pad), -777.0, dtype=_dt(dtype), device="cuda")
    view = buf[:, pad:] if layout == "odd" else buf[:, :H]
    if seed is not None:
        view.copy_(_randn((T, H), dtype, seed, std))
    return view, buf


def _norm_case(K, R, H, dtype, gate_kind, post=True, pre=True, has_y=True, dres=True, layout="plain", in_place=False, eps=1e-5, s=0.5):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, u = K * R, U[dtype]
    x, _ = _matrix(T, H, dtype, layout, 1, 2.0)
    y, _ = _matrix(T, H, dtype, layout, 2)
    y = y if has_y else None
    # weights: column ranges of a larger parameter matrix
    params = torch.full((K, 3 * H + 8), 5.0, device="cuda")
    wa, wb, gr = params[:, :H], params[:, H:2 * H], params[:, 2 * H:3 * H]
    for i, w in enumerate((wa, wb, gr)):
        w.copy_(1.0 + 0.3 * _randn((K, H), "f32", 5 + i))
    gate = {None: None, "channel": gr, "element": _matrix(T, H, dtype, layout, 8)[0]}[gate_kind]
    wa, wb = (wa if post else None), (wb if pre else None)
    ref_x, ref_n = O.block_norm(_np(x), _np(y), _np(gate), gate_kind, _np(wa), _np(wb), K, eps, s)
    if in_place:
        xn, xbuf = x, None
    else:
        xn, xbuf = _matrix(T, H, dtype, layout)
    n, nbuf = _matrix(T, H, dtype, layout) if pre else (None, None)
    x0 = _np(x)
    fgd.fgd_block_norm_forward(x, y, gate, wa, wb, xn, n, eps, s)
    fp = F32 * (16 + H / 16)                                             # statistics: sums of H terms over at least 32 lanes
    mag = np.abs(x0) + np.abs(ref_x - x0)
    _near(xn, ref_x, u * np.abs(ref_x) + fp * mag + TINY[dtype], "x_new")
    if pre:
        rx = np.abs(ref_n) / np.maximum(np.abs(ref_x), 1e-30)            # r_x |w|
        _near(n, ref_n, u * np.abs(ref_n) + fp * (np.abs(ref_n) + rx * mag) + TINY[dtype], "n")
        if layout != "plain":
            _untouched(n, nbuf, "n")
    if xbuf is not None and layout != "plain":
        _untouched(xn, xbuf, "x_new")

    dn = _matrix(T, H, dtype, layout, 11)[0] if pre else None
    dr = _matrix(T, H, dtype, layout, 12)[0] if dres else None
    if dn is None and dr is None:
        return
    dx, dxbuf = _matrix(T, H, dtype, layout)
    dy = _matrix(T, H, dtype, layout)[0] if has_y else None
    dparams = torch.full((K, 3 * H + 8), 5.0, device="cuda")
    dwa, dwb = (dparams[:, :H] if post else None), (dparams[:, H:2 * H] if pre else None)
    dgate = {None: None, "channel": dparams[:, 2 * H:3 * H], "element": _matrix(T, H, dtype, layout)[0]}[gate_kind]

    def back(dx_):
        fgd.fgd_block_norm_backward(dn, dr, xn, y, gate, wa, wb, dx_, dy, dgate, dwa, dwb, eps, s)

    back(dx)
    g, m = O.block_norm_grad(_np(dn), _np(dr), _np(xn), _np(y), _np(gate), gate_kind, _np(wa), _np(wb), K, eps, s)
    got = {"dx": dx, "dy": dy, "dgate": dgate, "dw_post": dwa, "dw_pre": dwb}
    assert {k for k, t in got.items() if t is not None} == set(g)
    rows_fp = fp + F32 * (8 + R / 8)                                      # column sums over the rows of a worker
    for k, ref in g.items():
        fp32_out = k in ("dw_post", "dw_pre") or (k == "dgate" and gate_kind == "channel")
        bound = 4 * rows_fp * m[k] if fp32_out else u * np.abs(ref) + 8 * fp * m[k] + TINY[dtype]
        _near(got[k], ref, bound, k)
    assert bool((dparams[:, 3 * H:] == 5.0).all()), "columns beside the gradients were written"
    if layout != "plain":
        _untouched(dx, dxbuf, "dx")
    keep = {k: t.clone() for k, t in got.items() if t is not None}
    back(dx)
    for k, t in keep.items():
        assert torch.equal(t, got[k]), f"{k} differs from run to run"
    if dr is not None:                                                    # dx in place of dres
        back(dr)
        assert torch.equal(dr, keep["dx"])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("K,R,H", [(1, 1, 1), (1, 3, 7), (2, 5, 64), (1, 33, 1001), (4, 9, 256), (1, 2, 1024), (8, 3, 2048), (3, 200, 136), (1, 4, 4096), (2, 2, 5000),
                                   (1, 3, 8192), (1, 2, 16384), (1, 2, 16001), (1, 700, 40)])
def test_block_norm(K, R, H, dtype):
    _norm_case(K, R, H, dtype, "channel")


@pytest.mark.parametrize("gate_kind", [None, "channel", "element"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("dtype,H", [("bf16", 512), ("f32", 77)])
def test_block_norm_parts(gate_kind, post, dtype, H):
    _norm_case(2, 6, H, dtype, gate_kind, post=post)
    _norm_case(2, 6, H, dtype, gate_kind, post=post, in_place=True)
    _norm_case(2, 6, H, dtype, gate_kind, post=post, dres=False)
    if post:
        _norm_case(2, 6, H, dtype, gate_kind, pre=False)


def test_block_norm_only_norm():
    for dtype, H in (("bf16", 768), ("f16", 33)):
        _norm_case(2, 5, H, dtype, None, post=False, has_y=False)


@pytest.mark.parametrize("layout", ["padded", "odd"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_norm_layouts(layout, dtype):
    for gate_kind in ("channel", "element"):
        _norm_case(2, 7, 264, dtype, gate_kind, layout=layout)


def test_block_norm_zero_rows_and_constant_rows():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((1, 64), device="cuda")
    n, xn = torch.empty_like(x), torch.empty_like(x)
    fgd.fgd_block_norm_forward(x, x.clone(), None, w, w, xn, n)          # all-zero rows: eps keeps them finite
    assert bool((n == 0).all()) and bool((xn == 0).all())
    z = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    dw, dp = torch.full((2, 64), 7.0, device="cuda"), torch.full((2, 64), 7.0, device="cuda")
    w2 = torch.ones((2, 64), device="cuda")
    fgd.fgd_block_norm_backward(z, z, z, z, None, w2, w2, z.clone(), z.clone(), None, dp, dw)     # no rows: gradients of weights are zero
    assert bool((dw == 0).all()) and bool((dp == 0).all())


def test_block_norm_side_stream():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, H = 64, 512
    dn, dr, x, y = (_randn((T, H), "bf16", i) for i in range(4))
    w = torch.ones((1, H), device="cuda")
    outs = [[torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)] for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o, st in zip(outs, (None, side)):
        fgd.fgd_block_norm_backward(dn, dr, x, y, None, w, w, o[0], o[1], None, o[2], o[3], stream=st)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_block_norm_refusals():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x, w = _randn((6, 64), "bf16", 0), torch.ones((2, 64), device="cuda")
    y, n = x.clone(), torch.empty_like(x)

    def refused(status, *a, **kw):
        with pytest.raises(fgd.FgdError) as e:
            fgd.fgd_block_norm_forward(*a, **kw)
        assert e.value.status == status, e.value

    refused(fgd.FGD_ERR_ALIAS, x, y, None, w, w, y, n)                    # x_new on top of y
    refused(fgd.FGD_ERR_ALIAS, x, y, None, w, w, torch.empty_like(x), x)
    refused(fgd.FGD_ERR_INVALID_ARG, x, y, None, w, w, None, n)           # x_new is needed
    refused(fgd.FGD_ERR_INVALID_ARG, x, None, None, w, w, torch.empty_like(x), n)   # w_post without y
    refused(fgd.FGD_ERR_INVALID_ARG, x, y, None, w, None, torch.empty_like(x), n)   # n without w_pre
    wide = torch.zeros((2, 16400), dtype=torch.bfloat16, device="cuda")
    refused(fgd.FGD_ERR_UNSUPPORTED, wide, wide.clone(), None, None, torch.ones((1, 16400), device="cuda"), torch.empty_like(wide), torch.empty_like(wide))
    with pytest.raises(ValueError):
        fgd.fgd_block_norm_forward(x[:5], y[:5], None, w, w, n[:5], torch.empty_like(x[:5]))     # 5 rows over 2 workers
    with pytest.raises(TypeError):
        fgd.fgd_block_norm_forward(x, y, None, w.bfloat16(), w, n, torch.empty_like(x))
    with pytest.raises(fgd.FgdError) as e:
        fgd.fgd_block_norm_backward(x, None, y, None, None, None, w, n, None, None, None, torch.empty_like(w), workspace=torch.empty(4, dtype=torch.uint8, device="cuda"))
    assert e.value.status == fgd.FGD_ERR_INVALID_ARG and "workspace" in e.value.message


# ------------------------------------------------------------------------------- 8-bit checkpoints
def _values8(R, W, dtype, seed):
    torch = _torch()
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((R, W), generator=gen) * torch.exp(2 * torch.randn((R, 1), generator=gen))
    if R > 2:
        x[1] = 0
        x[2, ::3] *= 1e-6
    return x.to(_dt(dtype)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,W,layout", [(1, 1, "plain"), (3, 31, "plain"), (5, 32, "plain"), (4, 33, "plain"), (7, 777, "plain"), (9, 40, "plain"), (6, 256, "padded"),
                                        (5, 96, "odd"), (2, 4104, "plain"), (300, 64, "plain"), (1000, 8, "plain")])
def test_act8(R, W, layout, dtype):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x, _ = _matrix(R, W, dtype, layout)
    x.copy_(_values8(R, W, dtype, 3))
    q = torch.full((R, W + 8), 99, dtype=torch.int8, device="cuda")
    e = torch.full((R, -(-W // 32) + 3), 99, dtype=torch.uint8, device="cuda")
    fgd.fgd_act_save8(x, q[:, :W], e[:, :-3])
    rq, re = O.save8(_np(x))
    assert np.array_equal(q[:, :W].cpu().numpy(), rq) and np.array_equal(e[:, :-3].cpu().numpy(), re)
    assert bool((q[:, W:] == 99).all()) and bool((e[:, -3:] == 99).all())
    out, buf = _matrix(R, W, dtype, layout)
    fgd.fgd_act_load8(q[:, :W], e[:, :-3], out)
    want = torch.from_numpy(O.load8(rq, re)).to(_dt(dtype))
    assert torch.equal(out.cpu(), want)
    if dtype == "bf16":
        assert np.array_equal(_np(out), O.load8(rq, re)), "a bf16 value read back is exactly the stored one"
    if layout != "plain":
        _untouched(out, buf, "out")


@pytest.mark.parametrize("W", [64, 65])
def test_act8_non_finite_and_extremes(W):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x = torch.ones((6, W), device="cuda")
    x[0, 3], x[1, 40], x[2, 0] = float("inf"), float("nan"), -float("inf")
    x[3] = 3.4e38
    x[4] = 1e-41                                       # subnormal: below the smallest step
    x[5, 1] = 127.75 / 128                             # rounds beyond 127 steps: held there
    x[5, 2] = -x[5, 1]
    q, e = torch.empty((6, W), dtype=torch.int8, device="cuda"), torch.empty((6, -(-W // 32)), dtype=torch.uint8, device="cuda")
    back = torch.empty_like(x)
    fgd.fgd_act_save8(x, q, e)
    fgd.fgd_act_load8(q, e, back)
    rq, re = O.save8(_np(x))
    ok = re != 255
    assert np.array_equal(e.cpu().numpy(), re) and np.array_equal(q.cpu().numpy()[np.repeat(ok, 32, 1)[:, :W]], rq[np.repeat(ok, 32, 1)[:, :W]])
    assert torch.equal(torch.isnan(back).cpu(), torch.from_numpy(np.repeat(~ok, 32, 1)[:, :W]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,F,layout", [(1, 1, "plain"), (3, 33, "plain"), (5, 64, "plain"), (4, 1000, "plain"), (2, 2051, "plain"), (17, 136, "padded"), (6, 96, "odd"), (257, 32, "plain")])
def test_swiglu8(R, F, layout, dtype):
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    u = U[dtype]
    gu, _ = _matrix(R, 2 * F, dtype, layout, 1, 2.0)
    h, hbuf = _matrix(R, F, dtype, layout)
    q, e = torch.empty((R, 2 * F), dtype=torch.int8, device="cuda"), torch.empty((R, 2 * -(-F // 32)), dtype=torch.uint8, device="cuda")
    fgd.fgd_swiglu8_forward(gu, h, q, e)
    x = _np(gu)
    (qg, eg), (qu, eu) = O.save8(x[:, :F]), O.save8(x[:, F:])
    assert np.array_equal(q.cpu().numpy(), np.hstack([qg, qu])) and np.array_equal(e.cpu().numpy(), np.hstack([eg, eu]))
    # sigmoid from a fast exponential and division: a few units of 2^-21 (the exponent's rounding grows with |g|)
    ref = O.swiglu(x[:, :F], x[:, F:])
    fp = 2.0 ** -20 * (1 + np.abs(x[:, :F]))
    _near(h, ref, (u + fp) * np.abs(ref) + TINY[dtype], "h")
    g8, u8 = O.load8(qg, eg), O.load8(qu, eu)
    dh, _ = _matrix(R, F, dtype, layout, 7)
    dgu, dbuf = _matrix(R, 2 * F, dtype, layout)
    h2, _ = _matrix(R, F, dtype, layout)
    fgd.fgd_swiglu8_backward(dh, q, e, dgu, h2)
    rg, ru = O.swiglu_grad(_np(dh), g8, u8)
    fp8 = 2.0 ** -20 * (1 + np.abs(g8))
    mag = np.abs(_np(dh) * u8) / (1 + np.exp(-g8)) * (1 + np.abs(g8))
    _near(dgu[:, :F], rg, u * np.abs(rg) + fp8 * mag + TINY[dtype], "dg")
    _near(dgu[:, F:], ru, (u + fp8) * np.abs(ru) + TINY[dtype], "du")
    ref8 = O.swiglu(g8, u8)
    _near(h2, ref8, (u + fp8) * np.abs(ref8) + TINY[dtype], "h again")
    if layout != "plain":
        _untouched(h, hbuf, "h")
        _untouched(dgu, dbuf, "dgu")
    keep = dgu.clone()
    fgd.fgd_swiglu8_backward(dh, q, e, dgu)              # without h
    assert torch.equal(keep, dgu)


def test_swiglu8_large_gates():
    """Far tails of the sigmoid stay finite."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    gu = torch.ones((1, 64), device="cuda")
    gu[0, :32] = torch.linspace(-200, 200, 32)
    h, q, e = torch.empty((1, 32), device="cuda"), torch.empty((1, 64), dtype=torch.int8, device="cuda"), torch.empty((1, 2), dtype=torch.uint8, device="cuda")
    fgd.fgd_swiglu8_forward(gu, h, q, e)
    ref = O.swiglu(_np(gu)[:, :32], _np(gu)[:, 32:])
    _near(h, ref, 1e-4 * np.abs(ref) + 1e-30, "h")
    dgu = torch.empty_like(gu)
    fgd.fgd_swiglu8_backward(torch.ones_like(h), q, e, dgu)
    assert bool(torch.isfinite(dgu).all())


class _Anywhere:
    """Copies of tensors at odd offsets and strides inside guarded buffers."""

    def __init__(self, seed):
        self.rng, self.kept = np.random.default_rng(seed), []

    def __call__(self, t):
        torch = _torch()
        if t is None:
            return None
        R, W = t.shape
        at, ld = int(self.rng.integers(1, 9)), W + int(self.rng.integers(0, 6))
        buf = torch.full((at + R * ld + 9,), 77, dtype=t.dtype, device="cuda")
        view = buf[at:at + R * ld].view(R, ld)[:, :W]
        view.copy_(t)
        free = torch.ones_like(buf, dtype=torch.bool)
        free[at:at + R * ld].view(R, ld)[:, :W] = False
        self.kept.append((buf, free))
        return view

    def check(self):
        for buf, free in self.kept:
            assert bool((buf[free] == 77).all()), "written outside a tensor"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,W", [(1, 8), (2, 16), (7, 24), (40, 8), (3, 264), (5, 520), (2, 1032), (3, 2056), (2, 4104), (9, 8192)])
def test_rows_that_start_anywhere(R, W, dtype):
    """The same bits as with aligned rows, and nothing beside the rows touched."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    K, G = 2, -(-W // 32)
    for seed in range(3):
        place = _Anywhere(100 * W + R + seed)
        x, y, dn, dr, gate = (_randn((K * R, W), dtype, i, 2.0) for i in range(5))
        wa, wb = 1.0 + 0.3 * _randn((K, W), "f32", 6), 1.0 + 0.3 * _randn((K, W), "f32", 7)
        outs = []
        for f in (lambda t: t, place):
            a = [f(t) for t in (x, y, gate, wa, wb)]
            e = [f(torch.zeros_like(x)) for _ in range(5)]
            d = [f(torch.zeros_like(wa)) for _ in range(2)]
            fgd.fgd_block_norm_forward(*a, e[0], e[1], 1e-5, 0.5)
            fgd.fgd_block_norm_backward(f(dn), f(dr), e[0], *a[1:], e[2], e[3], e[4], *d, 1e-5, 0.5)
            q, s = f(torch.zeros((K * R, W), dtype=torch.int8, device="cuda")), torch.zeros((K * R, G), dtype=torch.uint8, device="cuda")
            back = f(torch.zeros_like(x))
            fgd.fgd_act_save8(a[0], q, s)
            fgd.fgd_act_load8(q, s, back)
            gu, h, q2, s2 = f(torch.cat((x, y), 1)), f(torch.zeros_like(x)), f(torch.zeros((K * R, 2 * W), dtype=torch.int8, device="cuda")), torch.zeros((K * R, 2 * G), dtype=torch.uint8, device="cuda")
            dgu, h2 = f(torch.zeros_like(gu)), f(torch.zeros_like(x))
            fgd.fgd_swiglu8_forward(gu, h, q2, s2)
            fgd.fgd_swiglu8_backward(f(dn), q2, s2, dgu, h2)
            outs.append(e + d + [q, s, back, h, q2, s2, dgu, h2])
        for i, (a, b) in enumerate(zip(*outs)):
            assert torch.equal(a, b), f"output {i} differs"
        place.check()


def test_act8_refusals():
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    x = _randn((4, 64), "bf16", 0)
    q, e = torch.empty((4, 64), dtype=torch.int8, device="cuda"), torch.empty((4, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        fgd.fgd_act_save8(x, q[:, :63], e)
    with pytest.raises(ValueError):
        fgd.fgd_act_save8(x, q, e[:, :1])
    with pytest.raises(TypeError):
        fgd.fgd_act_save8(x, q.to(torch.uint8), e)
    with pytest.raises(TypeError):
        fgd.fgd_act_save8(x.cpu(), q, e)
    with pytest.raises(TypeError):
        fgd.fgd_act_load8(q, e, x.to(torch.float64))
    with pytest.raises(fgd.FgdError) as err:
        fgd.fgd_act_save8(x, x.view(torch.int8)[:, :64], e)               # the checkpoint on top of its source
    assert err.value.status == fgd.FGD_ERR_ALIAS
    gu, h = _randn((4, 128), "bf16", 0), torch.empty((4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(fgd.FgdError) as err:
        fgd.fgd_swiglu8_forward(gu, gu[:, 32:96], torch.empty((4, 128), dtype=torch.int8, device="cuda"), torch.empty((4, 4), dtype=torch.uint8, device="cuda"))
    assert err.value.status == fgd.FGD_ERR_ALIAS
    # no rows: nothing to do
    fgd.fgd_act_save8(x[:0], q[:0], e[:0])
    fgd.fgd_swiglu8_backward(h[:0], torch.empty((0, 128), dtype=torch.int8, device="cuda"), torch.empty((0, 4), dtype=torch.uint8, device="cuda"), gu[:0])

"""The inner step's operators at the ends of their types' ranges, with non-finite values, on other streams and through autograd: cases in
which a result can be wrong although ordinary values are right.

Tolerances as in the operators' own tests: u is the unit roundoff of the activations' type, fp32 arithmetic adds multiples of 2^-24.
"""
import numpy as np
import pytest

from oracle import inner as O

from .test_gpu_inner_ops import F32, TINY, U, _dt, _near, _norm_case, _np, _randn, _torch

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------- 8-bit checkpoints
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W", [64, 72, 65])
def test_act8_reads_back_every_magnitude(W, dtype):
    """Groups whose largest magnitude is 2^-126 to 2^128: what is read back is q8 2^(e8 - 127), bit for bit, zeros and small members too."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    gen = torch.Generator().manual_seed(W)
    powers = torch.arange(-126, 128, dtype=torch.float64)[:, None]
    x = 2 * torch.rand((254, W), generator=gen, dtype=torch.float64) - 1
    x[:, 5::7] *= 1e-3
    x[:, 3::11] = 0
    x[:, 1], x[:, 33], x[:, -1] = 1.0, -1.984375, 1.0            # (127 steps exactly, and beyond: held there)
    x = (x * 2.0 ** powers).to(_dt(dtype)).cuda()
    q, e = torch.empty((254, W), dtype=torch.int8, device="cuda"), torch.empty((254, -(-W // 32)), dtype=torch.uint8, device="cuda")
    back = torch.empty_like(x)
    fgd.fgd_act_save8(x, q, e)
    fgd.fgd_act_load8(q, e, back)
    rq, re = O.save8(_np(x))
    assert re.min() == 1 and re.max() == 248
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(e.cpu().numpy(), re)
    assert np.array_equal(_np(back), O.load8(rq, re))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("F", [64, 72, 65])
def test_swiglu8_backward_of_large_values(F, dtype):
    """u from 2^-90 to 2^120 beside a moderate g."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    u = U[dtype]
    powers = torch.arange(-90, 121, 3)[:, None]
    R = len(powers)
    gu = torch.cat((_randn((R, F), "f32", 1).cpu(), (_randn((R, F), "f32", 2).cpu().clamp(-4, 4) * 2.0 ** powers.double()).float()), 1).to(_dt(dtype)).cuda()
    h, h2 = torch.empty((R, F), dtype=gu.dtype, device="cuda"), torch.empty((R, F), dtype=gu.dtype, device="cuda")
    q, e = torch.empty((R, 2 * F), dtype=torch.int8, device="cuda"), torch.empty((R, 2 * -(-F // 32)), dtype=torch.uint8, device="cuda")
    dh, dgu = _randn((R, F), dtype, 3), torch.empty_like(gu)
    fgd.fgd_swiglu8_forward(gu, h, q, e)
    fgd.fgd_swiglu8_backward(dh, q, e, dgu, h2)
    x = _np(gu)
    (qg, eg), (qu, eu) = O.save8(x[:, :F]), O.save8(x[:, F:])
    assert np.array_equal(q.cpu().numpy(), np.hstack([qg, qu])) and np.array_equal(e.cpu().numpy(), np.hstack([eg, eu])) and eu.max() >= 240
    g8, u8 = O.load8(qg, eg), O.load8(qu, eu)
    fp8 = 2.0 ** -20 * (1 + np.abs(g8))
    rg, ru = O.swiglu_grad(_np(dh), g8, u8)
    _near(dgu[:, :F], rg, u * np.abs(rg) + fp8 * np.abs(_np(dh) * u8) / (1 + np.exp(-g8)) * (1 + np.abs(g8)), "dg")
    _near(dgu[:, F:], ru, (u + fp8) * np.abs(ru), "du")
    ref = O.swiglu(g8, u8)
    _near(h2, ref, (u + fp8) * np.abs(ref), "h again")


# ------------------------------------------------------------------------------- streams
@pytest.mark.parametrize("given_as", ["stream", "handle"])
def test_block_norm_workspace_belongs_to_the_calls_stream(given_as):
    """Without a workspace the call takes one from its own stream's memory: a block that was freed on the current stream, and is still to be
    written there, is not handed to a call on another stream."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, H = 512, 1024
    dn, dr, x, y = (_randn((T, H), "bf16", i) for i in range(4))
    w = torch.ones((1, H), device="cuda")
    want = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)]
    got = [torch.empty_like(t) for t in want]
    need = fgd.fgd_block_norm_workspace(fgd.FGD_BF16, 1, T, H)
    fgd.fgd_block_norm_backward(dn, dr, x, y, None, w, w, want[0], want[1], None, want[2], want[3])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for _ in range(5):
        blocks = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda._sleep(20_000_000)                                     # the current stream is behind, and then writes the blocks
        for b in blocks:
            for _ in range(20):
                b.fill_(0x7F)
        del blocks, b
        fgd.fgd_block_norm_backward(dn, dr, x, y, None, w, w, got[0], got[1], None, got[2], got[3],
                                    stream=side if given_as == "stream" else side.cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_attention_plan_is_ready_on_every_stream():
    """A plan can be used on a stream that does not wait for the default one as soon as it exists."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    rng = np.random.default_rng(0)
    side = torch.cuda.Stream()
    hq, hk, d, T = 4, 2, 64, 3000
    q, k, v = (_randn((T, h, d), "bf16", i) for i, h in enumerate((hq, hk, hk)))
    torch.cuda.synchronize()
    for _ in range(8):
        cu = np.concatenate([[0], np.sort(rng.integers(0, T, 600)), [T]])
        o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
        torch.cuda.synchronize()
        plan = fgd.AttnPlan(cu)
        fgd.fgd_attn_forward(plan, q, k, v, o, lse, stream=side)
        side.synchronize()
        o2, lse2 = torch.empty_like(q), torch.empty_like(lse)
        fgd.fgd_attn_forward(plan, q, k, v, o2, lse2)
        fgd.fgd_attn_status(plan)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


# ------------------------------------------------------------------------------- autograd
def test_second_derivatives_are_refused():
    """The backward passes are not differentiable: a second derivative through them is an error, not a result without their terms."""
    from paper_2606_22768_b200 import AttnPlan, inner
    torch = _torch()
    plan = AttnPlan([0, 20, 32])

    def leaf(shape, seed, dtype="bf16"):
        return _randn(shape, dtype, seed).requires_grad_(True)

    q, k, v = leaf((32, 4, 64), 0), leaf((32, 2, 64), 1), leaf((32, 2, 64), 2)
    x, y, w_post, w_pre = leaf((32, 64), 3), leaf((32, 64), 4), leaf((2, 64), 5, "f32"), leaf((2, 64), 6, "f32")
    gu, w = leaf((32, 128), 7), leaf((2, 48, 64), 8)
    for name, out, t in (("attention", inner.attention(q, k, v, plan), q), ("block_norm", inner.block_norm(x, y, None, w_post, w_pre)[1], x),
                         ("swiglu8", inner.swiglu8(gu), gu), ("linear8", inner.linear8(x, w), w)):
        for loss in (out.float().square().sum(), out.float().sum()):      # (the gradient that comes in depends on the inputs, or is constant)
            with pytest.raises(RuntimeError, match="differentiable twice"):
                g, = torch.autograd.grad(loss, t, create_graph=True, retain_graph=True)
                torch.autograd.grad((g * t).float().sum(), t)
                pytest.fail(f"{name}: a second derivative came back")
            torch.autograd.grad(loss, t, retain_graph=True)               # the first derivative is there as before


# ------------------------------------------------------------------------------- attention: masked and non-finite values
@pytest.mark.parametrize("d", [64, 128])
def test_attention_large_values_of_later_tokens_do_not_leak(d):
    """Finite values of later tokens, up to the type's largest, leave an earlier token's output as it was, bit for bit."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q, k, v = (_randn((300, h, d), "bf16", i) for i, h in enumerate((4, 2, 2)))
    plan = fgd.AttnPlan([0, 300])
    res = []
    for value in (None, 3e38, -3e38):
        v2 = v.clone()
        if value is not None:
            v2[150:] = value
        o, lse = torch.empty_like(q), torch.empty((4, 300), device="cuda")
        fgd.fgd_attn_forward(plan, q, k, v2, o, lse)
        res.append(o[:150])
    assert torch.equal(res[0], res[1]) and torch.equal(res[0], res[2])


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (64, "f32")])
def test_attention_nan_key_in_any_column(d, dtype):
    """A NaN key makes every row that sees it NaN, output and lse, wherever in a block of keys it stands; the rows before it stay."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, hq, hk = 300, 4, 2
    q, k, v = (_randn((T, h, d), dtype, i) for i, h in enumerate((hq, hk, hk)))
    plan = fgd.AttnPlan([0, T])
    o0, lse0 = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o0, lse0)
    for at in list(range(16)) + [62, 63, 126, 127, 142, 143, 255, 270, 299]:
        bad = k.clone()
        bad[at] = float("nan")
        o, lse = torch.empty_like(q), torch.empty_like(lse0)
        fgd.fgd_attn_forward(plan, q, bad, v, o, lse)
        assert torch.equal(o[:at], o0[:at]) and torch.equal(lse[:, :at], lse0[:, :at]), f"key {at}"
        assert bool(o[at:].isnan().all()) and bool(lse[:, at:].isnan().all()), f"key {at}"


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (64, "f32")])
def test_attention_minus_infinity_scores(d, dtype):
    """A key whose scores are all -inf has no weight, also where it is the only key that a row sees of its own block of 128: the row is the
    softmax of the others, however low their scores."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, hq, hk, scale = 300, 4, 2, 0.125
    q, k, v = (_randn((T, h, d), dtype, i) for i, h in enumerate((hq, hk, hk)))
    q[..., 0], k[..., 0] = 1.0, 0.0
    q[..., 1], k[..., 1] = 16.0, -200.0                                   # every score is about -400
    k[256, :, 0] = float("-inf")
    plan = fgd.AttnPlan([0, T])
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse, scale)
    fgd.fgd_attn_status(plan)
    ref, ref_lse, mag = O.attention(_np(q), _np(k), _np(v), [0, T], scale)
    u, fp = U[dtype], F32 * (16 + d / 4 + 8 * 450)
    _near(o, ref, u * np.abs(ref) + (1.01 * u + fp) * mag + TINY[dtype], "o")
    _near(lse, ref_lse, fp + 4 * F32 * np.abs(ref_lse), "lse")


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16"), (64, "f32")])
def test_attention_row_without_a_finite_score(d, dtype):
    """A row that sees scores of -inf alone has no softmax: NaN, and an lse that is not finite; the rows beside it are as without it."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    q, k, v = (_randn((41, h, d), dtype, i).abs() for i, h in enumerate((4, 2, 2)))
    plan = fgd.AttnPlan([0, 1, 41])
    res = []
    for value in (1.0, float("-inf")):
        k[0] = value
        o, lse = torch.empty_like(q), torch.empty((4, 41), device="cuda")
        fgd.fgd_attn_forward(plan, q, k, v, o, lse)
        res.append((o, lse))
    assert bool(res[1][0][0].isnan().all()) and not bool(torch.isfinite(res[1][1][:, 0]).any())
    assert torch.equal(res[0][0][1:], res[1][0][1:]) and torch.equal(res[0][1][:, 1:], res[1][1][:, 1:])


# ------------------------------------------------------------------------------- attention: gradients of any size in fp16
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [-13, 12])
def test_attention_gradient_scales_with_dout_f16(d, power):
    """dout times a power of two gives the gradients times that power, but for the rounding of the results: nothing between loses bits to the
    type's smallest values or runs over its largest.  (dout in steps of 1/8, so that it stays exact; long rows, so that P is small.)"""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    lens, hq, hk, u = (1900, 200), 4, 2, U["f16"]
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    q, k = _randn((T, hq, d), "f16", 0), _randn((T, hk, d), "f16", 1)
    v = _randn((T, hk, d), "f16", 2, 4.0)
    do = (torch.round(_randn((T, hq, d), "f32", 3) * 8) / 8).clamp(-3.875, 3.875).half()
    plan = fgd.AttnPlan(cu)
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse)
    f, res = 2.0 ** power, []
    for g in (do, do * f):
        delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        fgd.fgd_attn_backward(plan, q, k, v, o, g, lse, delta, dq, dk, dv)
        res.append((dq, dk, dv))
    fgd.fgd_attn_status(plan)
    for n, a, b in zip(("dq", "dk", "dv"), *res):
        want, b = _np(a) * f, _np(b)
        inside = np.abs(want) < 65504 * (1 - 4 * u)                       # (a few results are beyond the type)
        assert inside.mean() > 0.999 and (np.abs(b[~inside]) > 65504 * (1 - 8 * u)).all()
        _near(b[inside], want[inside], 2.02 * u * np.abs(want[inside]) + (1 + f) * 2.0 ** -25, n)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_gradient_of_small_dout_f16(d):
    """Gradients of a dout around 2^-13 against 64 bits.  dS is held times a power of two that takes max |dout| max |v| to 2^6 or more, so a term
    loses at most 2^-25 max |dout| max |v| / 64, below 2^-27 max |dout| here (max |v| < 16); P, held times 2^10, 2^-35."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    lens, hq, hk, u = (1200, 70), 4, 2, U["f16"]
    cu = np.concatenate([[0], np.cumsum(lens)])
    T = int(cu[-1])
    q, k, v = (_randn((T, h, d), "f16", i) for i, h in enumerate((hq, hk, hk)))
    do = _randn((T, hq, d), "f16", 3, 2.0 ** -13)
    plan = fgd.AttnPlan(cu)
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse)
    delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv)
    g, m = O.attention_grad(_np(q), _np(k), _np(v), _np(do), cu, d ** -0.5)
    n, amax = max(lens), float(do.abs().max())
    assert float(v.abs().max()) < 16
    floor = {"dq": n * 2.0 ** -27 * amax * d ** -0.5 * float(k.abs().max()), "dk": 2 * n * 2.0 ** -27 * amax * d ** -0.5 * float(q.abs().max()),
             "dv": 2 * n * 2.0 ** -35 * amax}
    fp = F32 * (16 + d / 4 + 8 * d ** -0.5 * float(_np(q).__pow__(2).sum(2).max() * _np(k).__pow__(2).sum(2).max()) ** 0.5)
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        _near(t, g[name], u * np.abs(g[name]) + (2.02 * u + 4 * fp) * m[name] + TINY["f16"] + floor[name], name)


# ------------------------------------------------------------------------------- block norm
@pytest.mark.parametrize("H", [64, 77])
def test_block_norm_weight_gradient_without_dn(H):
    """The norm before the next block unused (no dn): its weight's gradient is zero, not what the memory held."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    dr, x, y = (_randn((6, H), "bf16", i) for i in range(3))
    w = torch.ones((2, H), device="cuda")
    for rows in (6, 0):
        out = [torch.full((rows, H), 7.0, dtype=x.dtype, device="cuda") for _ in range(2)]
        dpost, dpre = torch.full((2, H), 7.0, device="cuda"), torch.full((2, H), 7.0, device="cuda")
        fgd.fgd_block_norm_backward(None, dr[:rows], x[:rows], y[:rows], None, w, w, out[0], out[1], None, dpost, dpre)
        assert bool((dpre == 0).all())
        assert torch.equal(out[0], dr[:rows])


# ------------------------------------------------------------------------------- the inner steps
def test_inner_step_refuses_invalid_gradients():
    """A device-side wait that gave up leaves invalid gradients: the step raises, and parameters and moments stay as they were."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    torch = _torch()
    K, lens, cfg = 2, [200, 60], inner.DecoderConfig()
    rows = sum(lens)
    layout, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 1)
    gen = torch.Generator().manual_seed(2)
    tokens, targets = (torch.randint(cfg.vocab, (K, rows), generator=gen).cuda() for _ in range(2))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    want = inner.InnerSteps(theta.clone(), cfg)
    want.step(tokens, targets, plan, positions)
    steps = inner.InnerSteps(theta.clone(), cfg)
    fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SPIN_LIMIT, 4096)
    fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SKIP_TILE, 1)
    with pytest.raises(fgd.FgdError) as e:
        steps.step(tokens, targets, plan, positions)
    assert e.value.status == fgd.FGD_ERR_TIMEOUT
    assert torch.equal(steps.theta, theta) and not bool(steps.m.any()) and not bool(steps.v.any()) and steps.t == 0
    fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SPIN_LIMIT, 0)
    fgd.fgd_attn_debug_set(plan, fgd.FGD_DEBUG_SKIP_TILE, -1)
    steps.step(tokens, targets, plan, positions)
    behind = layout["0.attn.pre"][0]      # (the embedding's own gradient is a sum by atomics, torch's, whose bits do not repeat)
    assert torch.equal(steps.theta[:, behind:], want.theta[:, behind:])


@pytest.mark.parametrize("F", [64, 65])
def test_swiglu8_sigmoid_in_fp32(F):
    """fp32 activations get an fp32 sigmoid.  Exponential within 2 units, denominator, quotient and two products half a unit each: 2^-21 of the
    result, whatever the gate's size."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    gate = torch.linspace(-86, 86, 40 * F).view(40, F)
    gu = torch.cat((gate, _randn((40, F), "f32", 1).cpu()), 1).cuda()
    h, h2 = torch.empty((40, F), device="cuda"), torch.empty((40, F), device="cuda")
    q, e = torch.empty((40, 2 * F), dtype=torch.int8, device="cuda"), torch.empty((40, 2 * -(-F // 32)), dtype=torch.uint8, device="cuda")
    fgd.fgd_swiglu8_forward(gu, h, q, e)
    x = _np(gu)
    ref = O.swiglu(x[:, :F], x[:, F:])
    _near(h, ref, 2.0 ** -21 * np.abs(ref), "h")
    dh, dgu = _randn((40, F), "f32", 2), torch.empty_like(gu)
    fgd.fgd_swiglu8_backward(dh, q, e, dgu, h2)
    g8, u8 = O.load8(*O.save8(x[:, :F])), O.load8(*O.save8(x[:, F:]))
    _, ru = O.swiglu_grad(_np(dh), g8, u8)
    _near(dgu[:, F:], ru, 2.0 ** -21 * np.abs(ru), "du")
    ref = O.swiglu(g8, u8)
    _near(h2, ref, 2.0 ** -21 * np.abs(ref), "h again")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("F", [32, 33])
def test_swiglu8_forward_of_extreme_gates(F, dtype):
    """g sigmoid(g) u at the ends: the gate itself above, zero below, an infinite one infinite above and NaN below (inf x 0), NaN stays."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    top = torch.finfo(_dt(dtype)).max
    gate = torch.tensor([float("inf"), float("-inf"), float("nan"), top, -top, top / 8, -top / 8, 0.0, 1e4, -1e4, 130.0, -130.0])
    gu = torch.ones((len(gate), 2 * F), dtype=_dt(dtype), device="cuda")
    gu[:, :F] = gate[:, None].to(_dt(dtype)).cuda()
    h = torch.empty((len(gate), F), dtype=gu.dtype, device="cuda")
    q, e = torch.empty((len(gate), 2 * F), dtype=torch.int8, device="cuda"), torch.empty((len(gate), 2 * -(-F // 32)), dtype=torch.uint8, device="cuda")
    fgd.fgd_swiglu8_forward(gu, h, q, e)
    want = torch.where(gate > 0, gu[:, 0].cpu().float(), torch.where(gate < 0, torch.zeros(()), gate))
    want[1] = float("nan")
    assert torch.equal(torch.nan_to_num(h.float().cpu(), nan=-7.0), torch.nan_to_num(want, nan=-7.0)[:, None].expand(-1, F).contiguous())


@pytest.mark.parametrize("dtype,off", [("f32", 1e-4), ("f16", 0.005)])
def test_decoder_in_other_types(dtype, off):
    """Loss, logits and gradients of the decoder in fp32 and fp16 against fp64: the logits see the type's roundings alone (a few dozen of 2^-11
    in fp16; library products and sums in fp32), the gradients also the 8-bit checkpoints, about 1.5 % of the values' norm each."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    from .test_gpu_inner_path import _plain_logits
    torch = _torch()
    cfg = inner.DecoderConfig(vocab=96, width=128, layers=2, n_q_heads=4, n_kv_heads=2, head_dim=32, ffn=160)
    lens, K = [70, 1, 130, 33], 2
    rows = sum(lens)
    layout, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 1)
    gen = torch.Generator().manual_seed(2)
    theta += (0.05 * torch.randn(theta.shape, generator=gen)).cuda()
    tokens, targets = (torch.randint(cfg.vocab, (K, rows), generator=gen).cuda() for _ in range(2))
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    leaf, ref = theta.clone().requires_grad_(True), theta.double().requires_grad_(True)
    logits, want = inner.decoder_logits(leaf, tokens, plan, positions, cfg, _dt(dtype)), _plain_logits(ref, tokens, lens, cfg)
    inner.worker_losses(logits, targets).sum().backward()
    loss = -torch.gather(torch.log_softmax(want, -1), 2, targets[:, :, None]).mean((1, 2))
    loss.sum().backward()
    fgd.fgd_attn_status(plan)
    assert float((logits.detach().double() - want.detach()).norm() / want.detach().norm()) < off
    for name, (at, shape) in layout.items():
        n = int(np.prod(shape))
        g, w = leaf.grad[:, at:at + n].double(), ref.grad[:, at:at + n]
        assert float((g - w).norm() / w.norm()) < 0.08, name


# ------------------------------------------------------------------------------- refusals of the C entry points
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_attention_refuses_pointers_between_elements(dtype):
    """Refused before anything is launched (torch makes no such tensors, so the arguments are packed here)."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, hq, hk, d = 40, 2, 1, 64
    plan = fgd.AttnPlan([0, T])
    q, o, do, dq = (_randn((T, hq, d), dtype, i) for i in range(4))
    k, v, dk, dv = (_randn((T, hk, d), dtype, 4 + i) for i in range(4))
    lse, delta = torch.zeros((hq, T), device="cuda"), torch.zeros((hq, T), device="cuda")
    heads = [(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, k, v, o, do, dq, dk, dv)]
    code = {"bf16": fgd.FGD_BF16, "f16": fgd.FGD_F16, "f32": fgd.FGD_F32}[dtype]

    def pack(off):
        at = [(p + (1 if i == off else 0), s, h) for i, (p, s, h) in enumerate(heads)]
        return fgd._ATTN_ARGS.pack(code, hq, hk, d, *at[0], *at[1], *at[2], *at[3], lse.data_ptr() + 2 * (off == 8), 0.125, *at[4],
                                   delta.data_ptr() + 2 * (off == 9), *at[5], *at[6], *at[7])

    for off in range(10):
        if off in (0, 1, 2, 3, 8):
            assert fgd._lib.fgd_attn_forward(plan._h, pack(off), None) == fgd.FGD_ERR_INVALID_ARG
            assert "boundary" in fgd.fgd_last_error(None)
        assert fgd._lib.fgd_attn_backward(plan._h, pack(off), None) == fgd.FGD_ERR_INVALID_ARG
        assert "boundary" in fgd.fgd_last_error(None)
    assert fgd._lib.fgd_attn_forward(plan._h, pack(-1), None) == fgd.FGD_OK
    fgd.fgd_attn_status(plan)


# ------------------------------------------------------------------------------- what a block keeps
def test_swiglu8_linear():
    """Output and gradients of the fused pair, and that beside the weights only the checkpoint of g and u is kept: 2 bytes and a little per element
    of the hidden width.  The gradients are those at the checkpointed values, with one rounding of each factor: u of every term."""
    from paper_2606_22768_b200 import inner
    torch = _torch()
    K, R, F, N, u = 2, 40, 96, 48, U["bf16"]
    gu, w, dy = _randn((K * R, 2 * F), "bf16", 0), _randn((K, N, F), "bf16", 1, F ** -0.5), _randn((K * R, N), "bf16", 2)
    gu.requires_grad_(True), w.requires_grad_(True)
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        y = inner.swiglu8_linear(gu, w)
    assert sum(t.numel() * t.element_size() for t in kept if t is not w and t.data_ptr() != w.data_ptr()) == K * R * 2 * (F + F // 32)
    y.backward(dy)
    x, wd, dyd = _np(gu), _np(w), _np(dy).reshape(K, R, N)
    h = O.swiglu(x[:, :F], x[:, F:]).reshape(K, R, F)
    ref, mag = h @ wd.transpose(0, 2, 1), np.abs(h) @ np.abs(wd).transpose(0, 2, 1)
    _near(y, ref.reshape(-1, N), u * np.abs(ref.reshape(-1, N)) + 1.1 * u * mag.reshape(-1, N), "y")
    g8, u8 = O.load8(*O.save8(x[:, :F])), O.load8(*O.save8(x[:, F:]))
    h8 = O.swiglu(g8, u8).reshape(K, R, F)
    ref, mag = dyd.transpose(0, 2, 1) @ h8, np.abs(dyd).transpose(0, 2, 1) @ np.abs(h8)
    _near(w.grad, ref, u * np.abs(ref) + 1.1 * u * mag, "dw")
    dh, dh_mag = (dyd @ wd).reshape(-1, F), (np.abs(dyd) @ np.abs(wd)).reshape(-1, F)
    rg, ru = O.swiglu_grad(dh, g8, u8)
    mg, mu = O.swiglu_grad(dh_mag, g8, u8)
    _near(gu.grad, np.hstack([rg, ru]), u * np.abs(np.hstack([rg, ru])) + 1.1 * u * np.abs(np.hstack([mg, mu])), "dgu")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", ["inf", "nan"])
def test_attention_gradient_beside_a_non_finite_dout_f16(d, bad):
    """A row whose dout is not finite has no say in how the factors of others are held: rows beside it, and keys that it does not see, get the
    bits that they get with zeros there."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    T, hq, hk, at = 300, 4, 2, 290
    q, k, v = (_randn((T, h, d), "f16", i) for i, h in enumerate((hq, hk, hk)))
    do = _randn((T, hq, d), "f16", 3, 2.0 ** -13)
    plan = fgd.AttnPlan([0, T])
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse)
    res = []
    for value in (0.0, float(bad)):
        do[at] = value
        delta, dq, dk, dv = torch.empty_like(lse), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        fgd.fgd_attn_backward(plan, q, k, v, o, do, lse, delta, dq, dk, dv)
        res.append((dq, dk))
    (dq0, dk0), (dq1, dk1) = res
    assert torch.equal(dq0[:at], dq1[:at]) and torch.equal(dq0[at + 1:], dq1[at + 1:])
    assert torch.equal(dk0[at + 1:], dk1[at + 1:])
    assert not bool(torch.isfinite(dq1[at]).any())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("K", [1, 2, 8])
def test_block_norm_channel_gate_alone_with_one_row_per_worker(K, dtype):
    """A gate per channel says how many workers there are, also where each has a single row and no norm has weights."""
    _norm_case(K, 1, 33, dtype, "channel", post=False, pre=False)
    _norm_case(K, 3, 33, dtype, "channel", post=False, pre=False)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_f16_gradient_on_streams_in_graphs_and_after_a_timeout(d):
    """The fp16 gradient hands values on in rows of dq that are not written yet: the same bits on another stream, from a replayed graph, with two
    plans' calls in flight at once, and by a plan whose wait ran out before."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    cu, T, hq, hk = [0, 700, 900], 900, 4, 2
    q, k, v, do = (_randn((T, h, d), "f16", i) for i, h in enumerate((hq, hk, hk, hq)))
    plan, other = fgd.AttnPlan(cu), fgd.AttnPlan(cu)
    o, lse = torch.empty_like(q), torch.empty((hq, T), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse)

    def outputs():
        return [torch.full_like(t, 7.0) for t in (lse, q, k, v)]

    def back(p, out, stream=None):
        fgd.fgd_attn_backward(p, q, k, v, o, do, lse, *out, stream=stream)

    want = outputs()
    back(plan, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = [outputs() for _ in range(6)]
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        back((plan, other)[i % 2], out, side if i % 3 == 0 else None)
    torch.cuda.synchronize()
    g, out = torch.cuda.CUDAGraph(), outputs()
    with torch.cuda.graph(g):
        back(plan, out)
        back(plan, out)
    for t in out:
        t.fill_(-1)
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    fgd.fgd_attn_debug_set(other, fgd.FGD_DEBUG_SPIN_LIMIT, 4096)
    fgd.fgd_attn_debug_set(other, fgd.FGD_DEBUG_SKIP_TILE, 1)
    back(other, outputs())
    with pytest.raises(fgd.FgdError) as e:
        fgd.fgd_attn_status(other)
    assert e.value.status == fgd.FGD_ERR_TIMEOUT
    fgd.fgd_attn_debug_set(other, fgd.FGD_DEBUG_SPIN_LIMIT, 0)
    fgd.fgd_attn_debug_set(other, fgd.FGD_DEBUG_SKIP_TILE, -1)
    after = outputs()
    back(other, after)
    fgd.fgd_attn_status(other)
    fgd.fgd_attn_status(plan)
    for res in got + [out, after]:
        for a, b in zip(want[1:], res[1:]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_small_weights_f16(d):
    """Weights down to 2^-21 of the largest keep the type's relative precision: pairs of tokens whose second one gives the first, with a large v, a
    weight from 1/2 to e^-14."""
    import paper_2606_22768_b200 as fgd
    torch = _torch()
    n, u = 300, U["f16"]
    q, k, v = torch.zeros((2 * n, 2, d)), torch.zeros((2 * n, 1, d)), _randn((2 * n, 1, d), "f32", 0).cpu() * 1000
    q[..., 0] = 1.0
    k[0::2, 0, 0] = -torch.linspace(0, 14, n)
    v[1::2] = 0
    q, k, v = (t.half().cuda() for t in (q, k, v))
    cu = list(range(0, 2 * n + 1, 2))
    plan = fgd.AttnPlan(cu)
    o, lse = torch.empty_like(q), torch.empty((2, 2 * n), device="cuda")
    fgd.fgd_attn_forward(plan, q, k, v, o, lse, 1.0)
    ref, ref_lse, mag = O.attention(_np(q), _np(k), _np(v), cu, 1.0)
    fp = F32 * (16 + d / 4 + 8 * 14)
    _near(o, ref, u * np.abs(ref) + (1.01 * u + fp) * mag + TINY["f16"], "o")
    _near(lse, ref_lse, fp + 4 * F32 * np.abs(ref_lse), "lse")

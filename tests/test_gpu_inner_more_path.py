"""Embeddings, head norms with rotation and dropout as autograd functions, and together in the decoder's training step."""
import numpy as np
import pytest

from oracle import inner as O
from tests.test_gpu_inner_ops import _dt, _np, _randn, _torch

pytestmark = pytest.mark.gpu


def _plain_logits(theta, tokens, lens, cfg, draw):
    """The decoder in fp64 with autograd, one worker and one sequence at a time, nothing quantised; dropout's masks from the oracle."""
    torch = _torch()
    from paper_2606_22768_b200 import inner
    layout, _ = inner.param_layout(cfg)
    K, rows = tokens.shape
    masks = []
    if draw is not None and cfg.dropout > 0:
        seed, step = draw
        masks = [torch.from_numpy(O.dropout_keeps(K * rows, cfg.width, cfg.dropout, seed, (site << 32) + step)).cuda() / (1 - cfg.dropout) for site in range(1 + 2 * cfg.layers)]
    out = []
    for m in range(K):
        p = {name: theta[m, at:at + int(np.prod(shape))].view(shape) for name, (at, shape) in layout.items()}
        rms = lambda t, w: t / (t.square().mean(-1, keepdim=True) + cfg.eps).sqrt() * w  # noqa: E731
        at = 0
        for n in lens:
            mine = slice(m * rows + at, m * rows + at + n)
            drop = lambda t, site: t * masks[site][mine] if masks else t  # noqa: E731
            tok = tokens[m, at:at + n]
            x = cfg.embed_scale * torch.where(tok[:, None] < 0, 0.0, p["embed"][tok.clamp_min(0)])
            x = drop(x, 0)
            at += n
            pos = torch.arange(n, device=x.device, dtype=torch.float64)
            angle = pos[:, None] * cfg.rope_base ** (-torch.arange(0, cfg.head_dim, 2, device=x.device, dtype=torch.float64) / cfg.head_dim)
            turn = torch.complex(angle.cos(), angle.sin())[:, None]

            def rot(t):
                z = torch.complex(*t.chunk(2, -1)) * turn
                return torch.cat((z.real, z.imag), -1)

            for i in range(cfg.layers):
                h = (rms(x, p[f"{i}.attn.pre"]) @ p[f"{i}.qkv"].T).view(n, -1, cfg.head_dim)
                q, k, v = h.split((cfg.n_q_heads, cfg.n_kv_heads, cfg.n_kv_heads), 1)
                if cfg.qk_norm:
                    q, k = rms(q, p[f"{i}.q_norm"]), rms(k, p[f"{i}.k_norm"])
                q, k = rot(q), rot(k)
                g = cfg.n_q_heads // cfg.n_kv_heads
                s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(g, 1)) * cfg.head_dim ** -0.5
                s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), -float("inf"))
                y = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v.repeat_interleave(g, 1)).reshape(n, -1) @ p[f"{i}.out"].T
                x = x + cfg.res_scale * p[f"{i}.attn.gate"] * rms(drop(y, 1 + 2 * i), p[f"{i}.attn.post"])
                a, b = (rms(x, p[f"{i}.mlp.pre"]) @ p[f"{i}.up"].T).chunk(2, -1)
                y = (torch.nn.functional.silu(a) * b) @ p[f"{i}.down"].T
                x = x + cfg.res_scale * p[f"{i}.mlp.gate"] * rms(drop(y, 2 + 2 * i), p[f"{i}.mlp.post"])
            out.append(rms(x, p["final"]) @ p["head"].T)
    return torch.cat(out).view(K, rows, -1)


@pytest.mark.parametrize("dtype,off", [("f32", 1e-4), ("f16", 0.005), ("bf16", 0.03)])
@pytest.mark.parametrize("qk_norm,dropout,scale", [(True, 0.2, 3.0), (True, 0.0, 1.0), (False, 0.1, 1.0)])
def test_decoder(qk_norm, dropout, scale, dtype, off):
    """Logits and the gradient of every parameter against fp64.  The logits see the type's roundings (a few dozen of them in a row), the gradients also
    the 8-bit checkpoints, about 1.5 % of the values' norm each: a few percent of each gradient's norm."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    torch = _torch()
    cfg = inner.DecoderConfig(vocab=96, width=128, layers=2, n_q_heads=4, n_kv_heads=2, head_dim=32, ffn=160, qk_norm=qk_norm, dropout=dropout, embed_scale=scale)
    lens, K = [70, 1, 130, 33], 2
    rows = sum(lens)
    layout, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 1)
    gen = torch.Generator().manual_seed(2)
    theta += (0.05 * torch.randn(theta.shape, generator=gen)).cuda()       # workers apart, norms and gates away from 1
    tokens, targets = (torch.randint(cfg.vocab, (K, rows), generator=gen).cuda() for _ in range(2))
    tokens[:, -5:] = -1                                                     # padding
    targets[:, -5:] = -1
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    draw = (77, 5)
    leaf, ref = theta.clone().requires_grad_(True), theta.double().requires_grad_(True)
    logits, want = inner.decoder_logits(leaf, tokens, plan, positions, cfg, _dt(dtype), draw), _plain_logits(ref, tokens, lens, cfg, draw)
    inner.worker_losses(logits, targets).sum().backward()
    keep = targets >= 0
    lp = torch.log_softmax(want, -1)
    (-(torch.gather(lp, 2, targets.clamp_min(0)[:, :, None])[:, :, 0] * keep).sum(1) / keep.sum(1)).sum().backward()
    fgd.fgd_attn_status(plan)
    assert float((logits.detach().double() - want.detach()).norm() / want.detach().norm()) < off
    for name, (at, shape) in layout.items():
        n = int(np.prod(shape))
        g, w = leaf.grad[:, at:at + n].double(), ref.grad[:, at:at + n]
        rel = float((g - w).norm() / w.norm())
        assert rel < 0.08, f"{name}: the gradient is {rel:.3f} of its norm off"
    if dropout > 0:      # another step, another mask; without a draw none
        other = inner.decoder_logits(theta, tokens, plan, positions, cfg, _dt(dtype), (77, 6))
        assert not torch.equal(other, logits)
        step = torch.full((1,), 5, dtype=torch.int64, device="cuda")
        assert torch.equal(inner.decoder_logits(theta, tokens, plan, positions, cfg, _dt(dtype), (77, step)), logits)
        none = inner.decoder_logits(theta, tokens, plan, positions, cfg, _dt(dtype))
        assert float((none.double() - _plain_logits(theta.double(), tokens, lens, cfg, None)).norm() / want.detach().norm()) < off


def test_layout_of_the_new_parameters():
    from paper_2606_22768_b200 import inner
    plain, _ = inner.param_layout(inner.DecoderConfig())
    normed, _ = inner.param_layout(inner.DecoderConfig(qk_norm=True))
    assert set(normed) - set(plain) == {f"{i}.{n}_norm" for i in range(2) for n in "qk"} and normed["1.q_norm"][1] == (64,)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_embedding_of_scale_one_is_the_rounded_table(dtype):
    from paper_2606_22768_b200 import inner
    torch = _torch()
    table = _randn((2, 50, 40), "f32", 0)
    tokens = torch.randint(50, (2, 30), generator=torch.Generator().manual_seed(1)).cuda()
    want = torch.gather(table.to(_dt(dtype)), 1, tokens[:, :, None].expand(-1, -1, 40)).reshape(60, 40)
    assert torch.equal(inner.embedding(tokens, table, 1.0, _dt(dtype)), want)


def test_functions_gradients():
    """Through autograd, with inputs that are views and gradients that come as they come."""
    from paper_2606_22768_b200 import inner
    torch = _torch()
    K, rows, V, W, hq, hk, d = 2, 90, 33, 64, 3, 1, 16
    T = K * rows
    theta = _randn((K, V * W + 2 * d + 7), "f32", 0).requires_grad_(True)
    table, w_q, w_k = theta[:, :V * W].unflatten(1, (V, W)), theta[:, V * W:V * W + d], theta[:, V * W + d:V * W + 2 * d]
    tokens = torch.randint(-1, V, (K, rows), generator=torch.Generator().manual_seed(1)).cuda()
    angle = torch.rand((T, d // 2), generator=torch.Generator().manual_seed(2)).cuda()
    proj = _randn((W, (hq + 2 * hk) * d), "f32", 3, W ** -0.5)
    gq, gk, gv = (_randn((T, h, d), "f32", 4 + i) for i, h in enumerate((hq, hk, hk)))

    def loss(embed, drop, rope):
        x = drop(embed())
        q, k, v = rope((x @ proj).view(T, hq + 2 * hk, d))
        return (q * gq).sum() + (k * gk).sum() + (v.transpose(0, 1) * gv.transpose(0, 1)).sum()

    got, = torch.autograd.grad(loss(lambda: inner.embedding(tokens, table, 0.5, torch.float32), lambda x: inner.dropout(x, 0.3, 9, 1),
                                    lambda h: inner.qkv_rope(h, hq, hk, angle.cos(), angle.sin(), None, w_q, w_k)), theta)
    ref = theta.detach().double().requires_grad_(True)
    rt, rq, rk = ref[:, :V * W].unflatten(1, (V, W)), ref[:, V * W:V * W + d], ref[:, V * W + d:V * W + 2 * d]
    keep = torch.from_numpy(O.dropout_keeps(T, W, 0.3, 9, 1)).cuda()

    def plain_embed():
        rows_ = torch.gather(rt, 1, tokens.clamp_min(0)[:, :, None].expand(-1, -1, W)) * 0.5
        return torch.where(tokens[:, :, None] < 0, 0.0, rows_).reshape(T, W)

    def plain_rope(h):
        out = []
        for x, w in ((h[:, :hq], rq), (h[:, hq:hq + hk], rk)):
            z = x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.repeat_interleave(rows, 0)[:, None]
            z = torch.complex(*z.chunk(2, -1)) * torch.complex(angle.double().cos(), angle.double().sin())[:, None]
            out.append(torch.cat((z.real, z.imag), -1))
        return *out, h[:, hq + hk:]

    proj, gq, gk, gv = proj.double(), gq.double(), gk.double(), gv.double()
    want, = torch.autograd.grad(loss(plain_embed, lambda x: x * keep / 0.7, plain_rope), ref)
    np.testing.assert_allclose(_np(got), _np(want), rtol=1e-4, atol=1e-4 * float(want.abs().max()))      # (angles' cos and sin, products in fp32)


def test_second_derivatives_are_refused():
    from paper_2606_22768_b200 import inner
    torch = _torch()
    table = _randn((1, 9, 16), "f32", 0).requires_grad_(True)
    x = inner.embedding(torch.arange(8, device="cuda")[None], table, 1.0, torch.float32)
    h = _randn((8, 4, 4), "f32", 1).requires_grad_(True)
    c = torch.ones((8, 2), device="cuda")
    for out, leaf in ((x, table), (inner.dropout(x, 0.5, 1), table), (inner.qkv_rope(h, 2, 1, c, c)[0], h)):
        with pytest.raises(RuntimeError, match="not differentiable twice"):
            torch.autograd.grad(out.sum(), leaf, create_graph=True)


def test_a_counter_that_moved_before_the_backward_pass_is_an_error():
    from paper_2606_22768_b200 import inner
    torch = _torch()
    x, counter = _randn((4, 32), "f32", 0).requires_grad_(True), torch.zeros(1, dtype=torch.int64, device="cuda")
    y = inner.dropout(x, 0.5, 1, 0, counter)
    counter.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_training_pass_in_a_graph():
    """The functions' forward and backward passes captured once; every replay drops by its own step and equals the eager pass of that step."""
    from paper_2606_22768_b200 import inner
    torch = _torch()
    K, rows, V, W, hq, hk, d = 2, 700, 300, 128, 4, 2, 16
    T = K * rows
    gen = torch.Generator().manual_seed(0)
    tokens = torch.randint(V, (K, rows), generator=gen).cuda()
    table, w = _randn((K, V, W), "f32", 1), 1.0 + _randn((K, d), "f32", 2, 0.1)
    angle = torch.rand((T, d // 2), generator=gen).cuda()
    cos, sin = angle.cos(), angle.sin()
    up = _randn((T, hq, d), "bf16", 3)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def passes(table, w, step):
        x = inner.dropout(inner.embedding(tokens, table), 0.25, 3, 1 << 32, step)
        q, k, v = inner.qkv_rope(x.view(T, hq + 2 * hk, d), hq, hk, cos, sin, None, w, w)
        return torch.autograd.grad((q * up).sum() + k.sum() + v.sum(), (table, w))

    want = []
    for i in range(3):
        want.append([g.clone() for g in passes(table.clone().requires_grad_(True), w.clone().requires_grad_(True), torch.full((1,), i, dtype=torch.int64, device="cuda"))])
    lt, lw = table.clone().requires_grad_(True), w.clone().requires_grad_(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        passes(lt, lw, step)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes(lt, lw, step)
    for i in range(3):
        step.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), f"step {i}"
    assert not torch.equal(want[0][0], want[1][0])


def test_inner_steps_with_everything():
    """A few steps run, are reproducible to the bit from the seed, and differ with another one."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    torch = _torch()
    cfg = inner.DecoderConfig(qk_norm=True, dropout=0.1, embed_scale=2.0)
    K, lens = 2, [100, 28]
    _, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 0)
    gen = torch.Generator().manual_seed(1)
    tokens, targets = (torch.randint(cfg.vocab, (K, sum(lens)), generator=gen).cuda() for _ in range(2))
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    runs = []
    for seed in (4, 4, 5):
        steps = inner.InnerSteps(theta.clone(), cfg, seed=seed)
        losses = [steps.step(tokens, targets, plan, positions) for _ in range(3)]
        assert all(bool(x.isfinite().all()) for x in losses)
        runs.append(steps.theta)
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0], runs[2])


def test_example_runs_with_norms_and_dropout():
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("inner_and_outer", os.path.join(root, "examples", "inner_and_outer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    history = ex.main(["--rounds", "2", "--inner", "2", "--workers", "2", "--qk-norm", "--dropout", "0.1"])
    assert len(history) == 2 and all(np.isfinite(v) for row in history for v in row)


@pytest.mark.parametrize("how", ["expanded", "transposed", "every second", "windows", "columns", "one worker", "int32"])
def test_decoder_takes_tokens_of_any_strides(how):
    """Logits and gradients are those of the same tokens laid out in rows."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    torch = _torch()
    cfg = inner.DecoderConfig()
    K, lens = 1 if how == "one worker" else 3, [60, 4]
    rows = sum(lens)
    many = torch.randint(cfg.vocab, (K * rows * 2,), generator=torch.Generator().manual_seed(1)).cuda()
    tokens = {"expanded": lambda: many[None, :rows].expand(K, -1), "transposed": lambda: many[:rows * K].view(rows, K).t(), "every second": lambda: many.view(K, 2 * rows)[:, ::2],
              "windows": lambda: many.unfold(0, rows, 1)[:K], "columns": lambda: many.view(K, 2 * rows)[:, 5:5 + rows], "one worker": lambda: many[:rows].view(rows, 1).t(),
              "int32": lambda: many[None, :rows].int().expand(K, -1)}[how]()
    assert tokens.shape == (K, rows)
    _, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 0)
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    got = []
    for t in (tokens, tokens.contiguous().clone()):
        leaf = theta.clone().requires_grad_(True)
        logits = inner.decoder_logits(leaf, t, plan, positions, cfg)
        logits.float().square().sum().backward()
        got.append((logits.detach(), leaf.grad))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("wrong", [256, 257, 2 ** 40])
def test_inner_steps_refuse_tokens_beyond_the_vocabulary(wrong):
    """Parameters, moments and the count of steps stay, and the next step is as if there had been none; padding is no such token."""
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    torch = _torch()
    cfg = inner.DecoderConfig(dropout=0.1)
    K, lens = 2, [100, 28]
    _, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 0)
    gen = torch.Generator().manual_seed(1)
    tokens, targets = (torch.randint(cfg.vocab, (K, sum(lens)), generator=gen).cuda() for _ in range(2))
    tokens[0, -3:] = targets[0, -3:] = -1
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    plain, steps = inner.InnerSteps(theta.clone(), cfg), inner.InnerSteps(theta.clone(), cfg)
    plain.step(tokens, targets, plan, positions)
    steps.step(tokens, targets, plan, positions)
    keep = [t.clone() for t in (steps.theta, steps.m, steps.v)]
    bad = tokens.clone()
    bad[1, 5] = wrong
    with pytest.raises(IndexError, match="vocabulary of 256"):
        steps.step(bad, targets, plan, positions)
    assert all(torch.equal(a, b) for a, b in zip(keep, (steps.theta, steps.m, steps.v))) and steps.t == 1
    assert torch.equal(plain.step(tokens, targets, plan, positions), steps.step(tokens, targets, plan, positions))
    assert torch.equal(plain.theta, steps.theta) and bool(steps.theta.isfinite().all())

"""The inner steps as they are used together: a decoder on the library's operators against the same decoder in plain operations,
and the example that alternates inner steps and outer rounds."""
import importlib.util
import os

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_param_layout():
    pytest.importorskip("torch")
    from paper_2606_22768_b200 import inner
    cfg = inner.DecoderConfig(vocab=100, width=48, layers=2, n_q_heads=3, n_kv_heads=1, head_dim=16, ffn=50)
    layout, P = inner.param_layout(cfg)
    spans = sorted((at, at + int(np.prod(shape))) for at, shape in layout.values())
    assert all(a % 32 == 0 for a, _ in spans) and P % 32 == 0 and spans[-1][1] <= P
    assert all(b <= c for (_, b), (c, _) in zip(spans, spans[1:]))
    assert layout["1.qkv"][1] == ((3 + 2) * 16, 48) and layout["0.up"][1] == (100, 48)


def _plain_logits(theta, tokens, lens, cfg):
    """The same decoder in fp64 with autograd, one worker and one sequence at a time, nothing quantised."""
    import torch
    from paper_2606_22768_b200 import inner
    layout, _ = inner.param_layout(cfg)
    out = []
    for m in range(theta.shape[0]):
        p = {name: theta[m, at:at + int(np.prod(shape))].view(shape) for name, (at, shape) in layout.items()}
        rms = lambda t, w: t / (t.square().mean(-1, keepdim=True) + cfg.eps).sqrt() * w  # noqa: E731
        logits, at = [], 0
        for n in lens:
            x = p["embed"][tokens[m, at:at + n]]
            at += n
            pos = torch.arange(n, device=x.device, dtype=torch.float64)
            freq = cfg.rope_base ** (-torch.arange(0, cfg.head_dim, 2, device=x.device, dtype=torch.float64) / cfg.head_dim)
            cos, sin = (pos[:, None] * freq).cos()[:, None], (pos[:, None] * freq).sin()[:, None]

            def rot(t):
                a, b = t.chunk(2, -1)
                return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

            for i in range(cfg.layers):
                h = rms(x, p[f"{i}.attn.pre"]) @ p[f"{i}.qkv"].T
                h = h.view(n, -1, cfg.head_dim)
                q, k, v = rot(h[:, :cfg.n_q_heads]), rot(h[:, cfg.n_q_heads:cfg.n_q_heads + cfg.n_kv_heads]), h[:, cfg.n_q_heads + cfg.n_kv_heads:]
                g = cfg.n_q_heads // cfg.n_kv_heads
                k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
                s = torch.einsum("ihd,jhd->hij", q, k) * cfg.head_dim ** -0.5
                s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), -float("inf"))
                y = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v).reshape(n, -1) @ p[f"{i}.out"].T
                x = x + cfg.res_scale * p[f"{i}.attn.gate"] * rms(y, p[f"{i}.attn.post"])
                a, b = (rms(x, p[f"{i}.mlp.pre"]) @ p[f"{i}.up"].T).chunk(2, -1)
                y = (torch.nn.functional.silu(a) * b) @ p[f"{i}.down"].T
                x = x + cfg.res_scale * p[f"{i}.mlp.gate"] * rms(y, p[f"{i}.mlp.post"])
            logits.append(rms(x, p["final"]) @ p["head"].T)
        out.append(torch.cat(logits))
    return torch.stack(out)


@pytest.mark.gpu
def test_decoder_against_plain():
    """Loss, logits and the gradient of every parameter.  bf16 activations (2^-9 relative each, a few dozen roundings in a row) and 8-bit
    checkpoints (a step of 2^-6 to 2^-7 of a group's largest value: about 1.5 % of the values' norm) against fp64: a few percent of each
    gradient's norm."""
    import torch
    import paper_2606_22768_b200 as fgd
    from paper_2606_22768_b200 import inner
    cfg = inner.DecoderConfig(vocab=96, width=128, layers=2, n_q_heads=4, n_kv_heads=2, head_dim=32, ffn=160)
    lens, K = [70, 1, 130, 33], 3
    rows = sum(lens)
    layout, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, 1)
    gen = torch.Generator().manual_seed(2)
    theta += (0.05 * torch.randn(theta.shape, generator=gen)).cuda()       # workers apart, norms and gates away from 1
    tokens = torch.randint(cfg.vocab, (K, rows), generator=gen).cuda()
    targets = torch.randint(cfg.vocab, (K, rows), generator=gen).cuda()
    targets[:, ::7] = -1
    plan = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens * K)]))
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    leaf = theta.clone().requires_grad_(True)
    logits = inner.decoder_logits(leaf, tokens, plan, positions, cfg)
    inner.worker_losses(logits, targets).sum().backward()
    ref = theta.double().requires_grad_(True)
    want = _plain_logits(ref, tokens, lens, cfg)
    lp = torch.log_softmax(want, -1)
    keep = targets >= 0
    loss = -(torch.gather(lp, 2, targets.clamp_min(0)[:, :, None])[:, :, 0] * keep).sum(1) / keep.sum(1)
    loss.sum().backward()
    assert torch.allclose(inner.worker_losses(logits, targets).detach().double(), loss.detach(), rtol=0.02)
    assert float((logits.detach().double() - want.detach()).norm() / want.detach().norm()) < 0.03
    for name, (at, shape) in layout.items():
        n = int(np.prod(shape))
        g, w = leaf.grad[:, at:at + n].double(), ref.grad[:, at:at + n]
        rel = float((g - w).norm() / w.norm())
        assert rel < 0.08, f"{name}: the gradient is {rel:.3f} of its norm off"
    fgd.fgd_attn_status(plan)


@pytest.mark.gpu
def test_example_learns():
    spec = importlib.util.spec_from_file_location("inner_and_outer", os.path.join(ROOT, "examples", "inner_and_outer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    history = ex.main(["--rounds", "4", "--inner", "15"])
    first, last = history[0], history[-1]
    assert last[1] < 0.8 * first[0], "four rounds of fifteen steps did not bring the loss down"
    assert all(np.isfinite(v) for row in history for v in row)
    assert all(0.0 <= row[3] <= 1.0 for row in history)

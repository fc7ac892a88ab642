"""K workers train a small decoder on one GPU: H inner steps on the library's operators, then one outer round, over and over.

    python examples/inner_and_outer.py [--workers 4] [--rounds 5] [--inner 20]

Every worker sees its own packed sequences of different lengths from one synthetic language (a fixed random successor table with
noise).  After every round: the workers' losses, the L2 consensus distance, and the JS distance between each worker's predictions and those of
the parameter-averaged model on a held-out batch.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2606_22768_b200 as fgd
from paper_2606_22768_b200 import inner
from paper_2606_22768_b200.round import OuterRound


def batch(rng, K, lens, vocab, successor):
    """tokens and targets [K, sum(lens)]: the next token is the successor of this one, or (one in ten) any token."""
    rows = sum(lens)
    tokens, targets = np.zeros((K, rows), dtype=np.int64), np.full((K, rows), -1, dtype=np.int64)
    for m in range(K):
        at = 0
        for n in lens:
            s = [int(rng.integers(vocab))]
            for _ in range(n):
                s.append(int(successor[s[-1]]) if rng.random() > 0.1 else int(rng.integers(vocab)))
            tokens[m, at:at + n], targets[m, at:at + n] = s[:n], s[1:]
            at += n
    return torch.from_numpy(tokens).cuda(), torch.from_numpy(targets).cuda()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=5)
    ap.add_argument("--inner", type=int, default=20)
    ap.add_argument("--lr", type=float, default=2e-3)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    K, cfg = a.workers, inner.DecoderConfig()
    _, P = inner.param_layout(cfg)
    theta = torch.zeros((K, P), device="cuda")
    inner.init_params(theta, cfg, a.seed)
    local, momentum = theta.clone(), torch.zeros_like(theta)
    steps, drv = inner.InnerSteps(local, cfg, lr=a.lr), OuterRound(K, P)
    rng = np.random.default_rng(a.seed)
    successor = rng.permutation(cfg.vocab)
    lens = [180, 65, 1, 138]
    rows = sum(lens)
    cu = np.concatenate([[0], np.cumsum(lens * K)])
    plan = fgd.AttnPlan(cu)
    positions = torch.cat([torch.arange(n) for n in lens * K]).cuda()
    held_tokens, _ = batch(rng, 1, lens, cfg.vocab, successor)
    one = fgd.AttnPlan(np.concatenate([[0], np.cumsum(lens)]))
    history = []
    for r in range(a.rounds):
        drv.launch_mix1(fgd.MixDesc.mean(K), theta)                # side stream, beside the inner steps
        local.copy_(theta)
        losses = [steps.step(*batch(rng, K, lens, cfg.vocab, successor), plan, positions) for _ in range(a.inner)]
        drv.step(fgd.MixDesc.ring(K), local, theta, momentum, theta, 0.7, 0.9)
        cd, _ = fgd.fgd_cd_finalize(drv.cd_sumsq.cpu().numpy())
        with torch.no_grad():
            work = inner.decoder_logits(theta, held_tokens.expand(K, -1).contiguous(), plan, positions, cfg).float().contiguous()
            mean = inner.decoder_logits(theta.mean(0, keepdim=True), held_tokens, one, positions[:rows], cfg).float().view(rows, cfg.vocab)
        top = 100
        idx = torch.empty((rows, top), dtype=torch.int32, device="cuda")
        d_js, worker_js = torch.empty((K, rows), dtype=torch.float64, device="cuda"), torch.empty(K, dtype=torch.float64, device="cuda")
        fgd.fgd_js_distance(work, mean, idx, d_js, worker_js, top_k=top)
        fgd.fgd_attn_status(plan)
        history.append((float(losses[0].mean()), float(losses[-1].mean()), cd, float(worker_js.mean())))
        print(f"round {r}: loss {history[-1][0]:.4f} -> {history[-1][1]:.4f}   CD_L2 {cd:.4f}   CD_JS {history[-1][3]:.4f}", flush=True)
    return history


if __name__ == "__main__":
    main()

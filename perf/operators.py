"""The training operators of a worker's inner step, as cases that can be timed and compared.

Every case is one pass through one operator: the framework's kernels where ``own`` is true, the same
operator in elementary torch operations (fp32 throughout, rounded once at the end) where it is false.

Operators and what a pass is:
  attn      causal attention over packed sequences with grouped heads: the forward pass, or the training
            step (forward and backward);
  norm      a block's output normalised, gated, scaled and added to the residual stream, and the
            norm that the next block reads: the forward pass, or the backward pass from the stream as
            it was stored, for the K workers' weights at once;
  act8      activations saved in 8 bits and read back;
  swiglu8   SwiGLU with its inputs kept in 8 bits: forward and backward from the checkpoint.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GROUP = 32          # values that share one scale in an 8-bit checkpoint
EPS = 1e-5          # of the norms


# --------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a handful of short prompts, one of a single token: launch latency
        {"name": "attn_fwd_few", "op": "attn", "train": False, "lens": "17,1,110", "hq": 4, "hk": 2, "d": 64, "dtype": "f16"},
        # documents of different lengths packed into one evaluation batch, none a multiple of a tile
        {"name": "attn_fwd_packed", "op": "attn", "train": False, "lens": "1024,2011,517,130,1499,733,1,1250,1027", "hq": 16, "hk": 4, "d": 128,
         "dtype": "bf16"},
        # one long document
        {"name": "attn_fwd_long", "op": "attn", "train": False, "lens": "16384", "hq": 16, "hk": 4, "d": 128, "dtype": "bf16"},
        # a few short sequences in training, an empty one among them; head width and group size that fill no tile
        {"name": "attn_train_few", "op": "attn", "train": True, "lens": "200,56,1,0,31", "hq": 6, "hk": 2, "d": 80, "dtype": "bf16"},
        # a training batch of sixteen sequences of 1024 tokens, one key head per query head
        {"name": "attn_train_batch", "op": "attn", "train": True, "lens": ",".join(["1024"] * 16), "hq": 16, "hk": 16, "d": 64, "dtype": "bf16"},
        # long-context training
        {"name": "attn_train_long", "op": "attn", "train": True, "lens": "8192", "hq": 16, "hk": 4, "d": 128, "dtype": "bf16"},
        # a short evaluation batch at an odd width: launch latency
        {"name": "norm_fwd_small", "op": "norm", "backward": False, "workers": 1, "rows": 33, "width": 1001, "gate": "row", "dtype": "f16"},
        # eight workers' batches in one call, per-channel gate
        {"name": "norm_bwd_workers", "op": "norm", "backward": True, "workers": 8, "rows": 4096, "width": 2048, "gate": "row", "dtype": "bf16"},
        # fp32 activations with a gate for every element, odd row count
        {"name": "norm_fwd_gated", "op": "norm", "backward": False, "workers": 1, "rows": 5003, "width": 4096, "gate": "full", "dtype": "f32"},
        # a small activation of odd width through the checkpoint: launch latency
        {"name": "act8_small", "op": "act8", "rows": 40, "width": 777, "dtype": "bf16"},
        # a block's activations saved for the backward pass and read back
        {"name": "act8_large", "op": "act8", "rows": 32768, "width": 4096, "dtype": "bf16"},
        # the MLP of one block over a training batch
        {"name": "swiglu8_train", "op": "swiglu8", "rows": 16384, "width": 5632, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn", "norm", "act8", "swiglu8"))
    if op == "attn":
        train = rng.random() < 0.5
        most = 8192 if train else 16384
        hk = rng.choice((1, 2, 3, 4, 8))
        group = rng.choice((1, 2, 3, 4))
        hq = min(hk * group, 16) // hk * hk
        total, lens = _log(rng, 64, most), []
        while sum(lens) < total:
            lens.append(min(total - sum(lens), rng.choice((_log(rng, 1, total), _log(rng, 64, 4 * total)))))
            if rng.random() < 0.1:
                lens.append(rng.choice((0, 1)))
        lens = lens[:24]
        while len(lens) * max(lens) ** 2 * hq > 16 * most ** 2:      # the plain form pads every sequence to the longest
            lens.pop()
        return {"op": op, "train": train, "lens": ",".join(map(str, lens)), "hq": hq, "hk": hk, "d": rng.choice((32, 64, 72, 80, 96, 112, 128)),
                "dtype": rng.choice(("bf16", "f16"))}
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    wide = 2 if dtype == "f32" else 1
    width = _log(rng, 64, 8192)
    width += rng.choice((0, 1, -width % 8, -width % 64))
    width = min(width, 8192)
    if op == "norm":
        workers = rng.choice((1, 1, 2, 4, 8))
        rows = _log(rng, 1, max(1, 8 * 4096 * 2048 // (width * workers * wide)))
        return {"op": op, "backward": rng.random() < 0.6, "workers": workers, "rows": rows, "width": width, "gate": rng.choice(("none", "row", "full")), "dtype": dtype}
    rows = _log(rng, 1, max(1, 16384 * 5632 // (width * wide)))
    return {"op": op, "rows": rows, "width": width, "dtype": dtype}


# --------------------------------------------------------------------------------------- inputs
def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _randn(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"] == "attn":
        lens = _lens(case)
        T, hq, hk, d = sum(lens), case["hq"], case["hk"], case["d"]
        # q, k and v are slices of one projection's output, as a block's fused projection leaves them
        qkv = _randn(gen, (T, hq + 2 * hk, d), dt)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        s["scale"] = 1.0 / math.sqrt(d)
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        s["cu"] = cu
        s["o"] = torch.empty((T, hq, d), dtype=dt, device="cuda")
        s["lse"] = torch.empty((hq, T), dtype=torch.float32, device="cuda")
        if case["train"]:
            s["do"] = _randn(gen, (T, hq, d), dt)
            s["delta"] = torch.empty((hq, T), dtype=torch.float32, device="cuda")
            dqkv = torch.empty_like(qkv)
            s["dq"], s["dk"], s["dv"] = dqkv[:, :hq], dqkv[:, hq:hq + hk], dqkv[:, hq + hk:]
        # padded layout of the packed tokens: token of (sequence, position), and back
        L = max(lens)
        start = torch.tensor(cu[:-1], device="cuda")
        length = torch.tensor(lens, device="cuda")
        at = torch.arange(L, device="cuda")
        s["valid"] = at[None, :] < length[:, None]
        s["token"] = torch.where(s["valid"], start[:, None] + at[None, :], 0)
        if own:
            import paper_2606_22768_b200 as fgd
            s["plan"] = fgd.AttnPlan(cu)
        return s
    R, H = case["rows"], case["width"]
    if case["op"] == "norm":
        K = case["workers"]
        T = K * R
        s["x"] = _randn(gen, (T, H), dt, 2.0)        # backward: the stream as the forward pass stored it
        s["y"] = _randn(gen, (T, H), dt)
        s["w_post"] = 1.0 + _randn(gen, (K, H), torch.float32, 0.1)
        s["w_pre"] = 1.0 + _randn(gen, (K, H), torch.float32, 0.1)
        s["gate"] = {"none": lambda: None, "row": lambda: _randn(gen, (K, H), torch.float32, 0.5), "full": lambda: _randn(gen, (T, H), dt, 0.5)}[case["gate"]]()
        s["scale"] = 0.5
        if case["backward"]:
            s["dn"], s["dres"] = _randn(gen, (T, H), dt), _randn(gen, (T, H), dt)
            s["dx"], s["dy"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["dw_post"], s["dw_pre"] = torch.empty_like(s["w_post"]), torch.empty_like(s["w_pre"])
            s["dgate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
        else:
            s["x_new"], s["n"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        return s
    # activations with a few channels far above the rest
    spread = torch.exp(0.5 * torch.randn((2 * H if case["op"] == "swiglu8" else H,), generator=gen, device="cuda"))
    if case["op"] == "act8":
        s["x"] = (_randn(gen, (R, H), torch.float32) * spread).to(dt)
        s["back"] = torch.empty_like(s["x"])
        s["q8"] = torch.empty((R, H), dtype=torch.int8, device="cuda")
        s["e8"] = torch.empty((R, -(-H // GROUP)), dtype=torch.uint8, device="cuda")
        return s
    s["gu"] = (_randn(gen, (R, 2 * H), torch.float32) * spread).to(dt)
    s["dh"] = _randn(gen, (R, H), dt)
    s["h"], s["h_again"], s["dgu"] = torch.empty_like(s["dh"]), torch.empty_like(s["dh"]), torch.empty_like(s["gu"])
    s["q8"] = torch.empty((R, 2 * H), dtype=torch.int8, device="cuda")
    s["e8"] = torch.empty((R, 2 * -(-H // GROUP)), dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------------------------------- passes
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attn": _own_attn, "norm": _own_norm, "act8": _own_act8, "swiglu8": _own_swiglu8}[op](s)
    return {"attn": _plain_attn, "norm": _plain_norm, "act8": _plain_act8, "swiglu8": _plain_swiglu8}[op](s)


def _own_attn(s):
    import paper_2606_22768_b200 as fgd
    fgd.fgd_attn_forward(s["plan"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["scale"])
    if not s["case"]["train"]:
        return {"o": s["o"], "lse": s["lse"]}
    fgd.fgd_attn_backward(s["plan"], s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["delta"], s["dq"], s["dk"], s["dv"], s["scale"])
    return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _own_norm(s):
    import paper_2606_22768_b200 as fgd
    if not s["case"]["backward"]:
        fgd.fgd_block_norm_forward(s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["x_new"], s["n"], EPS, s["scale"])
        return {"x_new": s["x_new"], "n": s["n"]}
    fgd.fgd_block_norm_backward(s["dn"], s["dres"], s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"], s["dx"], s["dy"], s["dgate"], s["dw_post"], s["dw_pre"],
                                EPS, s["scale"])
    return {"dx": s["dx"], "dy": s["dy"], "dgate": s["dgate"], "dw_post": s["dw_post"], "dw_pre": s["dw_pre"]}


def _own_act8(s):
    import paper_2606_22768_b200 as fgd
    fgd.fgd_act_save8(s["x"], s["q8"], s["e8"])
    fgd.fgd_act_load8(s["q8"], s["e8"], s["back"])
    return {"back": s["back"]}


def _own_swiglu8(s):
    import paper_2606_22768_b200 as fgd
    fgd.fgd_swiglu8_forward(s["gu"], s["h"], s["q8"], s["e8"])
    fgd.fgd_swiglu8_backward(s["dh"], s["q8"], s["e8"], s["dgu"], s["h_again"])
    return {"h": s["h"], "dgu": s["dgu"], "h_again": s["h_again"]}


def _plain_attn(s):
    c = s["case"]
    hq, hk, d, dt = c["hq"], c["hk"], c["d"], s["q"].dtype
    B, L = s["valid"].shape
    valid, token = s["valid"], s["token"]

    def padded(x):        # [T, heads, d] -> [B, hk, heads / hk, L, d]; zeros behind a sequence's end
        p = x.float()[token].masked_fill(~valid[:, :, None, None], 0.0)
        return p.view(B, L, hk, -1, d).permute(0, 2, 3, 1, 4)

    def packed(x, heads):  # and back
        return x.permute(0, 3, 1, 2, 4).reshape(B, L, heads, d)[valid].to(dt)

    q, k, v = padded(s["q"]), padded(s["k"]), padded(s["v"])
    future = torch.ones((L, L), dtype=torch.bool, device="cuda").triu(1)
    p = (q @ k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(future, float("-inf"))
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / total
    lse = (top + total.log()).reshape(B, hq, L).permute(1, 0, 2)[:, valid]
    out = {"o": packed(o, hq), "lse": lse}
    if c["train"]:
        do = padded(s["do"])
        p.div_(total)
        dv = (p.transpose(-1, -2) @ do).sum(2, keepdim=True)
        ds = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
        dk = (ds.transpose(-1, -2) @ q).sum(2, keepdim=True)
        out |= {"dq": packed(ds @ k, hq), "dk": packed(dk, hk), "dv": packed(dv, hk)}
    return out


def _plain_norm(s):
    c = s["case"]
    K, R, H, dt = c["workers"], c["rows"], c["width"], s["x"].dtype
    x, y = s["x"].float().view(K, R, H), s["y"].float().view(K, R, H)
    wa, wb = s["w_post"][:, None], s["w_pre"][:, None]
    g = {"none": lambda: 1.0, "row": lambda: s["gate"][:, None], "full": lambda: s["gate"].float().view(K, R, H)}[c["gate"]]()
    ry = (y.square().mean(-1, keepdim=True) + EPS).rsqrt()
    yh = y * ry
    if not c["backward"]:
        xn = x + s["scale"] * g * (yh * wa)
        rx = (xn.square().mean(-1, keepdim=True) + EPS).rsqrt()
        return {"x_new": xn.to(dt).view(-1, H), "n": (xn * rx * wb).to(dt).view(-1, H)}
    dn, dres = s["dn"].float().view(K, R, H), s["dres"].float().view(K, R, H)
    rx = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xh = x * rx
    a = dn * wb
    dx = dres + rx * (a - xh * (a * xh).mean(-1, keepdim=True))
    t = s["scale"] * dx * g
    b = t * wa
    dy = ry * (b - yh * (b * yh).mean(-1, keepdim=True))
    dg = s["scale"] * dx * yh * wa
    dgate = {"none": lambda: None, "row": lambda: dg.sum(1), "full": lambda: dg.to(dt).view(-1, H)}[c["gate"]]()
    return {"dx": dx.to(dt).view(-1, H), "dy": dy.to(dt).view(-1, H), "dgate": dgate, "dw_post": (t * yh).sum(1), "dw_pre": (dn * xh).sum(1)}


def _kept8(x):
    """The values an 8-bit checkpoint of x stands for: groups of 32 along the row, a power-of-two step each."""
    R, H = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -H % GROUP)).view(R, -1, GROUP)
    top = g.abs().amax(-1, keepdim=True)
    step = ((torch.frexp(top)[1] - 7).clamp_min(-126) + 127).to(torch.int32).bitwise_left_shift(23).view(torch.float32)   # the power of two itself
    return ((g / step).round().clamp(-127, 127) * step).view(R, -1)[:, :H]


def _plain_act8(s):
    return {"back": _kept8(s["x"]).to(s["x"].dtype)}


def _plain_swiglu8(s):
    H, dt = s["case"]["width"], s["gu"].dtype
    g, u = s["gu"][:, :H].float(), s["gu"][:, H:].float()
    h = g / (1 + (-g).exp()) * u
    g, u = _kept8(s["gu"][:, :H]), _kept8(s["gu"][:, H:])
    sg = 1 / (1 + (-g).exp())
    dh = s["dh"].float()
    dg = dh * u * sg * (1 + g * (1 - sg))
    du = dh * g * sg
    return {"h": h.to(dt), "dgu": torch.cat((dg, du), 1).to(dt), "h_again": (g * sg * u).to(dt)}


# --------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "norm": _exact_norm, "act8": _exact_act8, "swiglu8": _exact_swiglu8}[case["op"]](s)


def _exact_attn(s):
    c, cu = s["case"], s["cu"]
    hq, hk = c["hq"], c["hk"]
    out = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), "lse": torch.zeros((hq, cu[-1]), dtype=torch.float64, device="cuda")}
    if c["train"]:
        out |= {"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"}
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        keep = torch.tril(torch.ones((b - a, b - a), dtype=torch.bool, device="cuda"))
        for h in range(hq):
            g = h * hk // hq
            q, k, v = s["q"][a:b, h].double(), s["k"][a:b, g].double(), s["v"][a:b, g].double()
            score = torch.where(keep, s["scale"] * (q @ k.T), -math.inf)
            lse = torch.logsumexp(score, 1)
            p = torch.exp(score - lse[:, None])
            o = p @ v
            out["o"][a:b, h], out["lse"][h, a:b] = o, lse
            if c["train"]:
                do = s["do"][a:b, h].double()
                ds = p * (do @ v.T - (do * o).sum(1)[:, None]) * s["scale"]
                out["dq"][a:b, h] = ds @ k
                out["dk"][a:b, g] += ds.T @ q
                out["dv"][a:b, g] += p.T @ do
    return out


def _exact_norm(s):
    c = s["case"]
    K, R, H = c["workers"], c["rows"], c["width"]
    x, y, wa, wb, gate = (None if s[n] is None else s[n].double() for n in ("x", "y", "w_post", "w_pre", "gate"))
    rms = lambda t: t / torch.sqrt(torch.mean(t * t, -1, keepdim=True) + EPS)  # noqa: E731

    def joined(y, wa, gate):      # what the block adds to the stream
        u = rms(y.view(K, R, H)) * wa.view(K, 1, H)
        if gate is not None:
            u = u * (gate.view(K, 1, H) if c["gate"] == "row" else gate.view(K, R, H))
        return s["scale"] * u

    if not c["backward"]:
        xn = x.view(K, R, H) + joined(y, wa, gate)
        return {"x_new": xn.view(-1, H), "n": (rms(xn) * wb.view(K, 1, H)).view(-1, H)}
    for leaf in (x, y, wa, wb, gate):
        if leaf is not None:
            leaf.requires_grad_(True)
    n = rms(x.view(K, R, H)) * wb.view(K, 1, H)
    (n * s["dn"].double().view(K, R, H)).sum().backward()
    dx = x.grad + s["dres"].double()
    (joined(y, wa, gate) * dx.view(K, R, H)).sum().backward()
    return {"dx": dx, "dy": y.grad, "dgate": None if gate is None else gate.grad, "dw_post": wa.grad, "dw_pre": wb.grad}


def _exact_kept8(x):
    """As an 8-bit checkpoint keeps x: the step is the power of two just above 1/128 of the group's largest magnitude."""
    R, H = x.shape
    out = torch.zeros((R, -(-H // GROUP) * GROUP), dtype=torch.float64, device=x.device)
    out[:, :H] = x.double()
    groups = out.view(R, -1, GROUP)
    largest = groups.abs().max(-1).values
    mantissa_off = largest.view(torch.int64) & (0x7FF << 52)                   # the power of two at or below it
    step = (mantissa_off.view(torch.float64) / 64).clamp_min(2.0 ** -126).unsqueeze(-1)
    groups.copy_(torch.clamp(torch.round(groups / step), -127, 127) * step)
    return out[:, :H]


def _exact_act8(s):
    return {"back": _exact_kept8(s["x"])}


def _exact_swiglu8(s):
    H = s["case"]["width"]
    full = s["gu"].double()
    h = torch.sigmoid(full[:, :H]) * full[:, :H] * full[:, H:]
    del full
    g = _exact_kept8(s["gu"][:, :H]).requires_grad_(True)
    u = _exact_kept8(s["gu"][:, H:]).requires_grad_(True)
    again = torch.sigmoid(g) * g * u
    again.backward(s["dh"].double())
    return {"h": h, "dgu": torch.cat((g.grad, u.grad), 1), "h_again": again.detach()}


# --------------------------------------------------------------------------------------- work
def work(case):
    """Bytes and operations one pass cannot do without."""
    b = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "attn":
        lens = _lens(case)
        T, hq, hk, d = sum(lens), case["hq"], case["hk"], case["d"]
        pairs = sum(n * (n + 1) // 2 for n in lens) * hq
        bytes_ = T * d * (2 * hq + 2 * hk) * b + 4 * T * hq          # q, k, v, o, lse
        flops = 4 * d * pairs
        if case["train"]:
            bytes_ += T * d * (2 * hq + 2 * hk) * b                  # do; dq, dk, dv
            flops += 10 * d * pairs
        return {"bytes": bytes_, "flops": flops}
    R, H = case["rows"], case["width"]
    if case["op"] == "norm":
        K = case["workers"]
        n = K * R * H
        gate = {"none": 0, "row": 4 * K * H, "full": n * b}[case["gate"]]
        if not case["backward"]:
            return {"bytes": 4 * n * b + 8 * K * H + gate, "flops": 10 * n}               # x, y; x_new, n; the weights
        return {"bytes": 6 * n * b + 16 * K * H + 2 * gate, "flops": 25 * n}              # dn, dres, x, y; dx, dy; the weights and their gradients
    groups = -(-H // GROUP)
    if case["op"] == "act8":
        return {"bytes": R * (2 * H * b + H + groups), "flops": 4 * R * H}
    return {"bytes": R * (7 * H * b + 2 * H + 2 * groups), "flops": 30 * R * H}   # gu, h, dh, dgu, h again; the checkpoint

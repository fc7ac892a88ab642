"""More operators of a worker's inner step, as cases that can be timed and compared: what stands between the tokens and the attention,
and dropout.

Every case is one pass through one operator: the framework's kernels where ``own`` is true, the same operator in elementary torch
operations (fp32 throughout, rounded once at the end) where it is false.

Operators and what a pass is:
  rope      queries and keys normalised per head (or not) and rotated by their positions: the forward pass, or the training step
            (forward and backward), for the K workers' norm weights at once;
  embed     the lookup of the K workers' scaled embeddings: the forward pass, or the training step (lookup and the gradient of the whole table);
  dropout   dropout from a counter-based generator: the forward pass, or the training step (the same mask on the activations and on the
            gradient).

The generator of dropout is Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011):
counter (column / 4, row, low and high word of the offset), key (low and high word of the seed); word column % 4 belongs to the value.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5          # of the norms
ROUNDS = 7          # of the generator


# --------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a handful of tokens in evaluation, the last of them a single one's step: launch latency
        {"name": "rope_fwd_few", "op": "rope", "train": False, "workers": 1, "rows": 3, "hq": 4, "hk": 2, "d": 64, "rot": 64, "norm": True, "inter": False,
         "seq": 512, "dtype": "f16"},
        # rotation alone over an evaluation batch
        {"name": "rope_fwd_plain", "op": "rope", "train": False, "workers": 1, "rows": 16384, "hq": 16, "hk": 4, "d": 128, "rot": 128, "norm": False, "inter": False,
         "seq": 4096, "dtype": "bf16"},
        # eight workers' training batches
        {"name": "rope_train_workers", "op": "rope", "train": True, "workers": 8, "rows": 4096, "hq": 16, "hk": 4, "d": 128, "rot": 128, "norm": True, "inter": False,
         "seq": 2048, "dtype": "bf16"},
        # fp32, heads of 80 of which 48 channels turn, neighbouring pairs, an odd number of tokens
        {"name": "rope_train_partial", "op": "rope", "train": True, "workers": 1, "rows": 5003, "hq": 6, "hk": 2, "d": 80, "rot": 48, "norm": True, "inter": True,
         "seq": 777, "dtype": "f32"},
        # a short evaluation batch at an odd width and vocabulary: launch latency
        {"name": "embed_fwd_small", "op": "embed", "train": False, "workers": 1, "rows": 33, "vocab": 257, "width": 1001, "pad": False, "dtype": "f16"},
        # four workers' batches of tokens as text has them
        {"name": "embed_fwd_workers", "op": "embed", "train": False, "workers": 4, "rows": 8192, "vocab": 32000, "width": 2048, "pad": False, "dtype": "bf16"},
        # training of the small decoder: a vocabulary of bytes, so that every token repeats
        {"name": "embed_train_bytes", "op": "embed", "train": True, "workers": 4, "rows": 384, "vocab": 256, "width": 256, "pad": False, "dtype": "bf16"},
        # training of four workers, sequences padded at their ends
        {"name": "embed_train_workers", "op": "embed", "train": True, "workers": 4, "rows": 8192, "vocab": 32000, "width": 2048, "pad": True, "dtype": "bf16"},
        # one long batch over a vocabulary of odd size
        {"name": "embed_train_long", "op": "embed", "train": True, "workers": 1, "rows": 65536, "vocab": 50257, "width": 1536, "pad": False, "dtype": "f16"},
        # a small activation of odd width: launch latency
        {"name": "dropout_small", "op": "dropout", "train": False, "rows": 40, "width": 777, "p": 0.1, "dtype": "bf16"},
        # a block's output in training and its gradient
        {"name": "dropout_train", "op": "dropout", "train": True, "rows": 32768, "width": 4096, "p": 0.1, "dtype": "bf16"},
        # fp32 activations whose rows start off the 16-byte boundaries
        {"name": "dropout_train_odd", "op": "dropout", "train": True, "rows": 5003, "width": 4097, "p": 0.25, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "embed", "dropout"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    wide = 2 if dtype == "f32" else 1
    train = rng.random() < 0.6
    if op == "rope":
        hk = rng.choice((1, 2, 3, 4, 8))
        hq = hk * rng.choice((1, 2, 3, 4))
        d = rng.choice((32, 64, 64, 72, 80, 96, 112, 128, 128, 192, 256))
        rot = d if rng.random() < 0.7 else max(2, d // rng.choice((2, 4)) // 2 * 2)
        workers = rng.choice((1, 1, 2, 4, 8))
        rows = _log(rng, 1, max(1, 32768 * 20 * 128 // ((hq + hk) * d * wide * workers)))
        return {"op": op, "train": train, "workers": workers, "rows": rows, "hq": hq, "hk": hk, "d": d, "rot": rot, "norm": rng.random() < 0.7,
                "inter": rng.random() < 0.3, "seq": _log(rng, 1, 8192), "dtype": dtype}
    if op == "embed":
        workers = rng.choice((1, 1, 2, 4, 8))
        vocab = _log(rng, 64, 131072)
        width = _log(rng, 64, 4096)
        width += rng.choice((0, 1, -width % 8, -width % 64))
        width = max(1, min(width, 4 * 32000 * 2048 // (workers * vocab)))
        rows = _log(rng, 1, max(1, min(65536 // workers, 4 * 8192 * 2048 // (width * wide * workers))))
        return {"op": op, "train": train, "workers": workers, "rows": rows, "vocab": vocab, "width": width, "pad": rng.random() < 0.3, "dtype": dtype}
    width = _log(rng, 64, 8192)
    width += rng.choice((0, 1, -width % 8, -width % 64))
    rows = _log(rng, 1, max(1, 32768 * 4096 // (width * wide)))
    return {"op": op, "train": train, "rows": rows, "width": width, "p": rng.choice((0.05, 0.1, 0.2, 0.5)), "dtype": dtype}


# --------------------------------------------------------------------------------------- inputs
def _randn(gen, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"] == "rope":
        K, R, hq, hk, d, rot = (case[n] for n in ("workers", "rows", "hq", "hk", "d", "rot"))
        T = K * R
        # q and k are slices of one projection's output, as a block's fused projection leaves them; their gradients come from attention
        qkv = _randn(gen, (T, hq + 2 * hk, d), dt, 1.5)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        s["q_out"], s["k_out"] = torch.empty((T, hq, d), dtype=dt, device="cuda"), torch.empty((T, hk, d), dtype=dt, device="cuda")
        s["w_q"] = s["w_k"] = s["dw_q"] = s["dw_k"] = None
        if case["norm"]:
            s["w_q"], s["w_k"] = (1.0 + _randn(gen, (K, d), torch.float32, 0.1) for _ in range(2))
            s["dw_q"], s["dw_k"] = torch.empty_like(s["w_q"]), torch.empty_like(s["w_k"])
        # the tables of the rotation, made once; angles in 64 bits
        at = torch.arange(case["seq"], dtype=torch.float64, device="cuda")
        freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        angle = at[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        first = int(torch.randint(case["seq"], (1,), generator=gen, device="cuda"))
        s["positions"] = (torch.arange(T, device="cuda") + first) % case["seq"]      # sequences packed one behind the other
        if case["train"]:
            s["dq_out"], s["dk_out"] = _randn(gen, (T, hq, d), dt), _randn(gen, (T, hk, d), dt)
            dqkv = torch.empty_like(qkv)
            s["dq"], s["dk"] = dqkv[:, :hq], dqkv[:, hq:hq + hk]
        return s
    if case["op"] == "embed":
        K, R, V, W = (case[n] for n in ("workers", "rows", "vocab", "width"))
        # tokens as text has them: the n-th commonest about 1 / n as often as the first
        u = torch.rand((K, R), generator=gen, device="cuda", dtype=torch.float64)
        tokens = ((V + 1.0) ** u).long().sub_(1).clamp_(0, V - 1)
        if case["pad"]:      # each worker's batch ends in padding
            tokens[:, R - R // 10:] = -1
        s["tokens"] = tokens
        s["table"] = _randn(gen, (K, V, W), torch.float32, 0.02)
        s["scale"] = math.sqrt(W)
        s["out"] = torch.empty((K * R, W), dtype=dt, device="cuda")
        if case["train"]:
            s["dout"] = _randn(gen, (K * R, W), dt)
            s["dtable"] = torch.empty_like(s["table"])
        return s
    R, W = case["rows"], case["width"]
    s["x"] = _randn(gen, (R, W), dt)
    s["out"] = torch.empty_like(s["x"])
    draw_ = torch.randint(2 ** 62, (2,), generator=gen, device="cuda").tolist()
    s["seed"], s["offset"] = draw_[0], draw_[1] % 2 ** 40
    if case["train"]:
        s["dout"] = _randn(gen, (R, W), dt)
        s["dx"] = torch.empty_like(s["x"])
    return s


# --------------------------------------------------------------------------------------- passes
def run(s):
    op = s["case"]["op"]
    if own:
        return {"rope": _own_rope, "embed": _own_embed, "dropout": _own_dropout}[op](s)
    return {"rope": _plain_rope, "embed": _plain_embed, "dropout": _plain_dropout}[op](s)


def _own_rope(s):
    import paper_2606_22768_b200 as fgd
    inter = s["case"]["inter"]
    fgd.fgd_qk_rope_forward(s["q"], s["k"], s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], s["q_out"], s["k_out"], EPS, inter)
    out = {"q_out": s["q_out"], "k_out": s["k_out"]}
    if s["case"]["train"]:
        fgd.fgd_qk_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], s["w_q"], s["w_k"], s["cos"], s["sin"], s["positions"], s["dq"], s["dk"], s["dw_q"],
                                 s["dw_k"], EPS, inter)
        out |= {"dq": s["dq"], "dk": s["dk"], "dw_q": s["dw_q"], "dw_k": s["dw_k"]}
    return out


def _own_embed(s):
    import paper_2606_22768_b200 as fgd
    fgd.fgd_embed_forward(s["tokens"], s["table"], s["out"], s["scale"])
    if not s["case"]["train"]:
        return {"out": s["out"]}
    fgd.fgd_embed_backward(s["tokens"], s["dout"], s["dtable"], s["scale"])
    return {"out": s["out"], "dtable": s["dtable"]}


def _own_dropout(s):
    import paper_2606_22768_b200 as fgd
    p = s["case"]["p"]
    fgd.fgd_dropout(s["x"], s["out"], p, s["seed"], s["offset"])
    if not s["case"]["train"]:
        return {"out": s["out"]}
    fgd.fgd_dropout(s["dout"], s["dx"], p, s["seed"], s["offset"])
    return {"out": s["out"], "dx": s["dx"]}


def _plain_rope(s):
    c = s["case"]
    K, R, d, rot, dt = c["workers"], c["rows"], c["d"], c["rot"], s["q"].dtype
    cos, sin = s["cos"][s["positions"]][:, None], s["sin"][s["positions"]][:, None]

    def pairs(x):
        return (x[..., 0:rot:2], x[..., 1:rot:2]) if c["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])

    def joined(a, b, rest):
        return torch.cat((torch.stack((a, b), -1).flatten(-2) if c["inter"] else torch.cat((a, b), -1), rest), -1)

    def normed(x, w):
        """x, its inverse root mean square and the weights, for every row"""
        x = x.float()
        if w is None:
            return x, None, None
        return x, (x.square().mean(-1, keepdim=True) + EPS).rsqrt(), w.repeat_interleave(R, 0)[:, None]

    out = {}
    for n in "qk":
        x, r, w = normed(s[n], s["w_" + n])
        z = x if r is None else x * r * w
        a, b = pairs(z)
        out[n + "_out"] = joined(a * cos - b * sin, b * cos + a * sin, z[..., rot:]).to(dt)
        if c["train"]:
            dy = s[f"d{n}_out"].float()
            a, b = pairs(dy)
            dz = joined(a * cos + b * sin, b * cos - a * sin, dy[..., rot:])
            dw = None
            if r is not None:
                xh = x * r
                dw = (dz * xh).view(K, -1, d).sum(1)
                g = dz * w
                dz = r * (g - xh * (g * xh).mean(-1, keepdim=True))
            out |= {"d" + n: dz.to(dt), "dw_" + n: dw}
    return out


def _plain_embed(s):
    tokens, table, dt = s["tokens"], s["table"], s["out"].dtype
    K, V, W = table.shape
    row = (tokens + V * torch.arange(K, device="cuda")[:, None]).flatten()
    real = (tokens >= 0).flatten()
    rows = table.view(K * V, W)[row.clamp_min(0)] * s["scale"]
    out = {"out": rows.masked_fill_(~real[:, None], 0.0).to(dt)}
    if s["case"]["train"]:
        d = torch.zeros((K * V, W), dtype=torch.float32, device="cuda")
        d.index_add_(0, row[real], s["dout"][real].float())
        out["dtable"] = d.mul_(s["scale"]).view(K, V, W)
    return out


def _philox(seed, offset, rows, groups):
    """[rows, groups, 4] random words as int64, of the counters (group, row, offset)."""
    low = 0xFFFFFFFF
    c = [torch.arange(groups, device="cuda")[None, :].expand(rows, -1), torch.arange(rows, device="cuda")[:, None].expand(-1, groups),
         torch.tensor(offset & low, device="cuda"), torch.tensor(offset >> 32 & low, device="cuda")]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(ROUNDS):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57      # whole products: the bits of 64 are kept, whatever their sign says
        c = [(q >> 32 & low) ^ c[1] ^ k0, q & low, (p >> 32 & low) ^ c[3] ^ k1, p & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(torch.broadcast_tensors(*c), -1)


def _plain_dropout(s):
    c = s["case"]
    R, W, p, dt = c["rows"], c["width"], c["p"], s["x"].dtype
    keep = (_philox(s["seed"], s["offset"], R, -(-W // 4)) >= round(p * 2 ** 32)).view(R, -1)[:, :W]
    scale = 1.0 / (1.0 - p)
    out = {"out": torch.where(keep, s["x"].float() * scale, 0.0).to(dt)}
    if c["train"]:
        out["dx"] = torch.where(keep, s["dout"].float() * scale, 0.0).to(dt)
    return out


# --------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "embed": _exact_embed, "dropout": _exact_dropout}[case["op"]](s)


def _exact_rope(s):
    c = s["case"]
    K, R, d, rot = c["workers"], c["rows"], c["d"], c["rot"]
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]].unsqueeze(1)
    out = {}
    for n in "qk":
        x = s[n].double().requires_grad_(c["train"])
        w = s["w_" + n]
        z = x
        if w is not None:
            w = w.double().requires_grad_(c["train"])
            z = x / torch.sqrt(torch.mean(x * x, -1, keepdim=True) + EPS)
            z = (z.view(K, R, -1, d) * w.view(K, 1, 1, d)).view(x.shape)
        turning = z[..., :rot]
        if c["inter"]:
            two = turning.reshape(*z.shape[:-1], rot // 2, 2)
            two = torch.view_as_real(torch.view_as_complex(two.contiguous()) * turn)
            turned = two.reshape(*z.shape[:-1], rot)
        else:
            two = torch.complex(*turning.split(rot // 2, -1)) * turn
            turned = torch.cat((two.real, two.imag), -1)
        y = torch.cat((turned, z[..., rot:]), -1)
        out[n + "_out"] = y.detach()
        if c["train"]:
            y.backward(s[f"d{n}_out"].double())
            out |= {"d" + n: x.grad, "dw_" + n: None if w is None else w.grad}
    return out


def _exact_embed(s):
    K, V, W = s["table"].shape
    outs, grads = [], []
    for m in range(K):
        tok = s["tokens"][m]
        table = s["table"][m].double() * s["scale"]
        outs.append(torch.where(tok[:, None] < 0, 0.0, table[tok.clamp_min(0)]))
        if s["case"]["train"]:
            g = torch.zeros((V + 1, W), dtype=torch.float64, device="cuda")      # padding's share goes to a row behind the last
            g.index_put_((torch.where(tok < 0, V, tok),), s["dout"].view(K, -1, W)[m].double(), accumulate=True)
            grads.append(g[:V] * s["scale"])
    out = {"out": torch.cat(outs)}
    if s["case"]["train"]:
        out["dtable"] = torch.stack(grads)
    return out


def _exact_words(seed, offset, row, column):
    """Philox on halves of 16 bits: no product of two of them leaves 32 bits."""
    def mulhilo(m, x):
        m1, m0, x1, x0 = m >> 16, m & 0xFFFF, x >> 16, x & 0xFFFF
        low, mid = m0 * x0, m1 * x0
        mid = mid + (low >> 16)
        mid2 = m0 * x1 + (mid & 0xFFFF)
        return m1 * x1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)

    x0, x1 = column // 4, row
    x2, x3 = torch.full_like(x0, offset % 2 ** 32), torch.full_like(x0, offset // 2 ** 32)
    for i in range(ROUNDS):
        key0, key1 = (seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32
        h0, l0 = mulhilo(0xD2511F53, x0)
        h1, l1 = mulhilo(0xCD9E8D57, x2)
        x0, x1, x2, x3 = h1 ^ x1 ^ key0, l1, h0 ^ x3 ^ key1, l0
    return x0, x1, x2, x3


def _exact_dropout(s):
    c = s["case"]
    R, W, p = c["rows"], c["width"], c["p"]
    out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("out", "dx") if n in s}
    step = max(1, 2 ** 26 // W)
    for a in range(0, R, step):      # some rows at a time: the words take 32 bytes a value
        b = min(R, a + step)
        row = torch.arange(a, b, device="cuda")[:, None].expand(-1, -(-W // 4))
        column = (4 * torch.arange(-(-W // 4), device="cuda"))[None, :].expand(b - a, -1)
        for j, word in enumerate(_exact_words(s["seed"], s["offset"], row, column)):
            kept = word.double() / 2.0 ** 32 >= round(p * 2 ** 32) / 2.0 ** 32
            mine = kept[:, :len(range(j, W, 4))]
            out["out"][a:b, j::4] = torch.where(mine, s["x"][a:b, j::4].double() / (1.0 - p), 0.0)
            if "dx" in out:
                out["dx"][a:b, j::4] = torch.where(mine, s["dout"][a:b, j::4].double() / (1.0 - p), 0.0)
    return out


# --------------------------------------------------------------------------------------- work
def work(case):
    """Bytes and operations one pass cannot do without."""
    b = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if case["op"] == "rope":
        T, d = case["workers"] * case["rows"], case["d"]
        n = T * (case["hq"] + case["hk"]) * d
        bytes_ = 2 * n * b + min(T, case["seq"]) * case["rot"] * 4 + 8 * T + (8 * case["workers"] * d if case["norm"] else 0)      # in, out; tables, positions, weights
        flops = n * (7 if case["norm"] else 3)
        if case["train"]:
            bytes_ += 2 * n * b + (8 * case["workers"] * d if case["norm"] else 0)      # gradients in, gradients out
            flops += n * (16 if case["norm"] else 3)
        return {"bytes": bytes_, "flops": flops}
    if case["op"] == "embed":
        K, R, V, W = (case[n] for n in ("workers", "rows", "vocab", "width"))
        real = R - R // 10 if case["pad"] else R
        # rows of the table that a worker's batch is expected to touch
        v = torch.arange(1, V + 1, dtype=torch.float64)
        share = torch.log((v + 1) / v) / math.log(V + 1)
        distinct = float((1 - (1 - share) ** real).sum())
        bytes_ = K * R * 8 + int(K * distinct * W * 4) + K * R * W * b
        flops = K * real * W
        if case["train"]:
            bytes_ += K * real * W * b + K * V * W * 4
            flops += K * real * W + int(K * distinct * W)
        return {"bytes": bytes_, "flops": flops}
    n = case["rows"] * case["width"] * (2 if case["train"] else 1)
    return {"bytes": 2 * n * b, "flops": n}

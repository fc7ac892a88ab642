"""What the entry points of head norms with rotation, embeddings and dropout refuse.  The checks come before anything touches a device, so stand-in
addresses do and no GPU is needed; every call here is refused."""
import ctypes

import pytest

import paper_2606_22768_b200 as fgd

INVALID, ALIAS, UNSUPPORTED = fgd.FGD_ERR_INVALID_ARG, fgd.FGD_ERR_ALIAS, fgd.FGD_ERR_UNSUPPORTED
A = 1 << 40      # addresses a terabyte apart


def _at(n):
    return A * (n + 1)


# ------------------------------------------------------------------------------- head norms and rotation
ROPE = dict(dtype=fgd.FGD_BF16, workers=2, rows=10, hq=4, hk=2, d=64, rot=64, inter=0, position_bytes=8, table_rows=100, eps=1e-5,
            cos=(_at(0), 32), sin=(_at(1), 32), positions=_at(2), w_q=(_at(3), 64), w_k=(_at(4), 64), q=(_at(5), 256, 64), k=(_at(6), 128, 64),
            q_out=(_at(7), 256, 64), k_out=(_at(8), 128, 64), dq_out=(_at(9), 256, 64), dk_out=(_at(10), 128, 64), dq=(_at(11), 256, 64), dk=(_at(12), 128, 64),
            dw_q=(_at(13), 64), dw_k=(_at(14), 64), workspace=(_at(15), 1 << 30))


def _rope(backward, **change):
    a = {**ROPE, **change}
    flat = []
    for v in a.values():
        flat += list(v) if isinstance(v, tuple) else [v]
    args = fgd._ROPE_ARGS.pack(*flat)
    return (fgd._lib.fgd_qk_rope_backward if backward else fgd._lib.fgd_qk_rope_forward)(0, args, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=3)), (INVALID, dict(workers=0)), (INVALID, dict(workers=65)), (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 31)), (INVALID, dict(hq=0)),
    (INVALID, dict(hk=-1)), (INVALID, dict(d=0)), (UNSUPPORTED, dict(d=257)), (INVALID, dict(rot=0)), (INVALID, dict(rot=63)), (INVALID, dict(rot=66)),
    (INVALID, dict(position_bytes=2)), (INVALID, dict(positions=0)), (INVALID, dict(positions=_at(2) + 4)), (INVALID, dict(position_bytes=0, table_rows=19)),
    (INVALID, dict(table_rows=-1)), (INVALID, dict(eps=-1e-9)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(eps=float("inf"))), (INVALID, dict(cos=(0, 32))),
    (INVALID, dict(sin=(_at(1), 31))), (INVALID, dict(cos=(_at(0) + 2, 32))), (INVALID, dict(w_q=(_at(3), 63))), (INVALID, dict(w_k=(_at(4) + 1, 64))), (INVALID, dict(hk=0)),
])
def test_rope_refuses(backward, status, change):
    assert _rope(backward, **change) == status


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(q=(0, 256, 64))), (INVALID, dict(k=(_at(6) + 1, 128, 64))), (INVALID, dict(q_out=(_at(7), -256, 64))), (INVALID, dict(q_out=(_at(7), 0, 64))),
    (INVALID, dict(k_out=(_at(8), 127, 64))), (ALIAS, dict(q_out=(_at(6), 256, 64))), (ALIAS, dict(q_out=(_at(5) + 128, 256, 64))), (ALIAS, dict(q_out=(_at(5), 320, 64))),
    (ALIAS, dict(k_out=(_at(7), 128, 64))), (ALIAS, dict(k_out=(_at(0), 128, 64))), (ALIAS, dict(q_out=(_at(3) - 512, 256, 64))), (ALIAS, dict(k_out=(_at(2), 128, 64))),
])
def test_rope_forward_refuses(status, change):
    assert _rope(False, **change) == status


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dq_out=(0, 256, 64))), (INVALID, dict(dk=(0, 128, 64))), (INVALID, dict(q=(0, 256, 64))), (INVALID, dict(dw_q=(0, 64))), (INVALID, dict(dw_k=(_at(14), 60))),
    (INVALID, dict(workspace=(0, 1 << 30))), (INVALID, dict(workspace=(_at(15) + 2, 1 << 30))), (ALIAS, dict(workspace=(_at(11) + 64, 1 << 30))), (ALIAS, dict(workspace=(_at(14), 1 << 20))), (ALIAS, dict(dq=(_at(5), 256, 64))),
    (ALIAS, dict(dk=(_at(11), 128, 64))), (ALIAS, dict(dw_q=(_at(13), 64), dw_k=(_at(13) + 128, 64))), (ALIAS, dict(dw_q=(_at(3), 64))), (ALIAS, dict(dw_k=(_at(6), 64))),
    (ALIAS, dict(dq=(_at(13), 256, 64))),
])
def test_rope_backward_refuses(status, change):
    assert _rope(True, **change) == status


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("eps", [1e39, 3.4028236e38])
def test_rope_refuses_eps_beyond_fp32(backward, eps):
    """Finite in 64 bits and infinite in the kernels, where every norm would be zero."""
    assert _rope(backward, eps=eps) == INVALID


def test_rope_null():
    assert fgd._lib.fgd_qk_rope_forward(0, None, None) == INVALID and fgd._lib.fgd_qk_rope_backward(0, None, None) == INVALID
    for args in ((0, 64), (65, 64), (1, 0), (1, 257)):
        with pytest.raises(fgd.FgdError):
            fgd.fgd_qk_rope_workspace(*args)


# ------------------------------------------------------------------------------- embeddings
EMBED = dict(dtype=fgd.FGD_BF16, workers=2, rows=10, vocab=50, width=64, tokens=_at(0), token_bytes=8, ld_tokens=10, table=_at(1), worker_stride=3200, row_stride=64, scale=1.0,
             x=_at(2), ld_x=64, workspace=_at(3), workspace_bytes=1 << 30)


def _embed(backward, **change):
    a = {**EMBED, **change}
    head = [0] + [a[n] for n in ("dtype", "workers", "rows", "vocab", "width", "tokens", "token_bytes", "ld_tokens")]
    table = [a[n] for n in ("table", "worker_stride", "row_stride")]
    if backward:
        return fgd._lib.fgd_embed_backward(*head, a["x"], a["ld_x"], a["scale"], *table, a["workspace"], a["workspace_bytes"], None)
    return fgd._lib.fgd_embed_forward(*head, *table, a["scale"], a["x"], a["ld_x"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=-1)), (INVALID, dict(workers=0)), (INVALID, dict(workers=65)), (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 31)), (INVALID, dict(vocab=0)),
    (INVALID, dict(vocab=(1 << 30) + 1)), (INVALID, dict(width=0)), (UNSUPPORTED, dict(width=65537)), (INVALID, dict(token_bytes=2)), (INVALID, dict(scale=float("inf"))),
    (INVALID, dict(table=0)), (INVALID, dict(tokens=0)), (INVALID, dict(x=0)), (INVALID, dict(ld_tokens=9)), (INVALID, dict(ld_x=63)), (INVALID, dict(row_stride=63)),
    (INVALID, dict(worker_stride=-64)), (INVALID, dict(tokens=_at(0) + 4)), (INVALID, dict(table=_at(1) + 2)), (INVALID, dict(x=_at(2) + 1)),
    (ALIAS, dict(x=_at(1) + 256)), (ALIAS, dict(x=_at(1) - 256)),
])
def test_embed_refuses(backward, status, change):
    assert _embed(backward, **change) == status


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("rows", [10, 1000])
@pytest.mark.parametrize("scale", [1e39, -1e39, 3.4028236e38])
def test_embed_refuses_scales_beyond_fp32(backward, rows, scale):
    """Finite in 64 bits and infinite in the kernels, where padding and absent tokens would be 0 times infinity."""
    assert _embed(backward, rows=rows, ld_tokens=rows, scale=scale) == INVALID


@pytest.mark.parametrize("backward,status,change", [
    (False, ALIAS, dict(x=_at(0))), (True, INVALID, dict(worker_stride=3199)), (True, INVALID, dict(worker_stride=0)), (True, ALIAS, dict(table=_at(0))), (True, ALIAS, dict(table=_at(3) + 16)), (True, ALIAS, dict(x=_at(3))), (True, INVALID, dict(workspace=0)),
    (True, INVALID, dict(workspace=_at(3) + 8)), (True, INVALID, dict(workspace_bytes=100)), (True, ALIAS, dict(workspace=_at(0))),
])
def test_embed_refuses_more(backward, status, change):
    """(With tokens enough that the gradient needs its workspace.)"""
    assert _embed(backward, **{"rows": 1000, "ld_tokens": 1000, **change}) == status


def test_embed_workspace():
    for args in ((0, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 65537)):
        with pytest.raises(fgd.FgdError):
            fgd.fgd_embed_workspace(*args)
    assert fgd.fgd_embed_workspace(2, 0, 50, 64) >= 0 and fgd.fgd_embed_workspace(2, 1000, 50, 64) > 0


# ------------------------------------------------------------------------------- dropout
DROP = dict(dtype=fgd.FGD_BF16, rows=10, width=64, x=_at(0), ld_x=64, out=_at(1), ld_out=64, p=0.1, seed=1, offset=2, counter=0)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dtype=7)), (INVALID, dict(rows=-1)), (INVALID, dict(rows=1 << 32)), (INVALID, dict(width=-1)), (INVALID, dict(width=1 << 31)), (INVALID, dict(p=1.0)), (INVALID, dict(p=-0.1)),
    (INVALID, dict(p=float("nan"))), (INVALID, dict(x=0)), (INVALID, dict(out=0)), (INVALID, dict(ld_x=63)), (INVALID, dict(ld_out=63)), (INVALID, dict(x=_at(0) + 1)),
    (INVALID, dict(out=_at(1) + 1)), (INVALID, dict(counter=_at(2) + 4)), (ALIAS, dict(out=_at(0) + 2)), (ALIAS, dict(out=_at(0), ld_out=72)), (ALIAS, dict(counter=_at(1) + 8)),
])
def test_dropout_refuses(status, change):
    assert fgd._lib.fgd_dropout(0, *{**DROP, **change}.values(), None) == status


# ------------------------------------------------------------------------------- the bindings, on CPU tensors
def test_bindings_refuse_cpu_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 2, 8))
    t = torch.zeros((4, 4))
    with pytest.raises(TypeError):
        fgd.fgd_qk_rope_forward(x, x, None, None, t, t, None, x, x)
    with pytest.raises(ValueError):
        fgd.fgd_qk_rope_forward(x[0], x, None, None, t, t, None, x, x)
    with pytest.raises(TypeError):
        fgd.fgd_embed_forward(torch.zeros((1, 4), dtype=torch.int64), torch.zeros((1, 5, 8)), torch.zeros((4, 8)))
    with pytest.raises(ValueError):
        fgd.fgd_dropout(x, x, 0.1, 0)
    with pytest.raises(TypeError):
        fgd.fgd_dropout(t, t, 0.1, 0)
    assert ctypes.sizeof(ctypes.c_int64) * 46 == fgd._ROPE_ARGS.size


@pytest.mark.parametrize("which", ["cos", "sin"])
def test_rotation_refuses_tables_that_ask_for_gradients(which):
    """There are none: the result would be differentiated as if the tables were constants."""
    torch = pytest.importorskip("torch")
    from paper_2606_22768_b200 import inner
    tables = {n: torch.zeros((4, 4), requires_grad=n == which) for n in ("cos", "sin")}
    with pytest.raises(ValueError, match="no gradients"):
        inner.qkv_rope(torch.zeros((4, 4, 8)), 2, 1, **tables)
    with torch.no_grad(), pytest.raises(TypeError, match="CUDA"):      # (without one it goes on to the next check)
        inner.qkv_rope(torch.zeros((4, 4, 8)), 2, 1, **tables)

"""The bindings of the inner step's operators on the host: what they hand to the library (a stand-in for it, so no GPU)."""
import types

import pytest


def test_attention_status_asks_on_the_plans_device(monkeypatch):
    """Without a stream: the current one of the plan's device, on which its kernels ran, whatever device is current."""
    torch = pytest.importorskip("torch")
    import paper_2606_22768_b200 as fgd
    asked = []
    plan = object.__new__(fgd.AttnPlan)
    plan._h, plan.device = None, 3
    monkeypatch.setattr(fgd, "_lib", types.SimpleNamespace(fgd_attn_status=lambda h, stream: asked.append(stream) or 0))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=1000 + (0 if device is None else torch.device(device).index)))
    fgd.fgd_attn_status(plan)
    fgd.fgd_attn_status(plan, types.SimpleNamespace(cuda_stream=7))
    fgd.fgd_attn_status(plan, 8)
    assert asked == [1003, 7, 8]

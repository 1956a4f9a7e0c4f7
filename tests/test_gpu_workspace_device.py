"""A workspace that is not in the memory of the call's device is refused before any launch, by either marshalling."""
import copy

import pytest
import torch

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def elsewhere(ws, buf):
    """The workspace, said to be in another memory (its pointer stays a good one)."""
    other = copy.copy(ws)
    other.buf, other.device_index = buf, buf.device.index
    return other


@gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("where", ["cpu", "meta"])
def test_workspace_elsewhere(rk, where, native, monkeypatch):
    from paper_2411_05787_amd import binding
    if not native:
        for name in ("rk_full_attn_q8", "rk_prompt_attn"):
            monkeypatch.setattr(binding._native, name, lambda *a: None)
    geom, n = rk.Geom(1, 4, 2, 128, 0.1), 600
    lens, buf = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.empty(1024, dtype=torch.uint8, device=where)
    K, V = (torch.ones(1, 2, 608, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.full((1, 1, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    ws, wp = rk.Workspace(geom, 608, 16), rk.PromptWorkspace(geom, 1, 608)
    cache = rk.Kv8.empty(geom, 608)
    with pytest.raises(ValueError):
        rk.rk_full_attn_q8(geom, q[:, 0], cache, lens, n, out[:, 0], workspace=elsewhere(ws, buf))
    with pytest.raises(ValueError):
        rk.rk_full_attn_q8(geom, q[:, 0], cache, lens, n, out[:, 0])
    with pytest.raises(ValueError):
        rk.rk_prompt_attn(geom, q, K, V, lens, n, out, workspace=elsewhere(wp, buf))
    assert bool((out == 5).all())
    rk.rk_prompt_attn(geom, q, K, V, lens, n, out, workspace=wp)
    assert bool((out == 1).all())
    rk.rk_full_attn_q8(geom, q[:, 0], cache, lens, n, out[:, 0], workspace=ws)
    assert bool((out == 0).all())

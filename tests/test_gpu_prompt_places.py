"""Places that a call of the layers for prompts must not use besides its inputs': the
handle's weights and its workspace.  Every call here is refused before anything is
launched."""
import ctypes

import pytest

from paper_2609_04895_amd import cmoe as B
from test_operators_abi import P, error, moe_cfg

INVALID = B.CMOE_ERR_INVALID_ARG


@pytest.mark.parametrize("weights", [0, 2])
@pytest.mark.parametrize("other", ["w_router", "logit_bias", "experts", "expert_scales"])
def test_a_workspace_over_the_weights_is_refused(weights, other):
    if other == "expert_scales" and not weights:
        return
    cfg = moe_cfg(weights=weights)
    size, n = B.cmoe_prompt_query(cfg), 2 * 16 * 3 * 256 * 128
    length = dict(w_router=2 * 16 * 256 * 2, logit_bias=2 * 16 * 4, experts=n // 2 if weights else 2 * n, expert_scales=n // 32)
    at = {k: (i + 1) * (64 * P) for i, k in enumerate(length)}
    for workspace in (at[other] + (length[other] - 1) // 256 * 256, at[other] - (size - 1) // 256 * 256):
        assert at[other] - size < workspace < at[other] + length[other]
        w, h = B.cmoe_moe_weights(**at), ctypes.c_void_p(5)
        assert B.lib().cmoe_prompt_init(ctypes.byref(cfg), ctypes.byref(w), workspace, None, ctypes.byref(h)) == INVALID
        assert "workspace overlaps" in error() and not h.value


def test_pools_beyond_any_memory_do_not_wrap_around():
    cfg = moe_cfg(L=2 ** 31 - 1, N=256, d=65536, F=65536)
    w, h = B.cmoe_moe_weights(w_router=P, logit_bias=None, experts=64 * P, expert_scales=None), ctypes.c_void_p()
    assert B.lib().cmoe_prompt_init(ctypes.byref(cfg), ctypes.byref(w), 1 << 45, None, ctypes.byref(h)) == INVALID
    assert "workspace overlaps" in error()


@pytest.mark.gpu
def test_outputs_in_the_weights_or_the_workspace_are_refused():
    torch = pytest.importorskip("torch")
    L, N, K, d, F, T = 2, 8, 2, 128, 64, 4
    cfg = B.make_moe_config(L, N, K, d, F, T, B.CMOE_BF16, B.CMOE_FORMAT_MX8)
    router = torch.zeros((L, N, d), dtype=torch.bfloat16, device="cuda")
    bias = torch.zeros((L, N), device="cuda")
    experts = torch.zeros((L, N, 3 * d * F), dtype=torch.uint8, device="cuda")
    scales = torch.full((L, N, 3 * d * F // 32), 127, dtype=torch.uint8, device="cuda")
    layers = B.PromptLayers(cfg, router, bias, experts, scales)
    h, y = (torch.zeros((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sel, gates = torch.zeros((T, K), dtype=torch.int32, device="cuda"), torch.zeros((T, K), device="cuda")
    good = dict(h=h, y=y, selected=sel, gates=gates)
    rows, picks = T * d * 2, T * K * 4

    def bf16(t, at=0):
        return t.view(-1)[at:at + rows].view(torch.bfloat16).view(T, d)

    def i32(t, at=0):
        return t.view(-1).view(torch.uint8)[at:at + picks].view(torch.int32).view(T, K)

    ws = layers.workspace
    for kw in (dict(y=router[1, :T]), dict(y=bf16(experts)), dict(y=bf16(experts, experts.numel() - rows)), dict(y=bf16(scales)), dict(y=bf16(ws)),
               dict(y=bf16(ws, ws.numel() - rows)), dict(h=bf16(ws, 256)), dict(selected=i32(bias)), dict(selected=i32(ws, 512)),
               dict(selected=i32(experts, 64)), dict(gates=i32(router, 32).view(torch.float32)), dict(gates=i32(ws).view(torch.float32)),
               dict(gates=i32(scales, scales.numel() - picks).view(torch.float32)), dict(n_tokens=ws[:4].view(torch.int32))):
        with pytest.raises(B.CmoeError) as err:
            layers.cmoe_prompt_layer(0, **{**good, **kw})
        assert err.value.status == INVALID and "overlaps" in str(err.value), list(kw)
    # h may lie in a weight: both are only read
    layers.cmoe_prompt_layer(0, h=router[0, :T], y=y, selected=sel, gates=gates)
    torch.cuda.synchronize()
    assert (y == 0).all() and sel.tolist() == [[0, 1]] * T and not router.any() and not experts.any()

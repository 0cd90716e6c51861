"""Outputs in the place of an input or of another output, which the header rules out
but for the sum in place and for y in delta's place, are refused before anything
reaches the GPU."""
import ctypes

import pytest

from paper_2609_04895_amd import cmoe as B
from test_operators_abi import P, error, norm

OUTPUTS = dict(residual_out=3 * P, h=5 * P, h8=6 * P, h8_scale=7 * P)
INPUTS = dict(residual=P, delta=2 * P, weight=4 * P, n_rows=8 * P)


@pytest.mark.parametrize("out,other", [(out, other) for out in OUTPUTS for other in [*INPUTS, *OUTPUTS]
                                       if out != other and (out, other) != ("residual_out", "residual")])
def test_norm_outputs_have_places_of_their_own(out, other):
    args = {**INPUTS, **OUTPUTS}
    args[out] = args[other]
    assert B.lib().cmoe_add_norm(ctypes.byref(norm(**args)), None) == B.CMOE_ERR_INVALID_ARG
    assert "place" in error()


@pytest.mark.gpu
def test_layer_and_block_outputs_have_places_of_their_own():
    torch = pytest.importorskip("torch")
    from test_gpu_moe_layer import Model
    N, K, d, F, T = 8, 2, 128, 64, 4
    m = Model("w8a8", 1, N, K, d, F, T, "places")
    layers = m.layers()
    h = m.hidden(T)
    eight, _ = m.eight(h)
    h = h.cuda()
    # views of one buffer: y's rows hold those of every other argument
    y = torch.zeros((T, d), device="cuda")
    as_y = y.view(torch.uint8).view(T, 4 * d)
    y_bf16, y_i32 = y.view(torch.bfloat16)[:, :d], y.view(torch.int32).view(-1)
    sel, gates = torch.zeros((T, K), dtype=torch.int32, device="cuda"), torch.zeros((T, K), device="cuda")
    n = torch.tensor([T], dtype=torch.int32, device="cuda")
    good = dict(h=h, y=y, selected=sel, gates=gates, n_tokens=n, **eight)
    for kw in (dict(h=y_bf16), dict(h8=as_y[:, :d]), dict(h8_scale=as_y[:, :d // 32]), dict(n_tokens=y_i32[:1]),
               dict(selected=y_i32[:T * K]), dict(gates=y.view(-1)[:T * K]), dict(gates=sel.view(torch.float32)),
               dict(selected=h.view(torch.int32).view(-1)[:T * K]), dict(gates=eight["h8"].view(-1)[:4 * T * K].view(torch.float32)),
               dict(n_tokens=sel.view(-1)[:1])):
        with pytest.raises(B.CmoeError) as err:
            layers.cmoe_moe_layer(0, **{**good, **kw})
        assert err.value.status == B.CMOE_ERR_INVALID_ARG and "place" in str(err.value), list(kw)
    res, out, delta = h.clone(), torch.zeros_like(h), torch.zeros((T, d), device="cuda")
    good = dict(residual=res, delta=delta, y=y, residual_out=out, selected=sel, gates=gates, n_tokens=n)
    weight = layers.norm_weight[0]
    for kw in (dict(residual=y_bf16), dict(residual_out=y_bf16), dict(selected=y_i32[:T * K]), dict(gates=y.view(-1)[:T * K]),
               dict(n_tokens=y_i32[:1]), dict(gates=sel.view(torch.float32)), dict(selected=res.view(torch.int32).view(-1)[:T * K]),
               dict(selected=out.view(torch.int32).view(-1)[:T * K]), dict(gates=delta.view(-1)[:T * K]),
               dict(selected=weight.view(torch.int32)[:T * K]), dict(n_tokens=out.view(torch.int32).view(-1)[:1])):
        with pytest.raises(B.CmoeError) as err:
            layers.cmoe_moe_block(0, **{**good, **kw})
        assert err.value.status == B.CMOE_ERR_INVALID_ARG and "place" in str(err.value), list(kw)
    # what the header allows
    layers.cmoe_moe_block(0, **{**good, "residual_out": res})
    layers.cmoe_moe_block(0, **{**good, "delta": y})
    layers.cmoe_moe_layer(0, h, y, selected=sel, gates=gates, n_tokens=n, **eight)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all()

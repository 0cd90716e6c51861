"""Weights of MoeLayers that are dropped while calls on the handle's stream are still
in flight: their memory is not handed out before those are done."""
import pytest

from test_gpu_moe_layer import Model, check, outputs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", ["bf16", "w8"])
def test_weights_dropped_with_calls_in_flight(kind):
    N, K, d, F, T = 16, 4, 512, 256, 6
    m = Model(kind, 1, N, K, d, F, T, f"lifetime {kind}")
    h = m.hidden(T)
    want = m.expected(0, h, h.double())
    st = torch.cuda.Stream()
    layers, hg = m.layers(stream=st), h.cuda()
    y, sel, gates = outputs(T, K, d)
    held = {t.untyped_storage().data_ptr(): t.numel() * t.element_size() for t in m.gpu.values() if t is not None}
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(200_000_000)  # some 0.1 s of waiting in front of the call
    layers.cmoe_moe_layer(0, hg, y, selected=sel, gates=gates)
    layers._keep = None
    del layers
    m.gpu.clear()
    assert not st.query()  # the call has not run yet
    new = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in held.values() for _ in range(2)]
    assert not {t.data_ptr() for t in new} & set(held)
    torch.cuda.synchronize()
    check((y, sel, gates), want, K)

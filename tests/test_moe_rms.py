"""The average-error bound of the MoE layer's tests notices an intermediate in bf16
and lets one in fp32 pass (oracle only, no GPU)."""
import pytest

import operator_reference as ref
from moe_rms import rms_bound, rms_error

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("d,F", [(64, 64), (704, 448), (2112, 2048)])
def test_bound_separates_bf16_from_fp32(d, F):
    g = torch.Generator().manual_seed(d + F)
    N, K, T = 3, 2, 6
    pool = [tuple((torch.randn(s, generator=g) * 0.02).bfloat16().double() for s in ((F, d), (F, d), (d, F))) for _ in range(N)]
    x = torch.randn((T, d), generator=g).bfloat16().double()
    sel, gates, _ = ref.route(x, torch.randn((N, d), generator=g).double() * 0.1, None, K)
    want, err = ref.experts(x, sel, gates, lambda e: pool[e], d, F)

    def layer(round_to):
        y = torch.zeros((T, d), dtype=torch.float32)
        for t in range(T):
            for k in range(K):
                wg, wu, wd = (w.float() for w in pool[sel[t, k]])
                u = wg @ x[t].float()
                a = (u * torch.sigmoid(u) * (wu @ x[t].float())).to(round_to).float()
                y[t] += gates[t, k].float() * (wd @ a)
        return y

    assert rms_error(layer(torch.float32), want) <= rms_bound(d, F, K)
    assert rms_error(layer(torch.bfloat16), want) > 8 * rms_bound(d, F, K)

"""How exact fp32 sums are, whatever the number of rows and however long the rows: the
root mean square of y's error against fp64.

A chain of c products, each rounded as it is added, is off by the roundings of its
partial sums: rounding i by at most u = 2^-24 of a sum that grows as sqrt(i), evenly
spread, so u / sqrt(3) rms; in all u sqrt(c / 6) of the result.  n / c chains that are
added up in turn give u sqrt(n / c / 6) more, in squares.  Chains here are of 256 values
at most and 64 at least."""
import math

import pytest

import mx4_reference as mx
from gpu_util import say, stable_seed

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, U8, U = torch.float32, torch.uint8, 2.0 ** -24


def bound(d, each=1):
    """each: roundings per value.  Two more for y's own and the join of wavefronts; a tenth
    for chance, over 4096 values and more."""
    return 1.1 * U * math.sqrt((256 * each + d / 64) / 6 + 2)


def close(y, want, most):
    assert y.numel() >= 4096
    rms = ((y.double() - want).norm() / want.norm()).item()
    say(f"  {rms / U:.2f} of at most {most / U:.2f} half steps")
    assert rms <= most


# few rows of a group; of several; as many as the few-row kernel takes; tiles
@pytest.mark.parametrize("d", [448, 4096, 65536])
@pytest.mark.parametrize("sizes,m", [([8], 512), ([1] * 8, 512), ([32], 256), ([200], 256)])
def test_grouped_products(sizes, m, d):
    from paper_2609_04895_amd import cmoe as B
    say(f"fp32 sums product {sizes} m {m} d {d}")
    g = torch.Generator(device="cuda").manual_seed(stable_seed(f"sums {sizes} {m} {d}"))
    N, rows = len(sizes), sum(sizes)
    x = torch.empty((rows, d), device="cuda").normal_(generator=g)
    w = torch.empty((N, 2 * m, d), device="cuda").normal_(0, 1 / math.sqrt(d), generator=g)
    first = torch.tensor([sum(sizes[:i]) for i in range(N + 1)], dtype=torch.int32, device="cuda")
    gates, ups = [], []
    for e in range(N):
        p = x[sum(sizes[:e]):sum(sizes[:e + 1])].double() @ w[e].double().t()
        gates.append(p[:, :m])
        ups.append(p[:, m:])
    gate, up = torch.cat(gates), torch.cat(ups)
    y = torch.empty((rows, m), device="cuda")
    B.cmoe_grouped_product(x, w[:, :m], first, y)
    close(y, gate, bound(d))
    # SwiGLU of values of variance 1: |silu'| <= 1.1 and E silu^2 = 0.356, so a sum's relative
    # error counts sqrt((1.21 + 0.356) / 0.356) = 2.1 times; and the roundings of silu
    B.cmoe_grouped_product(x, w, first, y, swiglu=True)
    close(y, torch.nn.functional.silu(gate) * up, 2.1 * bound(d) + 4 * U)


def dequantized(q, s):
    table = torch.cat((mx.E2M1, -mx.E2M1)).cuda()
    v = table[torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], -1).int()]
    return (v.view(*s.shape, 32) * torch.pow(2.0, s.double() - 127).unsqueeze(-1)).view(v.shape)


# few weight rows; many, one tile a wavefront; in two launches; two tiles a wavefront
@pytest.mark.parametrize("rows,m,d", [(16, 256, 4096), (1, 4096, 2048), (8, 512, 65536), (16, 256, 1 << 18), (16, 10240, 4096), (25, 10240, 4096),
                                      (16, 10240, 65536), (8, 131072, 512)])
def test_matvec(rows, m, d):
    """An fp32 x is three bf16 numbers: three products a value."""
    from paper_2609_04895_amd import cmoe as B
    say(f"fp32 sums matvec rows {rows} m {m} d {d}")
    g = torch.Generator(device="cuda").manual_seed(stable_seed(f"sums mv {rows} {m} {d}"))
    q = torch.randint(0, 256, (m, d // 2), dtype=U8, device="cuda", generator=g)
    s = torch.randint(124, 128, (m, d // 32), dtype=U8, device="cuda", generator=g)
    x = torch.empty((rows, d), device="cuda").normal_(generator=g)
    y = torch.empty((rows, m), device="cuda")
    B.cmoe_matvec(x, q, s, y)
    some = torch.arange(m, device="cuda") if m <= 4096 else torch.randperm(m, device="cuda", generator=g)[:512]
    close(y[:, some], x.double() @ dequantized(q[some], s[some]).t(), bound(d, 3))

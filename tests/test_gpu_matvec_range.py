"""cmoe_matvec with fp32 rows at the ends of the type's range: an fp32 x is taken whole,
so products with numbers next to the largest are finite where the definition is, and
of small numbers only what lies below 2^-133 is lost."""
import pytest

import mx4_reference as mx
from gpu_util import say, stable_seed

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, U8 = torch.float32, torch.uint8
LARGEST = torch.finfo(F32).max
# few weight rows; many, in two launches; many, two tiles a wavefront
SHAPES = [(3, 100, 512), (25, 10300, 96), (2, 131100, 64)]


def weights(m, d, byte, g):
    return torch.randint(0, 256, (m, d // 2), generator=g).to(U8), torch.full((m, d // 32), byte, dtype=U8)


def run(x, q, s):
    from paper_2609_04895_amd import cmoe as B
    y = torch.full((x.shape[0], q.shape[0]), 7.0, device="cuda")
    B.cmoe_matvec(x.cuda(), q.cuda(), s.cuda(), y)
    return y.cpu().double()


@pytest.mark.parametrize("rows,m,d", SHAPES)
def test_numbers_next_to_the_largest(rows, m, d):
    say(f"matvec range rows {rows} m {m} d {d}")
    g = torch.Generator().manual_seed(stable_seed(f"range {rows} {m} {d}"))
    q, s = weights(m, d, 127 - 20, g)  # sums stay in range
    q[::5] = 0                         # rows of zeros
    q[1::5] = 8 * 17                   # and of negative zeros
    # from a little below bf16's largest number to fp32's
    x = LARGEST * (1 - torch.rand((rows, d), generator=g) * 2.0 ** -7)
    x = x * (torch.randint(0, 2, (rows, d), generator=g) * 2 - 1)
    x[0, :] = LARGEST
    x[-1, :-1] = 0
    x[-1, -1] = -LARGEST
    y = run(x, q, s)
    want, err = mx.product(x.double(), mx.dequantize4(q, s))
    assert torch.isfinite(y).all()
    assert ((y - want).abs() <= err * 2 + mx.half_step(want, F32)).all()
    assert (y[:, ::5] == 0).all() and (y[:, 1::5] == 0).all()


@pytest.mark.parametrize("rows,m,d", SHAPES)
def test_every_bit_counts(rows, m, d):
    """x = 2^24 - 1, 24 ones: times one weight of a row that is not zero the products are
    whole, so any bit of x that is lost shows."""
    q = torch.zeros((m, d // 2), dtype=U8)
    at = torch.arange(m) % (d // 2)
    q[torch.arange(m), at] = 2  # 1, at value 2 at
    s = torch.full((m, d // 32), 127, dtype=U8)
    x = torch.full((rows, d), float(2 ** 24 - 1))
    x[:, 1::2] = -float(2 ** 24 - 3)
    x[0] *= 2.0 ** -100
    y = run(x, q, s)
    assert (y[1:] == 2 ** 24 - 1).all() and (y[0] == (2 ** 24 - 1) * 2.0 ** -100).all()


@pytest.mark.parametrize("rows,m,d", SHAPES)
def test_small_numbers(rows, m, d):
    say(f"matvec small rows {rows} m {m} d {d}")
    g = torch.Generator().manual_seed(stable_seed(f"small {rows} {m} {d}"))
    q, s = weights(m, d, 127 + 60, g)
    x = torch.randn((rows, d), generator=g) * 2.0 ** -118
    y = run(x, q, s)
    w = mx.dequantize4(q, s)
    want, err = mx.product(x.double(), w)
    lost = 2.0 ** -133 * w.abs().sum(1)  # the smallest bf16 number
    assert ((y - want).abs() <= err * 2 + lost + mx.half_step(want, F32)).all()


@pytest.mark.parametrize("rows,m,d", SHAPES)
def test_nan_of_any_payload_is_nan(rows, m, d):
    g = torch.Generator().manual_seed(5)
    q, s = weights(m, d, 127, g)
    x = torch.randn((rows, d), generator=g)
    bits = x.view(torch.int32)
    bits[0, 3], bits[1, d - 1] = 0x7F800001, 0x7FFFFFFF
    y = run(x, q, s)
    assert y[:2].isnan().all()
    want, err = mx.product(x[2:].double(), mx.dequantize4(q, s))
    assert ((y[2:] - want).abs() <= err * 2 + mx.half_step(want, F32)).all()

"""What cmoe_grouped_product rounds, and to what: 8-bit outputs are rounded from fp32 sums
of 8-bit rows, and bf16 ones from sums that are off by 2^-16 of a typical one; scales of
8-bit outputs block by block; products straight from a pool with every tensor strided;
rows out of range where a group has few."""
import math

import pytest

import mx4_reference as mx
import operator_reference as ref
from gpu_util import say, stable_seed
from test_gpu_product import FORMS, TYPES, Case, hold

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


def e4m3(v):
    return torch.tensor(v, dtype=F32).to(torch.float8_e4m3fn).view(U8)


@pytest.mark.parametrize("form", ["x8 w8", "x8 w4"])
@pytest.mark.parametrize("sizes,m", [([5], 64), ([3, 40], 64), ([300], 256), ([500, 700, 0, 520, 900], 12864)])
def test_sums_beside_the_middle_of_a_step(form, sizes, m):
    """Columns of 256 + 16 -+ 2^-7 and 288 + 16 -+ 2^-7, which lie between 256, 288 and 320 as
    e4m3 numbers: to 24 bits they go to the nearer one; to the 13 bits of a sum on the 8-bit
    core they would be the middle.  A column of 448 in each block makes its scale 1."""
    from paper_2609_04895_amd import cmoe as B
    say(f"rounding {form} {sizes} m {m}")
    rows, N, d = sum(sizes), len(sizes), 192
    # products of a value each: 256, 32 and 16 times one; 2^-6 times +-1/2
    for at in (0, 33, 128):
        x = torch.zeros((rows, d))
        x[:, at:at + 4] = torch.tensor([256.0, 32.0, 16.0, 2.0 ** -6])
        w = torch.zeros((m, d))
        sign = torch.tensor([1.0, -1.0]).repeat(m // 2)
        w[:, at], w[:, at + 1], w[:, at + 2], w[:, at + 3] = 1, (torch.arange(m) // 2 % 2).float(), 1, sign / 2
        w[::32, at:at + 4] = torch.tensor([1.5, 2.0, 0.0, 0.0])
        want = torch.where(sign > 0, torch.where(w[:, at + 1] > 0, 320.0, 288.0), torch.where(w[:, at + 1] > 0, 288.0, 256.0))
        want[::32] = 448
        # scales of 1 that these blocks would not get by themselves, and zeros elsewhere
        x8, xs = e4m3(x.tolist()), torch.full((rows, d // 32), 127, dtype=U8)
        if form == "x8 w8":
            q = e4m3(w.tolist())
        else:
            q = mx.pack((w.abs().unsqueeze(-1) == mx.E2M1.float()).int().argmax(-1) + 8 * (w < 0).long())
        ws = torch.full((N, m, d // 32), 127, dtype=U8)
        first = torch.tensor([sum(sizes[:i]) for i in range(N + 1)], dtype=torch.int32)
        y, s = torch.zeros((rows, m), dtype=U8, device="cuda"), torch.zeros((rows, m // 32), dtype=U8, device="cuda")
        B.cmoe_grouped_product(x8.cuda(), q.expand(N, *q.shape).contiguous().cuda(), first.cuda(), y, x_scale=xs.cuda(), w_scale=ws.cuda(),
                               y_scale=s)
        assert (s == 127).all()
        assert torch.equal(y.cpu(), e4m3(want.tolist()).expand(rows, m))


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes,m,d", [([3, 0, 5], 512, 320), ([40, 0, 128, 129, 25], 256, 320), ([300, 91, 257, 0, 448], 12864, 192)])
def test_outputs_are_the_rounded_sums(form, swiglu, sizes, m, d):
    """An error before a rounding moves a share of the values to the next step, so y differs
    from the rounded definition by sqrt(error x step) rms: with a step of 2^-7 and an
    error of 2^-15 of y, twice what the 8-bit core is off by, 2^-11; with fp32 sums an
    error of 2^-20, 2^-13.5.  (8-bit rows, bf16 y; fp32 y is compared elsewhere.)"""
    from paper_2609_04895_amd import cmoe as B
    say(f"rounded {form} swiglu {swiglu} {sizes} m {m}")
    c = Case(form, sizes, m // 2 if swiglu and m > 512 else m, d, swiglu, seed="rounded")
    if BF16 in TYPES[form]:
        want, _ = c.expected()
        y = torch.zeros((c.rows, c.m), dtype=BF16, device="cuda")
        c.run(B, y)
        want = want.to(BF16).double()
        off = ((y.cpu().double() - want).norm() / want.norm()).item()
        say(f"  bf16 off by {off:.2e}")
        assert off <= (2.0 ** -11 if form.startswith("x8") else 2.0 ** -13.5)
    if 8 in TYPES[form]:
        want, err = c.expected(exact=True)
        y = torch.zeros((c.rows, c.m), dtype=U8, device="cuda")
        s = torch.zeros((c.rows, c.m // 32), dtype=U8, device="cuda")
        c.run(B, y, s)
        y, s = y.cpu(), s.cpu()
        # the scale of every block: that of some value within the error
        amax = lambda v: v.reshape(c.rows, -1, 32).amax(-1)
        lo, hi = ref.quantize((want.abs() - err).clamp(min=0))[2], ref.quantize(want.abs() + err)[2]
        assert ((s >= lo) & (s <= hi)).all()
        assert (amax(want.abs()) > 0).all() and (s > 0).all()
        # at that scale, the value that some sum within the error rounds to
        got, at = ref.dequantize(y, s), ref.pow2(s.int() - 127).repeat_interleave(32, 1)

        def rounded(v):
            t = (v / at).clamp(-448, 448)
            step = ref.pow2(torch.frexp(t.abs().clamp(min=2.0 ** -6))[1] - 4)
            return torch.round(t / step) * step * at

        assert ((got >= rounded(want - err)) & (got <= rounded(want + err))).all()


@pytest.mark.parametrize("form", ["f32", "bf16", "x8 w8", "x8 w4", "bf16 w4", "bf16 w8"])
@pytest.mark.parametrize("sizes", [[3, 0, 4], [20, 0, 300]])
def test_both_halves_of_a_pool_with_strides(form, sizes):
    """gate and up, then down, straight from a pool [N][3 d F]; rows of x, y and all scales
    apart, bf16 y with rows that take 16-byte stores and with rows that do not."""
    from paper_2609_04895_amd import cmoe as B
    say(f"pool {form} {sizes}")
    g = torch.Generator().manual_seed(stable_seed(f"pool {form} {sizes}"))
    N, d, F, rows = 3, 192, 128, sum(sizes)
    wf = 8 if form.endswith("w8") else 4 if form.endswith("w4") else F32 if form == "f32" else BF16
    xf = 8 if form.startswith("x8") else F32 if form == "f32" else BF16
    w, ws, wv = hold(torch.randn((N, 3 * d * F), generator=g) * 0.1, wf)
    per = 2 if wf == 4 else 1
    first = [sum(sizes[:i]) for i in range(N + 1)]
    for up in (True, False):
        n, m = (d, F) if up else (F, d)
        def part(t, per):
            each = 3 * d * F // per
            at, length = (0, 2 * d * F // per) if up else (2 * d * F // per, d * F // per)
            return t.cuda().view(N, each)[:, at:at + length].view(N, -1, n // per)
        weight = wv.view(N, -1)[:, :2 * d * F].view(N, 2 * F, d) if up else wv.view(N, -1)[:, 2 * d * F:].view(N, d, F)
        x, xs, xv = hold(torch.randn((rows, n), generator=g), xf)
        wide = torch.zeros((rows, n + 48), dtype=x.dtype)
        wide[:, 16:16 + n] = x
        wide_s = None
        if xs is not None:
            wide_s = torch.full((rows, xs.shape[1] + 5), 255, dtype=U8)
            wide_s[:, 3:3 + xs.shape[1]] = xs
            wide_s = wide_s.cuda()[:, 3:3 + xs.shape[1]]
        mul = mx.product8 if xs is not None else mx.product
        for yt, left, gap in ((TYPES[form][0], 16, 32), (TYPES[form][0], 5, 13), (8, 4, 12)):
            if yt not in TYPES[form]:
                continue
            multiply = mx.product if yt == 8 else mul
            want, err = torch.zeros((rows, m), dtype=torch.float64), torch.zeros((rows, m), dtype=torch.float64)
            for e in range(N):
                a, b = first[e], first[e + 1]
                want[a:b], err[a:b] = mx.swiglu(xv[a:b], weight[e], m, multiply) if up else multiply(xv[a:b], weight[e])
            out = torch.full((rows, m + gap), 7, dtype=U8 if yt == 8 else yt, device="cuda")
            y, scale, out_s = out[:, left:left + m], None, None
            if yt == 8:
                out_s = torch.full((rows, m // 32 + 3), 7, dtype=U8, device="cuda")
                scale = out_s[:, 2:2 + m // 32]
            B.cmoe_grouped_product(wide.cuda()[:, 16:16 + n], part(w, per), torch.tensor(first, dtype=torch.int32).cuda(), y, x_scale=wide_s,
                                   w_scale=None if ws is None else part(ws, 32), swiglu=up, y_scale=scale)
            if yt == 8:
                got, most = ref.dequantize(y.cpu().contiguous(), scale.cpu().contiguous()), mx.mx8_error(want, err)
                assert (out_s[:, :2] == 7).all() and (out_s[:, 2 + m // 32:] == 7).all()
            else:
                got, most = y.cpu().double(), err + mx.half_step(want, yt)
            assert ((got - want).abs() <= most).all()
            assert (out[:, :left] == 7).all() and (out[:, left + m:] == 7).all()


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("form", FORMS)
def test_rows_out_of_range_of_small_groups(form, swiglu):
    """Rows that x_row names out of range are 0, whatever x holds, and no other row is."""
    from paper_2609_04895_amd import cmoe as B
    c = Case(form, [3, 0, 1, 4], 96, 128, swiglu, x_rows=6, seed="range")
    bad = torch.tensor([0, 3, 5])
    good = torch.tensor([1, 2, 4, 6, 7])
    if c.x_scale is not None:
        c.x_scale[0, 0], c.xv[0] = 255, math.nan
    else:
        c.x[0, 5], c.xv[0] = math.nan, math.nan
    c.x_row[good] = torch.tensor([1, 5, 2, 3, 1], dtype=torch.int32)
    for yt in TYPES[form]:
        c.x_row[bad] = torch.tensor([-1, 6, -2 ** 31], dtype=torch.int32)
        y = torch.full((8, 96), 9, dtype=U8 if yt == 8 else yt, device="cuda")
        s = torch.full((8, 3), 130, dtype=U8, device="cuda") if yt == 8 else None
        c.run(B, y, s)
        c.x_row[bad] = 1
        want, err = c.expected(exact=yt == 8)
        y = y.cpu()
        got = y.double() if yt != 8 else ref.dequantize(y, s.cpu())
        assert (y[bad] == 0).all() and (got[bad] == 0).all()
        most = err + mx.half_step(want, yt) if yt != 8 else mx.mx8_error(want, err)
        assert ((got - want).abs() <= most)[good].all() and (got[good] != 0).any(1).all()

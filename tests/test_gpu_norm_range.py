"""cmoe_add_norm where r * weight or the factor 1 / sqrt(mean r^2 + eps) leaves fp32's
range although h does not, and one rounding of h everywhere.

Tolerances: sums, factor and products in fp64 are off by (d + 8) 2^-53 at most, below
2^-39 for d <= 8192, so an fp32 h is off by half a step, 2^-24 of the value (1 + 2^-15
of that), or 2^-150 below fp32's normal range; a bf16 h by that and half a step of its
own, 2^-8 of the value (2^-134 below the normal range)."""
import pytest

import operator_reference as ref
from gpu_util import say, stable_seed
from test_gpu_norm import check_8bit

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32

# scale of r, scale of the weight, eps (a power of two: the same number in fp32 and fp64)
RANGES = [(1.0, 1.0, 2.0 ** -20), (2.0 ** 126, 1.0, 0.0), (2.0 ** 126, 1.0, 2.0 ** -20), (2.0 ** 120, 2.0 ** 40, 0.0),
          (2.0 ** -100, 2.0 ** -60, 0.0), (2.0 ** -130, 1.0, 0.0), (2.0 ** -130, 2.0 ** 20, 0.0), (2.0 ** -130, 2.0 ** 100, 2.0 ** -20)]


@pytest.mark.parametrize("scale,wscale,eps", RANGES)
@pytest.mark.parametrize("rows,d", [(3, 256), (1030, 320), (2, 8192), (2, 50), (2, 40000)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_norm_over_the_whole_range_of_fp32(scale, wscale, eps, rows, d, dtype):
    from paper_2609_04895_amd import cmoe as B
    say("norm range", scale, wscale, eps, rows, d, dtype)
    g = torch.Generator().manual_seed(stable_seed(f"range {scale} {wscale} {rows} {d}"))
    # |randn| <= 3.5 keeps r in range; weights between 1.1 and 1.4 put |r w| above 2^128
    res = (torch.randn((rows, d), generator=g).clamp(-3.5, 3.5) * scale).to(dtype)
    w = ((1.1 + 0.3 * torch.rand(d, generator=g)) * wscale).to(dtype)
    _, h64 = ref.norm(res, None, w, eps)
    h = torch.empty_like(res, device="cuda")
    kw = {}
    if d % 32 == 0:
        kw = dict(h8=torch.empty((rows, d), dtype=torch.uint8, device="cuda"),
                  h8_scale=torch.empty((rows, d // 32), dtype=torch.uint8, device="cuda"))
    B.cmoe_add_norm(res.cuda(), None, w.cuda(), eps, h=h, **kw)
    tol = 2.0 ** -24 * (1 + 2.0 ** -15) * h64.abs() + 2.0 ** -150
    if dtype == BF16:
        tol = tol + 2.0 ** -8 * h64.abs() + 2.0 ** -134
    off = (h.cpu().double() - h64).abs()
    assert (off <= tol).all(), f"{float(torch.nan_to_num(off / tol, nan=float('inf')).max()):.3g} times the bound"
    if kw:
        check_8bit(kw["h8"], kw["h8_scale"], h64, d)
        if dtype == F32:  # the 8-bit output is that of the fp32 h, bit for bit
            want, _, byte = ref.quantize(h.cpu())
            assert torch.equal(kw["h8_scale"].cpu().int(), byte.int())
            assert torch.equal(kw["h8"].cpu().view(torch.float8_e4m3fn).double(), want)


# every launch shape at its borders: a wavefront or a workgroup per row, cached and
# nontemporal outputs
@pytest.mark.parametrize("rows,d", [(1023, 512), (1024, 512), (1024, 520), (2047, 1024), (2048, 1024), (2049, 1032), (4095, 1032),
                                    (4096, 2048), (6143, 1536), (6144, 1536), (4097, 2880), (6143, 2080), (4096, 3080), (1030, 8192),
                                    (300, 8200)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_norm_launch_shapes(rows, d, dtype):
    from paper_2609_04895_amd import cmoe as B
    say("norm shapes", rows, d, dtype)
    g = torch.Generator(device="cuda").manual_seed(stable_seed(f"shapes {rows} {d}"))
    res = (torch.randn((rows, d), generator=g, device="cuda") * 4).to(dtype)
    delta, w = torch.randn((rows, d), generator=g, device="cuda"), (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    out, h = torch.empty_like(res), torch.empty_like(res)
    kw = {}
    if d % 32 == 0:
        kw = dict(h8=torch.empty((rows, d), dtype=torch.uint8, device="cuda"),
                  h8_scale=torch.empty((rows, d // 32), dtype=torch.uint8, device="cuda"))
    B.cmoe_add_norm(res, delta, w, 2.0 ** -20, residual_out=out, h=h, **kw)
    r, h64 = ref.norm(res.cpu(), delta.cpu(), w.cpu(), 2.0 ** -20)
    assert torch.equal(out.cpu(), r)
    off = (h.cpu().double() - h64).abs()
    assert (off <= 2.0 ** -24 * (1 + 2.0 ** -15) * h64.abs() + (2.0 ** -8 * h64.abs() if dtype == BF16 else 0.0) + 2.0 ** -150).all()
    if kw:
        check_8bit(kw["h8"], kw["h8_scale"], h64, d)


@pytest.mark.parametrize("rows,d", [(7, 64), (1030, 256), (5, 2880), (3, 50), (4, 8192)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_norm_infinities(rows, d, dtype):
    """An h beyond the type is infinite, so is one of an infinite weight; in a row with
    an infinity the finite places are 0, whatever their weights."""
    from paper_2609_04895_amd import cmoe as B
    g = torch.Generator().manual_seed(rows + d)
    res = (torch.randn((rows, d), generator=g) * torch.exp2(torch.arange(rows).float().remainder(40) - 20).unsqueeze(1)).to(dtype)
    res[:, 0], res[:, 1] = 0.0, res[:, 2] * 8  # a zero and a place with a large h
    res[2, 5], res[2, 7] = float("inf"), 2.0 ** 126
    w = torch.ones(d).to(dtype)
    w[1], w[7], w[9], w[11] = -2.0 ** 126, 2.0 ** 100, float("inf"), -float("inf")
    h = torch.empty_like(res, device="cuda")
    B.cmoe_add_norm(res.cuda(), None, w.cuda(), 2.0 ** -20, h=h)
    want = ref.norm(res, None, w, 2.0 ** -20)[1]
    got = h.cpu().double()
    largest = torch.finfo(dtype).max
    assert (want.abs() > 2 * largest).any() and torch.equal(got.isnan(), want.isnan())
    beyond, within = want.abs() > largest * (1 + 2.0 ** -8), want.abs() <= largest * (1 - 2.0 ** -7)
    assert (got[beyond].isinf() & (got[beyond].sign() == want[beyond].sign())).all()
    assert ((got - want).abs()[within] <= (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * (1 + 2.0 ** -14) * want.abs()[within]).all()
    assert (got[2][torch.isfinite(res[2]) & torch.isfinite(w)] == 0).all()

"""Outputs in other columns of a buffer that holds an input, and values with their scales
behind them in a row's record: calls that share no memory give what they give with
tensors of their own, and leave the rest of the buffer as it was."""
import pytest

import mx4_reference as mx
from gpu_util import stable_seed
from test_gpu_prompt import Model

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


def columns(buffer, at, cols, dtype):
    """Columns of a [rows][bytes] buffer as values of a type, from byte `at` on."""
    n = cols * torch.empty(0, dtype=dtype).element_size()
    first = at * cols // n
    return buffer.view(dtype)[:, first:first + cols]


def rows_of(bytes_, rows):
    return torch.full((rows, bytes_), 0x55, dtype=U8, device="cuda")


def untouched(buffer, *parts):
    """Whether all bytes but those of the parts (at, bytes) are as they were."""
    keep = torch.ones(buffer.shape[1], dtype=torch.bool, device="cuda")
    for at, n in parts:
        keep[at:at + n] = False
    return bool((buffer[:, keep] == 0x55).all())


@pytest.mark.parametrize("rows", [1, 7, 300])
def test_grouped_product_beside_its_input(rows):
    from paper_2609_04895_amd import cmoe as B
    g = torch.Generator().manual_seed(stable_seed(f"columns {rows}"))
    x = torch.randn((rows, 128), generator=g).to(BF16).cuda()
    w = torch.randn((2, 96, 128), generator=g).to(BF16).cuda()
    first = torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    # rows of 768 bytes: x, a gap of 16, y in bf16 or fp32 or 8 bits and its scales right behind
    for yt, each in ((BF16, 2), (F32, 4), (U8, 1)):
        buffer = rows_of(768, rows)
        bx, by = columns(buffer, 0, 128, BF16), columns(buffer, 272, 96, yt)
        bx.copy_(x)
        want, scale, by_scale = torch.empty((rows, 96), dtype=yt, device="cuda"), None, None
        if yt is U8:
            scale, by_scale = torch.empty((rows, 3), dtype=U8, device="cuda"), buffer[:, 272 + 96:272 + 99]
        B.cmoe_grouped_product(x, w, first, want, y_scale=scale)
        B.cmoe_grouped_product(bx, w, first, by, y_scale=by_scale)
        assert torch.equal(by, want) and torch.equal(bx, x)
        assert scale is None or torch.equal(by_scale, scale)
        assert untouched(buffer, (0, 256), (272, 96 * each + (3 if yt is U8 else 0)))


def test_one_row_between_the_rows_of_its_input():
    """x_row picks from many rows; y is the gap behind one of them."""
    from paper_2609_04895_amd import cmoe as B
    buffer = rows_of(512, 9)
    x, y = columns(buffer, 0, 64, BF16), columns(buffer, 128, 64, BF16)
    x.copy_(torch.arange(9 * 64, device="cuda").view(9, 64) % 13)
    w = torch.eye(64, device="cuda").to(BF16).unsqueeze(0)
    first, pick = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda")
    B.cmoe_grouped_product(x, w, first, y[4:5], x_row=pick)
    assert torch.equal(y[4], x[7]) and untouched(buffer[:4], (0, 128)) and untouched(buffer[4:5], (0, 256)) and untouched(buffer[5:], (0, 128))


@pytest.mark.parametrize("rows", [1, 5, 40])
def test_matvec_beside_its_input(rows):
    from paper_2609_04895_amd import cmoe as B
    g = torch.Generator().manual_seed(stable_seed(f"columns mv {rows}"))
    code, byte = mx.quantize4(torch.randn((77, 96), generator=g))
    x = torch.randn((rows, 96), generator=g).to(BF16).cuda()
    # a row of w is a record too: 48 bytes of values, their scales, 13 bytes of others
    wide = rows_of(64, 77)
    wide[:, :48], wide[:, 48:51] = mx.pack(code).cuda(), byte.to(U8).cuda()
    buffer = rows_of(768, rows)
    bx, by = columns(buffer, 0, 96, BF16), columns(buffer, 196, 77, F32)
    bx.copy_(x)
    want = torch.empty((rows, 77), device="cuda")
    B.cmoe_matvec(x, mx.pack(code).cuda(), byte.to(U8).cuda(), want)
    B.cmoe_matvec(bx, wide[:, :48], wide[:, 48:51], by)
    assert torch.equal(by, want) and torch.equal(bx, x) and untouched(buffer, (0, 192), (196, 77 * 4))


@pytest.mark.parametrize("format,each", [(1, 64), (2, 32)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_scales_and_source_in_one_record(format, each, dtype):
    from paper_2609_04895_amd import cmoe as B
    v = torch.randn((50, 64), generator=torch.Generator().manual_seed(format)).to(dtype).cuda()
    buffer = rows_of(400, 50)
    n = 64 * v.element_size()
    src, q, scale = columns(buffer, 0, 64, dtype), buffer[:, n:n + each], buffer[:, n + each:n + each + 2]
    src.copy_(v)
    want, want_scale = torch.empty((50, each), dtype=U8, device="cuda"), torch.empty((50, 2), dtype=U8, device="cuda")
    B.cmoe_quantize_as(format, v, want, want_scale)
    B.cmoe_quantize_as(format, src, q, scale)
    assert torch.equal(q, want) and torch.equal(scale, want_scale) and torch.equal(src, v) and untouched(buffer, (0, n + each + 2))


@pytest.mark.parametrize("kind", ["f32", "bf16", "w4a8"])
@pytest.mark.parametrize("T", [1, 30])
def test_prompt_layer_with_everything_in_one_buffer(kind, T):
    m = Model(kind, 1, 8, 2, 128, 64, T, f"columns {kind} {T}")
    h = m.hidden(T)
    eight, _ = m.eight(h)
    h = h.cuda()
    e, n = h.element_size(), 128 * h.element_size()
    buffer = rows_of(2 * n + 144, T)
    bh, by = columns(buffer, 0, 128, m.dtype), columns(buffer, n, 128, m.dtype)
    bh.copy_(h)
    kw = {}
    if eight:  # and h in 8 bits, its scales behind it
        kw = dict(h8=buffer[:, 2 * n:2 * n + 128], h8_scale=buffer[:, 2 * n + 128:2 * n + 132])
        kw["h8"].copy_(eight["h8"])
        kw["h8_scale"].copy_(eight["h8_scale"])
    want = torch.empty((T, 128), dtype=m.dtype, device="cuda")
    m.layers.cmoe_prompt_layer(0, h, want, **eight)
    m.layers.cmoe_prompt_layer(0, bh, by, **kw)
    assert torch.equal(by, want) and torch.equal(bh, h)
    assert untouched(buffer, (0, 2 * n + (132 if eight else 0)))

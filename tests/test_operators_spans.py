"""Whether an output shares memory with an input, for rows with strides: the library's own
check (csrc/places.h, host code) against every byte, and calls that it has to refuse.
No GPU needed; calls that it has to let through are in test_gpu_columns.py."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2609_04895_amd import cmoe as B
from test_operators_abi import P, error
from test_prompt_operators_abi import X8, Y8, product, vectors

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SRC = r"""
#include <cstdio>
#include "places.h"
int main() {
    long long v[8];
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6, v + 7) == 8) {
        using cmoe::host::Span;
        const Span a{(const void*)(uintptr_t)v[0], v[1], v[2], v[3]}, b{(const void*)(uintptr_t)v[4], v[5], v[6], v[7]};
        std::printf("%d%d%d\n", cmoe::host::meet(a, b), cmoe::host::meet(b, a), cmoe::host::apart({a}, {b}));
    }
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    """meet(a, b) of spans (address, rows, pitch, bytes of a row), in lists."""
    at = tmp_path_factory.mktemp("places")
    (at / "m.cpp").write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", "-I",
                    os.path.join(ROOT, "paper_2609_04895_amd", "csrc"), str(at / "m.cpp"), "-o", str(at / "m")], check=True)

    def run(pairs):
        text = "\n".join(" ".join(str(v) for v in (*a, *b)) for a, b in pairs)
        out = subprocess.run([str(at / "m")], input=text, check=True, capture_output=True, text=True).stdout.split()
        assert len(out) == len(pairs) and all(o in ("001", "110") for o in out)
        return [o == "110" for o in out]
    return run


def bytes_of(s):
    p, rows, pitch, row = s
    return {p + i * pitch + j for i in range(rows) for j in range(row)} if p else set()


def stretches_meet(a, b):
    return bool(bytes_of(a) and bytes_of(b)) and max(min(bytes_of(a)), min(bytes_of(b))) <= min(max(bytes_of(a)), max(bytes_of(b)))


def test_every_byte_of_small_spans(meet):
    rng = random.Random(3)
    pairs = []
    for _ in range(20000):
        pitch = rng.randint(1, 12)
        spans = []
        for k in range(2):
            own = pitch if rng.random() < 0.7 else rng.randint(1, 12)
            row = rng.randint(0, own) if rng.random() < 0.8 else own
            spans.append((rng.randint(100, 160), rng.randint(0, 6), own, row))
        pairs.append(tuple(spans))
    seen = set()
    for (a, b), got in zip(pairs, meet(pairs)):
        want = bool(bytes_of(a) & bytes_of(b))
        if got != want:  # rows at two distances, both with gaps: by their stretches
            assert got and stretches_meet(a, b) and a[2] != b[2] and min(a[1], b[1]) > 1 and a[2] != a[3] and b[2] != b[3], (a, b)
        seen.add((got, want, stretches_meet(a, b)))
    assert seen == {(False, False, False), (False, False, True), (True, True, True), (True, False, True)}


def test_long_spans(meet):
    """Far apart rows by their bytes; beyond 48 bits, whole, and without wrapping around."""
    at, far = 1 << 19, 1 << 30
    x = (at, 1 << 17, far, 256)
    assert meet([(x, (at + far, 1, 0, 1)), (x, (at + far - 1, 1, 0, 1)), (x, (at + 256, 1 << 17, far, far - 256)),
                 (x, (at + 256, 1 << 17, far, far - 255)), (x, (at + far // 2, 3, far, far // 2 + 1)), (x, (at + (far << 17) - 256, 4, far, far - 1)),
                 ((0, 4, 8, 8), (0, 4, 8, 8)), (x, (0, 5, 5, 5))]) == [True, False, False, True, True, False, False, False]
    x = (at, 1 << 30, 1 << 49, 256)
    assert meet([(x, (at + 300, 1, 0, 1)), (x, (at - 1, 1, 0, 1)), (x, (at + 300, 9, 1 << 49, 16))]) == [True, False, True]


# rows of x (bf16, 256 bytes) and of y (128 bytes) in one buffer of rows of 512 bytes
@pytest.mark.parametrize("at", [0, 128, 254, -126, 512 - 126, 7 * 512 + 254, -7 * 512 - 126, 3 * 512 + 100])
def test_columns_that_meet_are_refused(at):
    """y's first row `at` bytes behind x's."""
    assert B.lib().cmoe_grouped_product(ctypes.byref(product(x_stride=256, y=2 * P + at, y_stride=256)), None) == B.CMOE_ERR_INVALID_ARG
    assert "overlaps" in error()


def test_values_and_scales_that_meet_are_refused():
    """Records of 8-bit values with their scales behind them."""
    kw = dict(X8, **Y8, x_stride=256, x_scale=2 * P + 127, x_scale_stride=256, w_format=1, w_scale=5 * P, w_scale_stride=256)
    for y, scale in ((9 * P, 9 * P + 63), (9 * P, 9 * P + 255), (2 * P + 128, 7 * P), (2 * P + 132, 2 * P + 126), (2 * P + 132, 2 * P + 130)):
        a = product(**{**kw, "y": y, "y_stride": 256, "y_scale": scale, "y_scale_stride": 256})
        assert B.lib().cmoe_grouped_product(ctypes.byref(a), None) == B.CMOE_ERR_INVALID_ARG and "overlaps" in error()


def test_matvec_and_quantize_columns_that_meet_are_refused():
    a = vectors(x_stride=256, y=P + 188, y_stride=128)  # rows of 192 bytes of x, 512 apart
    assert B.lib().cmoe_matvec(ctypes.byref(a), None) == B.CMOE_ERR_INVALID_ARG and "overlaps" in error()
    for q, scale in ((P + 112, 3 * P), (2 * P, P + 127), (2 * P, 2 * P + 31), (P + 128, P + 159)):
        st = B.lib().cmoe_quantize_as(B.CMOE_FORMAT_MX4, P, B.CMOE_BF16, 4, 64, 128, q, 256, scale, 256, None)
        assert st == B.CMOE_ERR_INVALID_ARG and "overlaps" in error()


def test_8_bit_rows_that_meet_their_source_are_refused_too():
    for q, scale in ((P, 3 * P), (P + 112, 3 * P), (P - 48, 3 * P), (2 * P, P + 127), (2 * P, 2 * P + 63), (P + 128, P + 191)):
        st = B.lib().cmoe_quantize_as(B.CMOE_FORMAT_MX8, P, B.CMOE_BF16, 4, 64, 128, q, 256, scale, 256, None)
        assert st == B.CMOE_ERR_INVALID_ARG and "overlaps" in error()
    st = B.lib().cmoe_quantize_as(B.CMOE_FORMAT_MX8, P, B.CMOE_BF16, 4, 64, (1 << 48) + 64, 2 * P, 64, 3 * P, 2, None)
    assert st == B.CMOE_ERR_UNSUPPORTED and "2^48" in error()

"""The Python side of the operators without an expert cache, as far as it needs no
GPU: how a pool is cut into calls, and numbers that no argument can hold."""
import pytest

from paper_2609_04895_amd import cmoe as B

torch = pytest.importorskip("torch")

LIMIT = 1 << 34  # values of one cmoe_quantize call


@pytest.mark.parametrize("L,N,n", [(1, 256, 3 * 8192 * 4096),      # a layer beyond the limit
                                   (48, 128, 3 * 4096 * 1536),     # a model beyond it
                                   (3, 5, 3 * 65536 * 65536),      # the largest expert, an odd number of them
                                   (1, 2, LIMIT + 32),             # an expert beyond the limit
                                   (2, 3, 96), (0, 4, 96), (2, 0, 96)])
def test_quantize_experts_covers_pools_of_any_size(monkeypatch, L, N, n):
    """Every value goes into one call, its scale beside it, no call over the limit
    (tensors without memory)."""
    done = []

    def quantize(src, q, scale, stream=None):
        rows, cols = src.shape
        assert rows * cols <= LIMIT and cols % 32 == 0
        assert q.shape == (rows, cols) and scale.shape == (rows, cols // 32)
        assert src.is_contiguous() and q.is_contiguous() and scale.is_contiguous()
        at = src.storage_offset()
        assert at * 2 % 16 == 0 and q.storage_offset() == at and scale.storage_offset() == at // 32
        done.append((at, rows * cols))

    monkeypatch.setattr(B, "cmoe_quantize", quantize)
    pool = torch.empty((L, N, n), dtype=torch.bfloat16, device="meta")
    q, scale = B.quantize_experts(pool)
    assert q.shape == (L, N, n) and scale.shape == (L, N, n // 32) and q.dtype == scale.dtype == torch.uint8
    at = 0
    for start, count in sorted(done):
        assert start == at
        at += count
    assert at == L * N * n


def layers_on_the_host():
    """A MoeLayers without a library handle, on host tensors: its calls pack their
    arguments and are refused by the library at the latest."""
    m = object.__new__(B.MoeLayers)
    m.handle, m.device, m.L, m.K, m.d, m.dtype = None, -1, 2, 2, 64, torch.bfloat16
    m.norm_weight, m.norm_eps = None, 1e-6
    return m


@pytest.mark.parametrize("eps", [1e39, -1e300, float("inf"), float("nan")])
def test_norm_eps_that_fp32_cannot_hold(eps):
    r = torch.zeros((4, 64))
    with pytest.raises(B.CmoeError) as err:
        B.cmoe_add_norm(r, eps=eps, residual_out=r)
    assert err.value.status == B.CMOE_ERR_INVALID_ARG


@pytest.mark.parametrize("layer", [1 << 31, -(1 << 31) - 1, 1 << 80, 0.5])
def test_layers_that_no_argument_can_hold(layer):
    m, h, y = layers_on_the_host(), torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((4, 64))
    for call in (lambda: m.cmoe_moe_layer(layer, h, y), lambda: m.cmoe_moe_block(layer, h, None, y)):
        with pytest.raises(B.CmoeError) as err:
            call()
        assert err.value.status == B.CMOE_ERR_INVALID_ARG


def test_rows_that_no_argument_can_hold():
    r = torch.empty((1 << 31, 1), device="meta").as_strided((1 << 31, 1), (1, 1))
    with pytest.raises(B.CmoeError) as err:
        B.cmoe_add_norm(r, residual_out=r)
    assert err.value.status == B.CMOE_ERR_INVALID_ARG

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

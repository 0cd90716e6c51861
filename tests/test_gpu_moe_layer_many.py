"""cmoe_moe_layer with many tokens: experts of more than a unit of tokens over many
lines of weights per wavefront, in every format and with rows of whole and of half
lines, and the launches above 32 tokens with masks, padding, non-finite rows and
replays."""
import math

import pytest

import operator_reference as ref
import test_gpu_moe_layer as few
from gpu_util import say
from moe_rms import rms_bound, rms_error
from test_gpu_moe_layer import KINDS, Model, check, outputs
from test_gpu_norm import check_8bit, check_h

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# N, K, d, F, T and sizes of units (tokens of an expert in one pass) that have to occur
SHAPES = [(4, 2, 2112, 2112, 64, range(11, 17)), (4, 2, 2048, 2048, 64, range(11, 17)), (4, 2, 2112, 2048, 40, range(11, 17)),
          (4, 2, 2048, 2112, 40, range(11, 17)), (8, 2, 1088, 2112, 32, range(6, 11)), (8, 2, 1088, 2048, 32, range(6, 11)),
          (16, 2, 1088, 2112, 33, range(3, 6)), (16, 2, 2048, 1088, 33, range(3, 6))]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,K,d,F,T,units", SHAPES, ids=["x".join(map(str, s[:5])) for s in SHAPES])
def test_many_tokens_of_an_expert_over_many_lines(N, K, d, F, T, units, kind):
    """Every value within its bound, and their root mean square within what fp32 sums
    are off by on the average."""
    say("many", kind, N, K, d, F, T)
    m = Model(kind, 1, N, K, d, F, T, f"many {kind} {N} {K} {d} {F} {T}", sigma=0.02)
    layers, h = m.layers(), m.hidden(T)
    eight, x = m.eight(h)
    y, sel, gates = outputs(T, K, d)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
    want = m.expected(0, h, x)
    tokens = torch.bincount(want[0].flatten().long(), minlength=N).tolist()
    assert any(n in units for c in tokens for n in ([16] * (c // 16) + [c % 16]))
    check((y, sel, gates), want, K)
    assert rms_error(y.cpu(), want[2]) <= rms_bound(d, F, K)
    layers.cmoe_moe_destroy()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,K,d,F,T", [(128, 8, 2048, 768, 1), (60, 6, 704, 448, 13), (64, 4, 1024, 512, 3)])
def test_few_tokens_on_the_average(N, K, d, F, T, kind):
    say("average", kind, N, K, d, F, T)
    m = Model(kind, 1, N, K, d, F, T, f"average {kind} {N} {T}", sigma=0.02)
    h = m.hidden(T)
    eight, x = m.eight(h)
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
    want = m.expected(0, h, x)
    check((y, sel, gates), want, K)
    assert rms_error(y.cpu(), want[2]) <= rms_bound(d, F, K)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [33, 64])
def test_masks_above_32_tokens(kind, T):
    few.test_masks_that_leave_few_experts_or_none(kind, 12, T)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,n", [(64, n) for n in (-1, 0, 1, 17, 33, 61, 64, 99)] + [(33, 32)])
def test_padding_above_32_tokens(kind, T, n):
    few.test_rows_behind_the_last_token_are_left(kind, 16, T, n)


@pytest.mark.parametrize("kind", KINDS)
def test_non_finite_rows_above_32_tokens(kind):
    N, K, d, F, T = 16, 3, 128, 64, 50
    m = Model(kind, 1, N, K, d, F, T, f"nan many {kind}")
    h = m.hidden(T)
    eight, x = m.eight(h)
    want = m.expected(0, h, x)
    bad = h.clone()
    bad[4, 100], bad[40, 0], bad[40, 1], bad[49, 127] = math.nan, math.inf, -math.inf, math.nan
    eight, _ = m.eight(bad)
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, bad.cuda(), y, selected=sel, gates=gates, **eight)
    check((y, sel, gates), want, K, rows=[t for t in range(T) if t not in (4, 40, 49)])
    for t in (4, 40, 49):
        assert y[t].isnan().all()
    assert sel[4].tolist() == sel[49].tolist() == list(range(K)) and ((sel >= 0) & (sel < N)).all()


@pytest.mark.parametrize("kind", KINDS)
def test_graph_replays_above_32_tokens(kind):
    """A captured call, replayed with other inputs and counts from 56 down to none."""
    N, K, d, F, T = 20, 3, 256, 128, 56
    m = Model(kind, 1, N, K, d, F, T, f"graph many {kind}")
    st = torch.cuda.Stream()
    layers, h = m.layers(stream=st), m.hidden(T)
    eight, _ = m.eight(h)
    hg, n = h.cuda(), torch.tensor([T], dtype=torch.int32, device="cuda")
    y, sel, gates = outputs(T, K, d)

    def call():
        layers.cmoe_moe_layer(0, hg, y, n_tokens=n, selected=sel, gates=gates, **eight)

    torch.cuda.synchronize()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for live in (56, 40, 33, 32, 7, 0, 56):
        h = m.hidden(T)
        new, x = m.eight(h)
        for k in new:
            eight[k].copy_(new[k])
        hg.copy_(h)
        n.fill_(live)
        for t in (y, sel, gates):
            t.fill_(2)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, sel, gates)]
        check(tuple(t[:live] for t in got), m.expected(0, h[:live], x[:live]), K)
        assert all((t[live:] == 2).all() for t in got)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, sel, gates))), live


@pytest.mark.parametrize("kind", ["f32", "bf16", "w8a8"])
@pytest.mark.parametrize("T", [1, 40])
def test_the_last_norm_behind_the_layers(kind, T):
    """A decoder's end: the last block's output added to the residual in place, h and
    its 8-bit form for the head."""
    N, K, d, F = 24, 4, 256, 192
    m = Model(kind, 1, N, K, d, F, T, f"last {kind} {T}")
    res, y = m.hidden(T).cuda(), torch.zeros((T, d), device="cuda")
    m.layers().cmoe_moe_block(0, res, None, y)
    before = res.cpu()
    h, q, s = torch.empty_like(res), torch.empty((T, d), dtype=torch.uint8, device="cuda"), \
        torch.empty((T, d // 32), dtype=torch.uint8, device="cuda")
    m.B.cmoe_add_norm(res, y, m.norm_weight[0].cuda(), 1e-6, residual_out=res, h=h, h8=q, h8_scale=s)
    r, h64 = ref.norm(before, y.cpu(), m.norm_weight[0], 1e-6)
    assert torch.equal(res.cpu(), r) and not torch.equal(r, before)
    check_h(h, h64, d, m.dtype)
    check_8bit(q, s, h64, d)


def test_one_fp32_token_of_large_experts():
    """One token of 265 MB of fp32 experts."""
    N, K, d, F, T = 5, 4, 2880, 1920, 1
    m = Model("f32", 1, N, K, d, F, T, "one large", sigma=0.02)
    layers, h = m.layers(), m.hidden(T)
    y, sel, gates = outputs(T, K, d)
    for n in (0, 1):
        layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, n_tokens=torch.tensor([n], dtype=torch.int32, device="cuda"))
        if n == 0:
            assert (y == 7).all() and (sel == -9).all() and (gates == 9).all()
    want = m.expected(0, h, h.double())
    check((y, sel, gates), want, K)
    assert rms_error(y.cpu(), want[2]) <= rms_bound(d, F, K)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,d,T", [(24, 3, 2496, 1), (24, 3, 2560, 1), (24, 3, 1216, 2), (24, 3, 1280, 2), (48, 3, 640, 4), (48, 3, 576, 4)])
def test_tokens_alone_on_half_and_on_whole_tiles(kind, N, K, d, T):
    """Both sides of 160 tiles of outputs, where the down product's tiles change."""
    F = 192
    m = Model(kind, 1, N, K, d, F, T, f"tiles {kind} {d} {T}", sigma=0.02)
    layers, h = m.layers(), m.hidden(T)
    y, sel, gates = outputs(T, K, d)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates)
    want = m.expected(0, h, h.double())
    check((y, sel, gates), want, K)
    assert rms_error(y.cpu(), want[2]) <= rms_bound(d, F, K)
    y2, _, _ = outputs(T, K, d)
    layers.cmoe_moe_layer(0, h.cuda(), y2, n_tokens=torch.tensor([T - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(y2[:T - 1], y[:T - 1]) and (y2[T - 1:] == 7).all()

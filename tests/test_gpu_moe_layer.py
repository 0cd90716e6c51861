"""cmoe_moe_layer and cmoe_moe_block against fp64 forms: selections exactly,
gates and outputs within the bounds that operator_reference derives; sizes from
one token and one expert to 64 tokens, 256 experts and Top-64, weights in fp32,
bf16 and 8 bits, masks, ties, non-finite values, padding, strides, layers,
offsets past 32 bits, graphs, streams, and a run of all calls together."""
import math

import pytest

import operator_reference as ref
from gpu_util import say, stable_seed

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
KINDS = ["f32", "bf16", "w8", "w8a8"]


class Model:
    """L layers' weights on the device and as the fp64 values they stand for."""

    def __init__(self, kind, L, N, K, d, F, T, seed, bias=None, sigma=0.05):
        from paper_2609_04895_amd import cmoe as B
        g = torch.Generator().manual_seed(stable_seed(seed))
        self.B, self.kind, self.shape = B, kind, (L, N, K, d, F, T)
        self.dtype = F32 if kind == "f32" else BF16
        self.router = (torch.randn((L, N, d), generator=g) * 0.1).to(self.dtype)
        self.bias = bias
        pool = (torch.randn((L, N, 3 * d * F), generator=g) * sigma).to(self.dtype)
        self.gpu = dict(w_router=self.router.cuda(), logit_bias=None if bias is None else bias.cuda(), experts=pool.cuda(),
                        expert_scales=None)
        self.norm_weight = (1 + 0.1 * torch.randn((L, d), generator=g)).to(self.dtype)
        self.pool, self.scales = pool, None
        if kind in ("w8", "w8a8"):
            self.gpu["experts"], self.gpu["expert_scales"] = B.quantize_experts(pool.cuda())
            self.pool, self.scales = self.gpu["experts"].cpu(), self.gpu["expert_scales"].cpu()
        self.gen = g

    def config(self):
        B = self.B
        L, N, K, d, F, T = self.shape
        return B.make_moe_config(L, N, K, d, F, T, B.CMOE_F32 if self.kind == "f32" else B.CMOE_BF16,
                                 B.CMOE_FORMAT_MX8 if self.kind in ("w8", "w8a8") else B.CMOE_FORMAT_DTYPE,
                                 B.CMOE_FORMAT_MX8 if self.kind == "w8a8" else B.CMOE_FORMAT_DTYPE)

    def layers(self, stream=None):
        return self.B.MoeLayers(self.config(), **self.gpu, norm_weight=self.norm_weight.cuda(), stream=stream)

    def weights(self, layer):
        _, _, _, d, F, _ = self.shape

        def of(e):
            w = self.pool[layer, e]
            return ref.split_expert(w if self.scales is None else ref.dequantize(w, self.scales[layer, e]), d, F)
        return of

    def hidden(self, T):
        return torch.randn((T, self.shape[3]), generator=self.gen).to(self.dtype)

    def eight(self, h):
        """(arguments, fp64 values) of the experts' input for the rows h."""
        if self.kind != "w8a8":
            return {}, h.double()
        q = torch.empty(h.shape, dtype=torch.uint8, device="cuda")
        s = torch.empty((h.shape[0], h.shape[1] // 32), dtype=torch.uint8, device="cuda")
        self.B.cmoe_quantize(h.cuda(), q, s)
        return dict(h8=q, h8_scale=s), ref.dequantize(q.cpu(), s.cpu())

    def expected(self, layer, h, x):
        K, d, F = self.shape[2], self.shape[3], self.shape[4]
        sel, gates, _ = ref.route(h, self.router[layer], None if self.bias is None else self.bias[layer], K)
        y, err = ref.experts(x, sel, gates, self.weights(layer), d, F)
        return sel, gates, y, err


def outputs(T, K, d):
    return (torch.full((T, d), 7.0, device="cuda"), torch.full((T, K), -9, dtype=torch.int32, device="cuda"),
            torch.full((T, K), 9.0, device="cuda"))


def check(got, want, K, rows=slice(None)):
    y, sel, gates = got
    esel, egates, ey, err = want
    assert torch.equal(sel.cpu()[rows], esel[rows])
    # the difference D of two logits is rounded to fp32 before its exponential: off by u D, the gate by the factor e^(u D)
    gap = (egates[rows][:, :1].clamp(min=1e-300) / egates[rows].clamp(min=1e-300)).log()
    assert ((gates.cpu()[rows].double() - egates[rows]).abs() <= (2 * K + 16 + gap) * ref.U * egates[rows] + 1e-37).all()
    off = (y.cpu()[rows].double() - ey[rows]).abs()
    assert (off <= err[rows] + 1e-37).all(), f"{(off / err[rows].clamp(min=1e-300)).max():.3g} times the bound"


SHAPES = [(1, 1, 64, 64, 1), (5, 3, 64, 128, 2), (3, 1, 64, 64, 64), (4, 2, 128, 64, 33), (2, 2, 4160, 64, 5),
          (8, 2, 64, 4160, 3), (60, 6, 704, 448, 13), (128, 8, 256, 192, 64), (128, 8, 2048, 768, 1), (4, 2, 2880, 320, 7),
          (256, 64, 128, 64, 64), (200, 5, 192, 64, 61), (256, 6, 192, 320, 4), (64, 5, 128, 192, 3), (64, 64, 64, 64, 9), (130, 17, 320, 128, 17),
          (64, 64, 64, 64, 1), (256, 40, 128, 4160, 1), (2, 1, 65536, 64, 1), (2, 2, 65536, 64, 9), (2, 1, 64, 65536, 1), (2, 2, 64, 65536, 6)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,K,d,F,T", SHAPES)
def test_layer_matches_fp64(N, K, d, F, T, kind):
    say("moe layer", kind, N, K, d, F, T)
    m = Model(kind, 1, N, K, d, F, T, f"layer {kind} {N} {K} {d} {F} {T}", sigma=0.05 if N * d * F < 1e7 else 0.02)
    layers = m.layers()
    h = m.hidden(T)
    eight, x = m.eight(h)
    y, sel, gates = outputs(T, K, d)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
    want = m.expected(0, h, x)
    check((y, sel, gates), want, K)
    # fewer rows than the configuration takes, without the optional outputs, twice: the same values
    for t in {1, (T + 1) // 2, T}:
        y2 = torch.full((t, d), 7.0, device="cuda")
        layers.cmoe_moe_layer(0, h[:t].cuda(), y2, **{k: v[:t] for k, v in eight.items()})
        check((y2, sel[:t], gates[:t]), tuple(v[:t] for v in want), K)
        if t == T:
            assert torch.equal(y2, y)
    layers.cmoe_moe_destroy()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,T", [(12, 1), (12, 20), (48, 3)])
def test_masks_that_leave_few_experts_or_none(kind, N, T):
    """Bias -inf takes experts out, whatever their router row and weights hold."""
    K, d, F = 4, 128, 64
    for out in (3, N - 2, N):
        bias = torch.randn((1, N), generator=torch.Generator().manual_seed(out)) * 0.3
        bias[0, :out] = -math.inf
        m = Model(kind, 1, N, K, d, F, T, f"mask {kind} {out}", bias=bias)
        m.gpu["w_router"][0, :out] = math.nan
        if kind in ("w8", "w8a8"):
            m.gpu["experts"][0, :out] = 0x7F
            m.gpu["expert_scales"][0, :out] = 255
        else:
            m.gpu["experts"][0, :out] = math.nan
        m.router[0, :out] = 0.0
        layers = m.layers()
        h = m.hidden(T)
        eight, x = m.eight(h)
        y, sel, gates = outputs(T, K, d)
        layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
        check((y, sel, gates), m.expected(0, h, x), K)
        if out == N:
            assert (sel == -1).all() and (gates == 0).all() and (y == 0).all()
        else:
            assert ((sel >= out) | (sel == -1)).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_lowest_type_value_as_mask(kind):
    """A bias of the type's lowest value is a number: such experts come last, with gate 0, and are still selected."""
    N, K, d, F, T = 6, 4, 64, 64, 3
    bias = torch.zeros((1, N))
    bias[0, 2:] = torch.finfo(torch.float32).min
    m = Model(kind, 1, N, K, d, F, T, f"lowest {kind}", bias=bias)
    h = m.hidden(T)
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates)
    want = m.expected(0, h, h)
    check((y, sel, gates), want, K)
    assert (gates[:, 2:] == 0).all() and (sel[:, 2:] >= 2).all()


def test_equal_logits_take_the_lower_index():
    N, K, d, F, T = 70, 6, 64, 64, 5
    m = Model("f32", 1, N, K, d, F, T, "ties")
    m.router[0] = m.router[0, :7].repeat(10, 1)
    m.router[0, 65] = -0.0
    m.router[0, 3] = 0.0
    m.gpu["w_router"] = m.router.cuda()
    h = m.hidden(T)
    h[0] = 0.0   # every logit 0 or -0
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates)
    check((y, sel, gates), m.expected(0, h, h), K)
    assert sel[0].tolist() == list(range(K))


@pytest.mark.parametrize("kind", KINDS)
def test_non_finite_rows_stay_alone(kind):
    """NaN and infinity in some tokens' hidden states: those rows are NaN, the
    others what they are without them."""
    N, K, d, F, T = 16, 3, 128, 64, 24
    m = Model(kind, 1, N, K, d, F, T, f"nan {kind}")
    h = m.hidden(T)
    eight, x = m.eight(h)
    want = m.expected(0, h, x)
    bad = h.clone()
    bad[4, 100] = math.nan
    bad[9, 0] = math.inf
    bad[9, 1] = -math.inf
    eight, _ = m.eight(bad)
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, bad.cuda(), y, selected=sel, gates=gates, **eight)
    good = [t for t in range(T) if t not in (4, 9)]
    check((y, sel, gates), want, K, rows=good)
    assert y[4].isnan().all() and y[9].isnan().all() and gates[4].isnan().all()
    assert sel[4].tolist() == list(range(K)) and ((sel >= 0) & (sel < N)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,T,n", [(16, 20, n) for n in (-1, 0, 1, 17, 20, 99)] + [(64, 4, n) for n in (-1, 0, 1, 3, 4, 9)])
def test_rows_behind_the_last_token_are_left(kind, N, T, n):
    K, d, F = 3, 128, 64
    live = min(max(n, 0), T)
    m = Model(kind, 1, N, K, d, F, T, f"padding {kind}")
    h = m.hidden(T)
    h[live:] = math.nan
    eight, x = m.eight(h)
    y, sel, gates = outputs(T, K, d)
    layers = m.layers()
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, n_tokens=torch.tensor([n], dtype=torch.int32, device="cuda"), **eight)
    check(tuple(v[:live] for v in (y, sel, gates)), m.expected(0, h[:live], x[:live]), K)
    assert (y[live:] == 7).all() and (sel[live:] == -9).all() and (gates[live:] == 9).all()
    # a full call after it on the same workspace
    h = m.hidden(T)
    eight, x = m.eight(h)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
    check((y, sel, gates), m.expected(0, h, x), K)


@pytest.mark.parametrize("kind", KINDS)
def test_one_token_padded_away_and_one_of_nan(kind):
    """The single-token launches: no token leaves every output, a NaN is the token's own."""
    N, K, d, F = 16, 3, 128, 64
    m = Model(kind, 1, N, K, d, F, 1, f"one {kind}")
    layers, h = m.layers(), m.hidden(1)
    y, sel, gates = outputs(1, K, d)
    for n in (0, 1):
        eight, x = m.eight(h)
        layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, n_tokens=torch.tensor([n], dtype=torch.int32, device="cuda"), **eight)
        if n == 0:
            assert (y == 7).all() and (sel == -9).all() and (gates == 9).all()
        else:
            check((y, sel, gates), m.expected(0, h, x), K)
    bad = h.clone()
    bad[0, 5] = math.nan
    eight, _ = m.eight(bad)
    layers.cmoe_moe_layer(0, bad.cuda(), y, selected=sel, gates=gates, **eight)
    assert y.isnan().all() and gates.isnan().all() and sel.tolist() == [[0, 1, 2]]
    eight, x = m.eight(h)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates, **eight)
    check((y, sel, gates), m.expected(0, h, x), K)


@pytest.mark.parametrize("T", [1, 6])
@pytest.mark.parametrize("d,F", [(192, 64), (128, 192), (256, 256)])
def test_8_bit_blocks_of_zeros_and_of_tiny_values(T, d, F):
    """Scale bytes 0 (zeros) and near it, beside ordinary blocks; rows that end in half a line and rows that do not."""
    N, K = 5, 2
    m = Model("w8", 1, N, K, d, F, T, f"tiny {T} {d} {F}")
    pool = torch.randn((1, N, 3 * d * F), generator=m.gen) * 0.05
    b = pool.view(1, N, -1, 32)
    b[:, :, ::3] = 0.0
    b[:, :, 1::7] *= 2.0 ** -100
    b[:, 0] = 0.0
    m.gpu["experts"], m.gpu["expert_scales"] = m.B.quantize_experts(pool.cuda())
    m.pool, m.scales = m.gpu["experts"].cpu(), m.gpu["expert_scales"].cpu()
    assert (m.scales == 0).any()
    h = m.hidden(T)
    y, sel, gates = outputs(T, K, d)
    m.layers().cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates)
    check((y, sel, gates), m.expected(0, h, h), K)


@pytest.mark.parametrize("kind", KINDS)
def test_layers_and_rows_apart(kind):
    """Rows of [T][L][d] buffers, each layer with its own weights and bias."""
    L, N, K, d, F, T = 3, 10, 3, 192, 64, 6
    bias = torch.randn((L, N), generator=torch.Generator().manual_seed(2)) * 0.5
    m = Model(kind, L, N, K, d, F, T, f"layers {kind}", bias=bias)
    layers = m.layers()
    h = torch.stack([m.hidden(T) for _ in range(L)], 1)
    hg, y = h.cuda(), torch.full((T, L + 1, d), 7.0, device="cuda")
    for l in (2, 0, 1):
        eight, x = m.eight(h[:, l].contiguous())
        if eight:  # 8-bit rows apart too
            q, s = torch.zeros((T, d + 16), dtype=torch.uint8, device="cuda"), torch.zeros((T, d // 32 + 3), dtype=torch.uint8, device="cuda")
            q[:, :d], s[:, :d // 32] = eight["h8"], eight["h8_scale"]
            eight = dict(h8=q[:, :d], h8_scale=s[:, :d // 32])
        _, sel, gates = outputs(T, K, d)
        layers.cmoe_moe_layer(l, hg[:, l], y[:, l], selected=sel, gates=gates, **eight)
        check((y[:, l], sel, gates), m.expected(l, h[:, l], x), K)
    assert (y[:, L] == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "w8"])
def test_weight_offsets_past_32_bits(kind):
    """The last experts of a pool of more than 2^32 values."""
    N, K, d, F, T = 250, 4, 2880, 2048, 3
    from paper_2609_04895_amd import cmoe as B
    g = torch.Generator(device="cuda").manual_seed(4)
    router = (torch.randn((1, N, d), generator=g, device="cuda") * 0.1).to(BF16)
    bias = torch.zeros((1, N), device="cuda")
    bias[0, N - 6:] = 60.0
    n = 3 * d * F
    assert (N - 6) * n > 1 << 32
    pool = torch.zeros((1, N, n), dtype=BF16, device="cuda")
    pool[0, N - 6:].normal_(0.0, 0.02, generator=g)
    w8 = kind == "w8"
    experts, scales = B.quantize_experts(pool) if w8 else (pool, None)
    cfg = B.make_moe_config(1, N, K, d, F, T, B.CMOE_BF16, B.CMOE_FORMAT_MX8 if w8 else B.CMOE_FORMAT_DTYPE)
    layers = B.MoeLayers(cfg, router, bias, experts, scales)
    h = torch.randn((T, d), generator=torch.Generator().manual_seed(5)).to(BF16)
    y, sel, gates = outputs(T, K, d)
    layers.cmoe_moe_layer(0, h.cuda(), y, selected=sel, gates=gates)

    def weights(e):
        w = experts[0, e].cpu()
        return ref.split_expert(ref.dequantize(w, scales[0, e].cpu()) if w8 else w, d, F)
    esel, egates, _ = ref.route(h, router[0].cpu(), bias[0].cpu(), K)
    check((y, sel, gates), (esel, egates, *ref.experts(h.double(), esel, egates, weights, d, F)), K)
    assert (sel >= N - 6).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,with_delta", [(1, True), (9, True), (9, False)])
def test_block_is_norm_then_layer(kind, T, with_delta):
    """The same bits as the two calls, in place too."""
    L, N, K, d, F = 2, 16, 4, 256, 128
    m = Model(kind, L, N, K, d, F, T, f"block {kind}")
    B, layers = m.B, m.layers()
    res = (m.hidden(T) * 4).cuda()
    delta = torch.randn((T, d), generator=m.gen).cuda() if with_delta else None
    for l in range(L):
        r, h = torch.empty_like(res), torch.empty_like(res)
        kw = {}
        if kind == "w8a8":
            kw = dict(h8=torch.empty((T, d), dtype=torch.uint8, device="cuda"),
                      h8_scale=torch.empty((T, d // 32), dtype=torch.uint8, device="cuda"))
        B.cmoe_add_norm(res, delta, m.norm_weight[l].cuda(), 1e-6, residual_out=r, h=h, **kw)
        y, sel, gates = outputs(T, K, d)
        layers.cmoe_moe_layer(l, h, y, selected=sel, gates=gates, **kw)
        y2, sel2, gates2 = outputs(T, K, d)
        r2 = res.clone()
        layers.cmoe_moe_block(l, r2, delta, y2, residual_out=r2, selected=sel2, gates=gates2)
        assert torch.equal(r2, r) and torch.equal(y2, y) and torch.equal(sel2, sel) and torch.equal(gates2, gates)
        y3, _, _ = outputs(T, K, d)
        layers.cmoe_moe_block(l, res, delta, y3)
        assert torch.equal(y3, y)
        if with_delta:  # y in delta's place
            y4 = delta.clone()
            layers.cmoe_moe_block(l, res, y4, y4)
            assert torch.equal(y4, y)


@pytest.mark.parametrize("n", [0, 5])
def test_block_leaves_rows_behind_the_last_token(n):
    N, K, d, F, T = 16, 4, 256, 128, 8
    m = Model("bf16", 1, N, K, d, F, T, "block padding")
    layers = m.layers()
    res, delta = m.hidden(T).cuda(), torch.randn((T, d), generator=m.gen).cuda()
    y, sel, gates = outputs(T, K, d)
    r = torch.full_like(res, 3.0)
    layers.cmoe_moe_block(0, res, delta, y, residual_out=r, selected=sel, gates=gates,
                          n_tokens=torch.tensor([n], dtype=torch.int32, device="cuda"))
    assert (y[n:] == 7).all() and (r[n:] == 3).all() and (sel[n:] == -9).all() and (gates[n:] == 9).all()
    if n:
        y2, _, _ = outputs(n, K, d)
        layers.cmoe_moe_block(0, res[:n], delta[:n], y2)
        assert torch.equal(y2, y[:n])


@pytest.mark.parametrize("kind", ["f32", "bf16", "w8a8"])
def test_a_token_through_all_layers(kind):
    """The calls together as a decoder makes them: each layer's block on the
    residual stream, its output the next one's delta, then the last norm.  Each
    layer is compared with fp64 on the library's own inputs, so that a near tie
    of one layer cannot become the next one's difference."""
    L, N, K, d, F, T = 4, 24, 4, 256, 192, 5
    m = Model(kind, L, N, K, d, F, T, f"chain {kind}")
    B, layers = m.B, m.layers()
    res, delta = (m.hidden(T) * 2).cuda(), torch.randn((T, d), generator=m.gen).cuda()
    for l in range(L):
        before, before_delta = res.clone(), delta.clone()
        y, sel, gates = outputs(T, K, d)
        layers.cmoe_moe_block(l, res, delta, y, residual_out=res, selected=sel, gates=gates)
        r, h64 = ref.norm(before.cpu(), before_delta.cpu(), m.norm_weight[l], 1e-6)
        assert torch.equal(res.cpu(), r)
        h = torch.empty_like(res)
        kw = dict(h8=torch.empty((T, d), dtype=torch.uint8, device="cuda"),
                  h8_scale=torch.empty((T, d // 32), dtype=torch.uint8, device="cuda")) if kind == "w8a8" else {}
        B.cmoe_add_norm(before, before_delta, m.norm_weight[l].cuda(), 1e-6, h=h, **kw)
        tol = ref.norm_error(d) + (ref.HALF[BF16] if kind != "f32" else 0)
        assert ((h.cpu().double() - h64).abs() <= 1.01 * tol * h64.abs()).all()
        x = ref.dequantize(kw["h8"].cpu(), kw["h8_scale"].cpu()) if kw else h.cpu().double()
        check((y, sel, gates), m.expected(l, h.cpu(), x), K)
        delta = y
    last, q, s = torch.empty_like(res), torch.empty((T, d), dtype=torch.uint8, device="cuda"), \
        torch.empty((T, d // 32), dtype=torch.uint8, device="cuda")
    B.cmoe_add_norm(res, delta, None, 1e-6, residual_out=res, h=last, h8=q, h8_scale=s)
    assert torch.isfinite(last).all()


def test_same_selections_and_outputs_as_the_decode_step():
    """The layer and cmoe_step on one pool, one router: equal selections and
    gates, outputs within the step's bf16 bound (2e-2 of the largest)."""
    import synth
    from paper_2609_04895_amd import cmoe as B
    from paper_2609_04895_amd.workload import engine_for
    w = synth.WORKLOADS["qwen3_30b"].replace(name="layer_vs_step", L=3, N=32, K=4, C=8, d=256, F=128, S=12)
    inp = synth.device_inputs(w, T=2)
    eng = engine_for(w, inp)
    y = torch.empty((w.S, w.L, w.d), dtype=torch.float32, device="cuda")
    cfg = B.make_moe_config(w.L, w.N, w.K, w.d, w.F, w.S, B.CMOE_BF16)
    layers = B.MoeLayers(cfg, eng._keep[0], eng._keep[3], eng._keep[4])
    for t in range(2):
        eng.cmoe_step(inp["hidden"][t], y)
        step_sel, step_gates = eng.cmoe_read(B.CMOE_VIEW_SELECTED), eng.cmoe_read(B.CMOE_VIEW_GATES)
        h = inp["hidden"][t].view(w.S, w.L, w.d)
        for l in range(w.L):
            y2, sel, gates = outputs(w.S, w.K, w.d)
            layers.cmoe_moe_layer(l, h[:, l], y2, selected=sel, gates=gates)
            assert (sel.cpu().numpy() == step_sel[l]).all()
            assert abs(gates.cpu().numpy() - step_gates[l]).max() <= 2e-6
            off = (y2 - y[:, l]).abs().amax(1) / y2.abs().amax(1)
            assert float(off.max()) <= 2e-2
    eng.cmoe_destroy()


@pytest.mark.parametrize("kind", KINDS)
def test_graph_replays(kind):
    """A captured block and layer, replayed with other inputs and token counts
    between eager calls of the same handle."""
    N, K, d, F, T = 20, 3, 256, 128, 18
    m = Model(kind, 1, N, K, d, F, T, f"graph {kind}")
    st = torch.cuda.Stream()
    layers = m.layers(stream=st)
    res, delta = m.hidden(T).cuda(), torch.randn((T, d), generator=m.gen).cuda()
    h = m.hidden(T)
    eight, _ = m.eight(h)
    hg = h.cuda()
    n = torch.tensor([T], dtype=torch.int32, device="cuda")
    (yb, sb, gb), (yl, sl, gl) = outputs(T, K, d), outputs(T, K, d)
    r = torch.empty_like(res)

    def call():
        layers.cmoe_moe_block(0, res, delta, yb, residual_out=r, n_tokens=n, selected=sb, gates=gb)
        layers.cmoe_moe_layer(0, hg, yl, n_tokens=n, selected=sl, gates=gl, **eight)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        call()
    for i in range(5):
        h = m.hidden(T)
        new, x = m.eight(h)
        for k in new:
            eight[k].copy_(new[k])
        hg.copy_(h)
        res.copy_(m.hidden(T))
        live = T - 4 * i
        n.fill_(live)
        for t in (yb, yl, r):
            t.fill_(2.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (yb, yl, sb, sl, gb, gl, r)]
        check((yl[:live], sl[:live], gl[:live]), m.expected(0, h[:live], x[:live]), K)
        assert (yl[live:] == 2).all() and (yb[live:] == 2).all() and (r[live:] == 2).all()
        with torch.cuda.stream(st):
            call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (yb, yl, sb, sl, gb, gl, r))), i


def test_handles_on_two_streams_at_once():
    """Two handles that share weights, on two streams, each with its own workspace."""
    N, K, d, F, T = 64, 6, 512, 256, 40
    m = Model("bf16", 1, N, K, d, F, T, "two streams")
    streams = [torch.cuda.Stream() for _ in range(2)]
    handles = [m.layers(stream=s) for s in streams]
    hs = [m.hidden(T) for _ in range(2)]
    gs = [h.cuda() for h in hs]
    want = [m.expected(0, h, h) for h in hs]
    outs = [outputs(T, K, d) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                handles[i].cmoe_moe_layer(0, gs[i], outs[i][0], selected=outs[i][1], gates=outs[i][2])
    torch.cuda.synchronize()
    for i in range(2):
        check(outs[i], want[i], K)


def test_a_handle_on_another_stream_than_its_tensors():
    """Work of the current stream, waited for by the handle's stream, and back."""
    N, K, d, F, T = 32, 4, 256, 128, 10
    m = Model("bf16", 1, N, K, d, F, T, "other stream")
    st = torch.cuda.Stream()
    layers = m.layers(stream=st)
    for i in range(5):
        h = m.hidden(T)
        y, sel, gates = outputs(T, K, d)
        hg = h.cuda() + 0  # on the current stream
        st.wait_stream(torch.cuda.current_stream())
        layers.cmoe_moe_layer(0, hg, y, selected=sel, gates=gates)
        torch.cuda.current_stream().wait_stream(st)
        check((y, sel, gates), m.expected(0, h, h), K)


def test_concurrent_host_threads_with_a_handle_each():
    import threading
    N, K, d, F, T = 16, 3, 128, 64, 9
    m = Model("f32", 1, N, K, d, F, T, "threads")
    hs = [m.hidden(T) for _ in range(4)]
    want = [m.expected(0, h, h) for h in hs]
    got, streams = [None] * 4, [torch.cuda.Stream() for _ in range(4)]
    handles, gs = [m.layers(stream=s) for s in streams], [h.cuda() for h in hs]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(streams[i]):
            out = outputs(T, K, d)
            for _ in range(10):
                handles[i].cmoe_moe_layer(0, gs[i], out[0], selected=out[1], gates=out[2])
        got[i] = out
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(4):
        check(got[i], want[i], K)


@pytest.mark.parametrize("kind", KINDS)
def test_repeats_are_bit_identical(kind):
    N, K, d, F, T = 64, 6, 512, 256, 40
    m = Model(kind, 1, N, K, d, F, T, f"repeat {kind}")
    layers = m.layers()
    h = m.hidden(T)
    eight, _ = m.eight(h)
    hg, first = h.cuda(), None
    for _ in range(10):
        y, sel, gates = outputs(T, K, d)
        layers.cmoe_moe_layer(0, hg, y, selected=sel, gates=gates, **eight)
        if first is None:
            first = y
        assert torch.equal(first, y)


def test_calls_that_are_refused():
    from paper_2609_04895_amd import cmoe as B
    N, K, d, F, T = 8, 2, 128, 64, 4
    m = Model("w8a8", 1, N, K, d, F, T, "refused")
    layers = m.layers()
    h = m.hidden(T)
    eight, _ = m.eight(h)
    h, y = h.cuda(), torch.zeros((T, d), device="cuda")
    big, by = torch.zeros((T + 1, d), dtype=BF16, device="cuda"), torch.zeros((T + 1, d), device="cuda")
    for call in (lambda: layers.cmoe_moe_layer(1, h, y, **eight),
                 lambda: layers.cmoe_moe_layer(-1, h, y, **eight),
                 lambda: layers.cmoe_moe_layer(0, h, y),                                   # 8-bit input missing
                 lambda: layers.cmoe_moe_layer(0, big, by, **eight),
                 lambda: layers.cmoe_moe_layer(0, h, y[:2], **eight),
                 lambda: layers.cmoe_moe_layer(0, h.float(), y, **eight),
                 lambda: layers.cmoe_moe_layer(0, h, y.to(BF16), **eight),
                 lambda: layers.cmoe_moe_layer(0, h, y, n_tokens=torch.tensor([T]), **eight),
                 lambda: layers.cmoe_moe_layer(0, h.cpu(), y, **eight),
                 lambda: layers.cmoe_moe_block(1, h, None, y),
                 lambda: layers.cmoe_moe_block(0, h, None, y, residual_out=h[:, :64])):
        with pytest.raises(B.CmoeError) as err:
            call()
        assert err.value.status == B.CMOE_ERR_INVALID_ARG
    # rows that 16-byte accesses cannot take
    odd = torch.zeros((T, d + 4), dtype=BF16, device="cuda")[:, 4:]
    with pytest.raises(B.CmoeError) as err:
        layers.cmoe_moe_layer(0, odd, y, **eight)
    assert err.value.status == B.CMOE_ERR_UNSUPPORTED
    q = torch.zeros((T, d + 8), dtype=torch.uint8, device="cuda")[:, 8:]
    with pytest.raises(B.CmoeError) as err:
        layers.cmoe_moe_layer(0, h, y, h8=q, h8_scale=eight["h8_scale"])
    assert err.value.status == B.CMOE_ERR_UNSUPPORTED
    layers.cmoe_moe_layer(0, h[:0], y[:0], h8=eight["h8"][:0], h8_scale=eight["h8_scale"][:0])  # nothing to do
    plain = Model("bf16", 1, N, K, d, F, T, "refused too").layers()
    with pytest.raises(B.CmoeError):
        plain.cmoe_moe_layer(0, h, y, **eight)
    # weights in host memory
    host = Model("bf16", 1, N, K, d, F, T, "host")
    host.gpu["experts"] = host.gpu["experts"].cpu()
    with pytest.raises(B.CmoeError):
        host.layers()
    # a call goes on after a refusal
    layers.cmoe_moe_layer(0, h, y, **eight)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all()

"""Refusals of the operators without an expert cache: sizes, types, strides,
alignment and pointers that the header rules out are errors before anything
reaches the GPU (no GPU needed here)."""
import ctypes

import pytest

from paper_2609_04895_amd import cmoe as B

P = 1 << 20  # an aligned address that nothing reads


def moe_cfg(**kw):
    base = dict(L=2, N=16, K=2, d=256, F=128, T=8, dtype=B.CMOE_BF16, weights=0, activations=0)
    base.update(kw)
    return B.make_moe_config(**base)


def error():
    return B.lib().cmoe_last_error().decode()


@pytest.mark.parametrize("kw,status", [
    (dict(L=0), B.CMOE_ERR_INVALID_ARG),
    (dict(N=0), B.CMOE_ERR_INVALID_ARG),
    (dict(K=0), B.CMOE_ERR_INVALID_ARG),
    (dict(T=0), B.CMOE_ERR_INVALID_ARG),
    (dict(d=-64), B.CMOE_ERR_INVALID_ARG),
    (dict(K=17), B.CMOE_ERR_INVALID_ARG),
    (dict(dtype=2), B.CMOE_ERR_INVALID_ARG),
    (dict(weights=2), B.CMOE_ERR_INVALID_ARG),
    (dict(activations=-1), B.CMOE_ERR_INVALID_ARG),
    (dict(T=65), B.CMOE_ERR_UNSUPPORTED),
    (dict(N=257), B.CMOE_ERR_UNSUPPORTED),
    (dict(N=128, K=65), B.CMOE_ERR_UNSUPPORTED),
    (dict(d=96), B.CMOE_ERR_UNSUPPORTED),
    (dict(F=32), B.CMOE_ERR_UNSUPPORTED),
    (dict(d=65600), B.CMOE_ERR_UNSUPPORTED),
    (dict(weights=1, dtype=B.CMOE_F32), B.CMOE_ERR_UNSUPPORTED),
    (dict(activations=1), B.CMOE_ERR_UNSUPPORTED),
])
def test_moe_query_refuses(kw, status):
    with pytest.raises(B.CmoeError) as err:
        B.cmoe_moe_query(moe_cfg(**kw))
    assert err.value.status == status and error()


def test_moe_query_sizes():
    n = B.cmoe_moe_query(moe_cfg())
    # logits, selections, gates, the norm's output, three bf16 planes of the intermediate, fp32 outputs
    assert n >= 8 * 16 * 4 + 8 * 2 * 8 + 8 * 256 * 2 + 8 * 2 * 128 * 6 + 8 * 2 * 256 * 4 and n % 256 == 0
    assert B.cmoe_moe_query(moe_cfg(weights=1, activations=1)) > n
    assert B.lib().cmoe_moe_query(ctypes.byref(moe_cfg()), None) == B.CMOE_ERR_INVALID_ARG
    B.cmoe_moe_query(moe_cfg(N=256, K=64, T=64, d=65536, F=65536))  # the largest: no overflow
    assert B.cmoe_moe_query(moe_cfg(N=256, K=64, T=64, d=65536, F=65536)) > 64 * 64 * 65536 * 10


@pytest.mark.parametrize("kw,workspace,text", [
    (dict(w_router=None), P, "required"),
    (dict(experts=None), P, "required"),
    (dict(), None, "workspace"),
    (dict(), P + 64, "workspace"),
    (dict(w_router=P + 8), P, "aligned"),
    (dict(experts=P + 4), P, "aligned"),
    (dict(logit_bias=P + 2), P, "aligned"),
])
def test_moe_init_refuses(kw, workspace, text):
    w = B.cmoe_moe_weights(**{**dict(w_router=P, logit_bias=None, experts=P, expert_scales=None), **kw})
    h = ctypes.c_void_p()
    cfg = moe_cfg()
    st = B.lib().cmoe_moe_init(ctypes.byref(cfg), ctypes.byref(w), workspace, None, ctypes.byref(h))
    assert st == B.CMOE_ERR_INVALID_ARG and not h.value and text in error()
    assert B.lib().cmoe_moe_init(ctypes.byref(cfg), None, P, None, ctypes.byref(h)) == B.CMOE_ERR_INVALID_ARG
    assert B.lib().cmoe_moe_init(ctypes.byref(cfg), ctypes.byref(w), P, None, None) == B.CMOE_ERR_INVALID_ARG


def test_moe_init_needs_scales_with_8_bit_weights():
    w = B.cmoe_moe_weights(P, None, P, None)
    h = ctypes.c_void_p()
    cfg = moe_cfg(weights=1)
    st = B.lib().cmoe_moe_init(ctypes.byref(cfg), ctypes.byref(w), P, None, ctypes.byref(h))
    assert st == B.CMOE_ERR_INVALID_ARG and "expert_scales" in error()
    w = B.cmoe_moe_weights(P, None, P, P + 2)  # scales are read four at a time
    st = B.lib().cmoe_moe_init(ctypes.byref(cfg), ctypes.byref(w), P, None, ctypes.byref(h))
    assert st == B.CMOE_ERR_INVALID_ARG and "aligned" in error()


def test_moe_calls_without_a_handle():
    L = B.lib()
    assert L.cmoe_moe_layer(None, ctypes.byref(B.cmoe_moe_call())) == B.CMOE_ERR_INVALID_ARG
    assert L.cmoe_moe_block(None, ctypes.byref(B.cmoe_norm()), ctypes.byref(B.cmoe_moe_call())) == B.CMOE_ERR_INVALID_ARG
    assert L.cmoe_moe_destroy(None) == B.CMOE_OK


def norm(**kw):
    base = dict(rows=4, d=64, dtype=B.CMOE_BF16, delta_dtype=B.CMOE_F32, eps=1e-6, residual=P, residual_stride=64, delta=2 * P,
                delta_stride=64, residual_out=3 * P, residual_out_stride=64, weight=4 * P, h=5 * P, h_stride=64, h8=6 * P,
                h8_stride=64, h8_scale=7 * P, h8_scale_stride=2, n_rows=None)
    base.update(kw)
    return B.cmoe_norm(**base)


@pytest.mark.parametrize("kw,status,text", [
    (dict(rows=-1), B.CMOE_ERR_INVALID_ARG, "rows"),
    (dict(d=0), B.CMOE_ERR_INVALID_ARG, "d >= 1"),
    (dict(dtype=2), B.CMOE_ERR_INVALID_ARG, "dtype"),
    (dict(delta_dtype=3), B.CMOE_ERR_INVALID_ARG, "delta"),
    (dict(eps=-1e-6), B.CMOE_ERR_INVALID_ARG, "eps"),
    (dict(eps=float("nan")), B.CMOE_ERR_INVALID_ARG, "eps"),
    (dict(eps=float("inf")), B.CMOE_ERR_INVALID_ARG, "eps"),
    (dict(rows=(1 << 21) + 1), B.CMOE_ERR_UNSUPPORTED, "rows"),
    (dict(d=(1 << 24) + 32), B.CMOE_ERR_UNSUPPORTED, "d >"),
    (dict(d=2**31 - 1, h8=None, h8_scale=None), B.CMOE_ERR_UNSUPPORTED, "d >"),
    (dict(residual=None), B.CMOE_ERR_INVALID_ARG, "residual"),
    (dict(h=None, h8=None, h8_scale=None, residual_out=None), B.CMOE_ERR_INVALID_ARG, "output"),
    (dict(h8_scale=None), B.CMOE_ERR_INVALID_ARG, "together"),
    (dict(h8=None), B.CMOE_ERR_INVALID_ARG, "together"),
    (dict(d=48), B.CMOE_ERR_INVALID_ARG, "multiple of 32"),
    (dict(residual_stride=63), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(delta_stride=0), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(residual_out_stride=1), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(h_stride=-64), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(h8_stride=32), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(h8_scale_stride=1), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(residual=P + 1), B.CMOE_ERR_INVALID_ARG, "aligned"),
    (dict(delta=P + 2), B.CMOE_ERR_INVALID_ARG, "aligned"),
    (dict(weight=P + 1), B.CMOE_ERR_INVALID_ARG, "aligned"),
    (dict(n_rows=P + 2), B.CMOE_ERR_INVALID_ARG, "aligned"),
    (dict(residual_out=P, residual_out_stride=128), B.CMOE_ERR_INVALID_ARG, "in place"),
    (dict(h=P), B.CMOE_ERR_INVALID_ARG, "place"),
    (dict(h=2 * P), B.CMOE_ERR_INVALID_ARG, "place"),
    (dict(h8=3 * P), B.CMOE_ERR_INVALID_ARG, "place"),
    (dict(residual_out=2 * P), B.CMOE_ERR_INVALID_ARG, "place"),
])
def test_add_norm_refuses(kw, status, text):
    assert B.lib().cmoe_add_norm(ctypes.byref(norm(**kw)), None) == status
    assert text in error()


def test_add_norm_refuses_null():
    assert B.lib().cmoe_add_norm(None, None) == B.CMOE_ERR_INVALID_ARG


@pytest.mark.parametrize("kw,status,text", [
    (dict(rows=-1), B.CMOE_ERR_INVALID_ARG, "rows"),
    (dict(cols=-32), B.CMOE_ERR_INVALID_ARG, "cols"),
    (dict(dtype=2), B.CMOE_ERR_INVALID_ARG, "dtype"),
    (dict(cols=40), B.CMOE_ERR_INVALID_ARG, "multiple of 32"),
    (dict(src=None), B.CMOE_ERR_INVALID_ARG, "required"),
    (dict(q=None), B.CMOE_ERR_INVALID_ARG, "required"),
    (dict(scale=None), B.CMOE_ERR_INVALID_ARG, "required"),
    (dict(src_stride=32), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(q_stride=32), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(scale_stride=1), B.CMOE_ERR_INVALID_ARG, "stride"),
    (dict(src=P + 2), B.CMOE_ERR_UNSUPPORTED, "aligned"),
    (dict(q=2 * P + 8), B.CMOE_ERR_UNSUPPORTED, "aligned"),
    (dict(src_stride=68), B.CMOE_ERR_UNSUPPORTED, "aligned"),
    (dict(q_stride=72), B.CMOE_ERR_UNSUPPORTED, "aligned"),
    (dict(q=P), B.CMOE_ERR_INVALID_ARG, "place"),
    (dict(rows=1 << 40), B.CMOE_ERR_UNSUPPORTED, "2^34"),
])
def test_quantize_refuses(kw, status, text):
    a = {**dict(src=P, dtype=B.CMOE_BF16, rows=4, cols=64, src_stride=64, q=2 * P, q_stride=64, scale=3 * P, scale_stride=2), **kw}
    st = B.lib().cmoe_quantize(a["src"], a["dtype"], a["rows"], a["cols"], a["src_stride"], a["q"], a["q_stride"], a["scale"],
                               a["scale_stride"], None)
    assert st == status and text in error()


def test_binding_refuses_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    r = torch.zeros((4, 64), dtype=torch.bfloat16)
    for kw in (dict(h=torch.zeros((4, 64))),                            # type
               dict(h=torch.zeros((3, 64), dtype=torch.bfloat16)),      # rows
               dict(h=torch.zeros((64, 4), dtype=torch.bfloat16).t()),  # columns apart
               dict(delta=torch.zeros((4, 64), dtype=torch.float16)),
               dict(weight=torch.zeros(32, dtype=torch.bfloat16)),
               dict(h8=torch.zeros((4, 64), dtype=torch.int8)),
               dict(n_rows=torch.zeros(1, dtype=torch.int64)),
               dict(residual_out=torch.zeros_like(r))):                 # host memory
        with pytest.raises(B.CmoeError) as err:
            B.cmoe_add_norm(r, **kw)
        assert err.value.status == B.CMOE_ERR_INVALID_ARG
    q, s = torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    for args in ((r.half(), q, s), (r, q[:3], s), (r, q, s[:, :1]), (r, q.float(), s), (r, q, s)):
        with pytest.raises(B.CmoeError):
            B.cmoe_quantize(*args)


def test_packed_arguments_have_the_structures_layout():
    """The binding packs calls as bytes: field for field what the structures hold."""
    v = list(range(1, 6)) + [(1 << 40) + i for i in range(14)]
    v[4] = 0.5
    n = B.cmoe_norm.from_buffer_copy(B._NORM.pack(*v))
    assert ctypes.sizeof(B.cmoe_norm) == B._NORM.size
    assert [getattr(n, f) for f, _ in B.cmoe_norm._fields_] == v
    v = [3, 4] + [(1 << 40) + i for i in range(11)]
    c = B.cmoe_moe_call.from_buffer_copy(B._CALL.pack(*v))
    assert ctypes.sizeof(B.cmoe_moe_call) == B._CALL.size
    assert [getattr(c, f) for f, _ in B.cmoe_moe_call._fields_] == v

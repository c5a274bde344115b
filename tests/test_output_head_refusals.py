"""Argument checks of the output head's calls: the documented codes, before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.skipif(not os.path.exists(mm.LIB_PATH), reason="libmobile_moe.so not built")
BADARG, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6
P = 1 << 20                                     # an address that passes the alignment checks and is never read


def _int8(**kw):
    c = mm.moe_int8_config()
    c.T, c.N, c.K, c.x_dtype, c.out_dtype = 4, 32, 64, mm.MOE_BF16, mm.MOE_FP32
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _codes(c, x=P, x_scale=P, w=P, w_scale=P, bias=None, out=P):
    return mm.load_library().moe_matmul_int8(ctypes.byref(c) if c is not None else None, x, x_scale, w, w_scale, bias, out, None)


def _linear(c, x=P, w=P, w_scale=P, bias=None, out=P, ws=None, ws_bytes=0):
    return mm.load_library().moe_linear_int8(ctypes.byref(c) if c is not None else None, x, w, w_scale, bias, out, ws, ws_bytes, None)


@pytest.mark.parametrize("change, code", [
    (dict(T=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=-5), SHAPE), (dict(K=131072), UNSUPPORTED),
    (dict(out_dtype=2), BADARG), (dict(out_dtype=-1), BADARG), (dict(reserved=1), BADARG), (dict(ldx=-16), BADARG),
    (dict(ldw=48), SHAPE), (dict(ldw=72), UNSUPPORTED), (dict(K=63), UNSUPPORTED), (dict(ldo=31), SHAPE), (dict(ldw=1 << 22), UNSUPPORTED),
    (dict(ldo=1 << 22), UNSUPPORTED), (dict(ldx=48), SHAPE), (dict(ldo=-1), BADARG),
])
def test_product_configs(change, code):
    assert _codes(_int8(**change)) == code and mm.moe_last_error()
    assert _linear(_int8(**change)) == code
    assert mm.load_library().moe_linear_int8_workspace_bytes(ctypes.byref(_int8(**change))) == 0


def test_product_configs_of_one_call_only():
    assert _codes(_int8(ldx=72)) == UNSUPPORTED                       # rows of codes start on 16 bytes, float rows anywhere
    assert _linear(_int8(ldx=71)) == WORKSPACE
    assert _linear(_int8(x_dtype=2)) == BADARG
    assert _codes(_int8(x_dtype=2), x=None) == BADARG and "x is NULL" in mm.moe_last_error()
    assert _codes(None) == BADARG and _linear(None) == BADARG
    assert _codes(_int8(T=0), x=None, out=None) == 0 and _linear(_int8(T=0), x=None) == 0


@pytest.mark.parametrize("arg, value", [("x", None), ("x", P + 8), ("x_scale", None), ("x_scale", P + 2), ("w", None), ("w", P + 4),
                                        ("w_scale", None), ("bias", P + 1), ("out", None), ("out", P + 2)])
def test_product_pointers(arg, value):
    assert _codes(_int8(), **{arg: value}) == BADARG
    assert arg in mm.moe_last_error()


def test_linear_pointers_and_workspace():
    c = _int8(K=60, ldw=64)
    need = mm.moe_linear_int8_workspace_bytes(c)
    assert need == 256 + 256                                          # 4 rows of 64 codes, 4 scales
    assert _linear(c, x=P + 1, ws=P, ws_bytes=need) == BADARG
    assert _linear(_int8(x_dtype=mm.MOE_FP32), x=P + 2, ws=P, ws_bytes=need) == BADARG
    for ws, n in ((None, need), (P + 16, need), (P, need - 1)):
        assert _linear(c, ws=ws, ws_bytes=n) == WORKSPACE


def test_quantize_rows():
    def q(x=P, dtype=mm.MOE_BF16, rows=4, K=60, ldx=60, codes=P, ldq=64, scale=P):
        return mm.load_library().moe_quantize_rows(x, dtype, rows, K, ldx, codes, ldq, scale, None)
    for kw, code in ((dict(dtype=2), BADARG), (dict(rows=-1), SHAPE), (dict(K=0), SHAPE), (dict(K=131072, ldx=0), UNSUPPORTED), (dict(ldx=59), SHAPE),
                     (dict(ldq=48), SHAPE), (dict(ldq=60), UNSUPPORTED), (dict(ldq=0), UNSUPPORTED), (dict(ldx=1 << 22), UNSUPPORTED),
                     (dict(ldx=-1), BADARG), (dict(x=None), BADARG), (dict(x=P + 1), BADARG), (dict(dtype=mm.MOE_FP32, x=P + 2), BADARG),
                     (dict(codes=P + 8), BADARG), (dict(scale=None), BADARG)):
        assert q(**kw) == code, (kw, mm.moe_last_error())
    assert q(rows=0, x=None, codes=None, scale=None) == 0


def _lp(**kw):
    c = mm.moe_logprobs_config()
    c.T, c.V, c.dtype, c.n_given, c.n_top = 4, 1000, mm.MOE_FP32, 1, 5
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _logprobs(c, logits=P, tokens=P, token_logp=P, entropy=P, conf=P, top_idx=P, top_logp=P, ws=P, ws_bytes=1 << 30):
    return mm.load_library().moe_token_logprobs(ctypes.byref(c) if c is not None else None, logits, tokens, token_logp, entropy, conf,
                                                top_idx, top_logp, ws, ws_bytes, None)


@pytest.mark.parametrize("change, code", [
    (dict(T=-1), SHAPE), (dict(V=0), SHAPE), (dict(dtype=2), BADARG), (dict(n_given=-1), BADARG), (dict(n_top=-1), BADARG), (dict(ld=-1), BADARG),
    (dict(reserved=3), BADARG), (dict(V=4), SHAPE), (dict(n_top=33), UNSUPPORTED), (dict(n_given=65), UNSUPPORTED), (dict(ld=999), SHAPE),
    (dict(ld=1 << 22), UNSUPPORTED),
])
def test_logprob_configs(change, code):
    assert _logprobs(_lp(**change)) == code and mm.moe_last_error()
    assert mm.load_library().moe_token_logprobs_workspace_bytes(ctypes.byref(_lp(**change))) == 0


@pytest.mark.parametrize("arg, value", [("logits", None), ("logits", P + 2), ("tokens", None), ("token_logp", None), ("entropy", P + 1),
                                        ("conf", P + 2), ("top_idx", None), ("top_logp", P + 1)])
def test_logprob_pointers(arg, value):
    assert _logprobs(_lp(), **{arg: value}) == BADARG
    assert arg in mm.moe_last_error()


def test_logprob_workspace_and_empty_calls():
    assert _logprobs(None) == BADARG
    assert _logprobs(_lp(T=0), logits=None, tokens=None) == 0
    c = _lp(T=1, V=131072, n_top=32)
    need = mm.moe_token_logprobs_workspace_bytes(c)
    if need:
        for ws, n in ((None, need), (P + 128, need), (P, need - 1)):
            assert _logprobs(c, ws=ws, ws_bytes=n) == WORKSPACE

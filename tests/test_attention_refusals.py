"""Argument checks of the attention step's calls: the documented codes, before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2510_12357_amd import binding as mm

pytestmark = pytest.mark.skipif(not os.path.exists(mm.LIB_PATH), reason="libmobile_moe.so not built")
BADARG, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -6
P = 1 << 20                                     # addresses that pass the alignment checks and are never read
P2 = 1 << 30


def _made(c, kw):
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _rope(**kw):
    c = mm.moe_rope_config()
    c.T, c.heads, c.D, c.rotary_dim, c.mscale = 4, 3, 64, 32, 1.0
    return _made(c, kw)


def _cache(**kw):
    c = mm.moe_kv_cache()
    c.n_pages, c.page_size, c.heads, c.D, c.k, c.v = 10, 16, 2, 64, P, P2
    return _made(c, kw)


def _append(**kw):
    c = mm.moe_append_config()
    c.T, c.heads, c.rotary_dim, c.n_seqs, c.table_len, c.mscale = 4, 6, 64, 4, 3, 1.0
    return _made(c, kw)


def _attention(**kw):
    c = mm.moe_attention_config()
    c.B, c.heads, c.max_len, c.table_len, c.scale = 2, 6, 48, 3, 0.125
    return _made(c, kw)


def _ref(c):
    return None if c is None else ctypes.byref(c)


def rope(c, x=P, pos=P, freq=P, out=P2):
    return mm.load_library().moe_rope(_ref(c), x, pos, freq, out, None)


def append(c, cache, q=P, k=P, v=P, pos=P, seq=None, table=P, freq=P, q_out=P2):
    return mm.load_library().moe_kv_append(_ref(c), _ref(cache), q, k, v, pos, seq, table, freq, q_out, None)


def attend(c, cache, q=P, table=P, lengths=P, out=P2, lse=None, ws=None, ws_bytes=0, counters=None):
    return mm.load_library().moe_paged_attention(_ref(c), _ref(cache), q, table, lengths, out, lse, ws, ws_bytes, counters, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change, code", [
    (dict(T=-1), SHAPE), (dict(heads=0), SHAPE), (dict(D=0), SHAPE), (dict(D=63), UNSUPPORTED), (dict(D=258), UNSUPPORTED), (dict(dtype=4), BADARG),
    (dict(rotary_dim=-2), SHAPE), (dict(rotary_dim=66), SHAPE), (dict(rotary_dim=3), SHAPE), (dict(layout=2), BADARG), (dict(inverse=2), BADARG),
    (dict(mscale=NAN), BADARG), (dict(mscale=INF), BADARG), (dict(x_token=-1), BADARG), (dict(x_head=63), SHAPE), (dict(x_token=191), SHAPE),
    (dict(out_head=32), SHAPE), (dict(out_token=64, out_head=64), SHAPE), (dict(out_token=1 << 50), UNSUPPORTED), (dict(out_head=1 << 50), UNSUPPORTED),
])
def test_rope_configs(change, code):
    assert rope(_rope(**change)) == code and mm.moe_last_error()


@pytest.mark.parametrize("arg, value", [("x", None), ("x", P + 1), ("pos", None), ("pos", P + 2), ("freq", None), ("freq", P + 4), ("out", None), ("out", P + 1)])
def test_rope_pointers(arg, value):
    assert rope(_rope(), **{arg: value}) == BADARG and arg in mm.moe_last_error()


def test_rope_empty_and_in_place():
    assert rope(None) == BADARG
    assert rope(_rope(T=0), x=None, pos=None, freq=None, out=None) == 0
    assert rope(_rope(dtype=mm.MOE_FP32), x=P + 2) == BADARG
    assert rope(_rope(x_head=128), x=P, out=P) == BADARG and "in place" in mm.moe_last_error()


CACHES = [
    (dict(n_pages=0), SHAPE), (dict(heads=0), SHAPE), (dict(D=0), SHAPE), (dict(page_size=0), UNSUPPORTED), (dict(page_size=2), UNSUPPORTED),
    (dict(page_size=24), UNSUPPORTED), (dict(page_size=1 << 21), UNSUPPORTED), (dict(D=72), UNSUPPORTED), (dict(D=272), UNSUPPORTED), (dict(dtype=2), BADARG),
    (dict(reserved=1), BADARG), (dict(row=-64), BADARG), (dict(row=68), UNSUPPORTED), (dict(row=48), SHAPE), (dict(head=64), SHAPE), (dict(page=1024), SHAPE),
    (dict(head=1028), UNSUPPORTED), (dict(page=2052), UNSUPPORTED),
    (dict(page=1 << 50), UNSUPPORTED), (dict(row=1 << 50), UNSUPPORTED), (dict(dtype=mm.MOE_E4M3, row=72), UNSUPPORTED),
    (dict(k=None), BADARG), (dict(v=P2 + 8), BADARG), (dict(v=P), BADARG), (dict(dtype=mm.MOE_E4M3), BADARG),
    (dict(dtype=mm.MOE_E4M3, k_scale=P, v_scale=P + 4), BADARG), (dict(dtype=mm.MOE_E4M3, k_scale=P, v_scale=P), BADARG),
]


@pytest.mark.parametrize("change, code", CACHES)
def test_caches(change, code):
    assert append(_append(), _cache(**change)) == code and mm.moe_last_error()
    assert attend(_attention(), _cache(**change)) == code
    if "v" not in change and "k" not in change and "k_scale" not in change and change != dict(dtype=mm.MOE_E4M3):
        assert mm.load_library().moe_paged_attention_workspace_bytes(_ref(_attention()), _ref(_cache(**change))) == 0


@pytest.mark.parametrize("change, code", [
    (dict(T=-1), SHAPE), (dict(heads=-1), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(table_len=0), SHAPE), (dict(table_ld=2), SHAPE), (dict(table_ld=-3), BADARG),
    (dict(table_ld=1 << 50), UNSUPPORTED), (dict(dtype=4), BADARG), (dict(rotary_dim=66), SHAPE), (dict(layout=-1), BADARG), (dict(mscale=NAN), BADARG),
    (dict(k_head=60), SHAPE), (dict(v_token=100), SHAPE), (dict(q_head=1), SHAPE), (dict(out_token=5), SHAPE), (dict(q_token=-1), BADARG),
])
def test_append_configs(change, code):
    assert append(_append(**change), _cache()) == code and mm.moe_last_error()


@pytest.mark.parametrize("arg, value", [("q", None), ("q", P + 1), ("k", None), ("k", P + 1), ("v", None), ("pos", None), ("pos", P + 2), ("seq", P + 2),
                                        ("table", None), ("table", P + 1), ("freq", None), ("freq", P + 4), ("q_out", None), ("q_out", P2 + 1)])
def test_append_pointers(arg, value):
    assert append(_append(), _cache(), **{arg: value}) == BADARG and arg in mm.moe_last_error()


def test_append_empty_calls():
    assert append(None, _cache()) == BADARG and append(_append(), None) == BADARG
    assert append(_append(T=0), _cache(), q=None, k=None, table=None) == 0
    assert append(_append(q_head=128), _cache(), q=P, q_out=P) == BADARG


@pytest.mark.parametrize("change, code", [
    (dict(B=-1), SHAPE), (dict(heads=0), SHAPE), (dict(heads=5), SHAPE), (dict(dtype=4), BADARG), (dict(max_len=-1), BADARG), (dict(window=-1), BADARG),
    (dict(table_len=0), SHAPE), (dict(table_ld=1), SHAPE), (dict(max_len=2 ** 31 - 100), UNSUPPORTED), (dict(scale=NAN), BADARG), (dict(scale=-INF), BADARG),
    (dict(softcap=-1.0), BADARG), (dict(softcap=INF), BADARG), (dict(softcap=1e-40), UNSUPPORTED), (dict(softcap=2e38), UNSUPPORTED), (dict(scale=-1e38), UNSUPPORTED), (dict(q_head=63), SHAPE), (dict(out_token=-1), BADARG),
    (dict(B=1 << 30, heads=64), UNSUPPORTED),
])
def test_attention_configs(change, code):
    assert attend(_attention(**change), _cache()) == code and mm.moe_last_error()
    assert mm.load_library().moe_paged_attention_workspace_bytes(_ref(_attention(**change)), _ref(_cache())) == 0


@pytest.mark.parametrize("arg, value", [("q", None), ("q", P + 1), ("table", None), ("table", P + 2), ("lengths", None), ("lengths", P + 1), ("out", None),
                                        ("out", P2 + 1), ("lse", P + 2), ("counters", P + 2)])
def test_attention_pointers(arg, value):
    assert attend(_attention(), _cache(), **{arg: value}) == BADARG and arg in mm.moe_last_error()


def test_attention_workspace_and_empty_calls():
    assert attend(None, _cache()) == BADARG and attend(_attention(), None) == BADARG
    assert attend(_attention(B=0), _cache(), q=None, table=None) == 0
    long = _attention(max_len=100000, table_len=100000)
    need = mm.moe_paged_attention_workspace_bytes(long, _cache())
    assert need > 0
    for ws, n in ((None, need), (P + 128, need), (P, need - 1)):
        assert attend(long, _cache(), ws=ws, ws_bytes=n) == WORKSPACE
    # the table's rows bound the lengths, and with them the workspace
    assert mm.moe_paged_attention_workspace_bytes(_attention(max_len=100000), _cache()) == 0


def test_more_heads_than_a_token_can_have():
    """Of a token's heads and channels there are less than 2^29; the largest numbers below pass (an empty call)."""
    few, many = (1 << 23) - 2, 1 << 23                        # heads of 64 channels
    assert rope(_rope(heads=many)) == UNSUPPORTED and "heads" in mm.moe_last_error()
    assert append(_append(heads=many), _cache()) == UNSUPPORTED and "heads" in mm.moe_last_error()
    assert attend(_attention(heads=many), _cache()) == UNSUPPORTED and "heads" in mm.moe_last_error()
    assert append(_append(heads=0), _cache(heads=many)) == UNSUPPORTED and attend(_attention(heads=many), _cache(heads=many)) == UNSUPPORTED
    assert rope(_rope(T=0, heads=few)) == 0 and append(_append(T=0, heads=few), _cache(heads=few)) == 0 and attend(_attention(B=0, heads=few), _cache(heads=few)) == 0
    for heads in (1 << 30, (1 << 31) - 2):
        assert rope(_rope(heads=heads)) == UNSUPPORTED and attend(_attention(heads=heads), _cache()) == UNSUPPORTED


def test_attention_in_place_with_other_strides():
    """A workgroup would store results over queries that another one has still to read.  What is let through here ends at the workspace, which is missing."""
    long = dict(max_len=100000, table_len=100000)
    for change in (dict(q_head=128), dict(out_head=128), dict(q_token=6 * 64 + 8), dict(out_token=1024), dict(q_token=64, q_head=128), dict(out_head=72, dtype=mm.MOE_FP32)):
        assert attend(_attention(**long, **change), _cache(), q=P, out=P) == BADARG and "in place" in mm.moe_last_error(), change
        assert attend(_attention(**long, **change), _cache(), q=P, out=P2) == WORKSPACE, change
    # the same strides in other words, and strides of what there is only one of
    for change, cache in ((dict(), _cache()), (dict(q_head=64, out_token=6 * 64), _cache()), (dict(B=1, q_token=4096), _cache()), (dict(heads=1, q_head=256, q_token=64, out_token=64), _cache(heads=1))):
        assert attend(_attention(**long, **change), cache, q=P, out=P) == WORKSPACE, change

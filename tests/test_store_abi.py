"""Host-side checks of the store's and the weights' calls: refusals before anything touches the GPU."""
import ctypes
import re

import pytest
import torch

from paper_2506_11498_b200 import build as lib_build
from paper_2506_11498_b200 import lrsa

GOOD = dict(batch=1, n_q_heads=4, n_kv_heads=2, seq_len=1000, head_dim=128, lag=128, top_k=32, n_sink=4)
AT = 1 << 20      # an address that is aligned; nothing reads it


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def shape(params, **kw):
    st = lrsa.lrsa_store_t(**{**dict(list_type=1, block=64, keep=1, reserved=0), **kw})
    a, b, c = ctypes.c_int32(-1), ctypes.c_int32(-1), ctypes.c_size_t(0)
    rc = lrsa.lib().lrsa_store_shape(params.ref(), ctypes.byref(st), ctypes.byref(a), ctypes.byref(b), ctypes.byref(c))
    return rc, a.value, b.value, c.value


def test_shape():
    p = lrsa.Params(**GOOD)
    assert shape(p)[:3] == (0, 6, 64)             # chunk of the last token: 995 // 128 = 7
    assert shape(p, block=16)[:3] == (0, 6, 32) and shape(p, block=128)[:3] == (0, 6, 128)
    assert shape(lrsa.Params(**{**GOOD, "seq_len": 260}))[1] == 0
    assert shape(lrsa.Params(**{**GOOD, "seq_len": 261}))[1] == 1
    assert shape(p)[3] >= 256 and shape(p, keep=0)[3] >= 256


@pytest.mark.parametrize("params,store,status", [
    ({}, {}, 0), ({}, {"list_type": 3}, 1), ({}, {"list_type": -1}, 1), ({}, {"keep": 2}, 1), ({}, {"block": 0}, 2), ({}, {"block": 48}, 2),
    ({}, {"block": 256}, 2), ({"n_dense_prev": 0}, {}, 2), ({"cu_seqlens": (0, 500, 1000)}, {}, 2), ({"head_dim": 96}, {}, 2),
    ({"top_k": 0}, {}, 1),
])
def test_store_parameters(params, store, status):
    assert shape(lrsa.Params(**{**GOOD, **params}), **store)[0] == status


FULL = dict(list_type=1, block=64, keep=1, reserved=0, k_list=AT, v_list=AT, k_scale=AT, v_scale=AT, k_recent=AT, v_recent=AT,
            weight=AT, idx=AT)


@pytest.mark.parametrize("change", [{"k_list": 0}, {"v_list": AT + 8}, {"k_scale": 0}, {"v_scale": AT + 2}, {"k_recent": 0},
                                    {"v_recent": AT + 8}, {"weight": 0}, {"weight": AT + 2}, {"idx": 0}, {"idx": AT + 1}])
def test_store_tensors(change):
    p, st = lrsa.Params(**GOOD), lrsa.lrsa_store_t(**{**FULL, **change})
    L, need = lrsa.lib(), shape(lrsa.Params(**GOOD))[3]
    assert L.lrsa_store_append(p.ref(), ctypes.byref(st), AT, AT, None, 0, 1, AT, need, None) == 1
    assert L.lrsa_store_decode(p.ref(), ctypes.byref(st), AT, 1, AT, None, AT, need, None) == 1
    assert L.lrsa_store_rows(p.ref(), ctypes.byref(st), 1, AT, AT, None) == 1


def test_store_calls():
    p, st = lrsa.Params(**GOOD), lrsa.lrsa_store_t(**FULL)
    L, need, s = lrsa.lib(), shape(lrsa.Params(**GOOD))[3], ctypes.byref(st)
    app = lambda k=AT, v=AT, w=None, prev=0, n=1, ws=AT, size=need: L.lrsa_store_append(p.ref(), s, k, v, w, prev, n, ws, size, None)
    assert app(k=None) == 1 and app(v=AT + 2) == 1 and app(w=AT + 1) == 1 and app(prev=-1) == 1 and app(n=0) == 1
    assert app(prev=1000) == 1 and app(prev=999, n=2) == 1 and app(ws=AT + 16) == 1 and app(ws=None) == 1 and app(size=need - 1) == 3
    assert app(prev=2 ** 31 - 1, n=2 ** 31 - 1) == 1
    # windows of the call's own tokens are cut by weight: their weights have to be given
    assert app(n=261) == 1 and app(prev=100, n=161) == 1
    lag = lrsa.lrsa_store_t(**{**FULL, "keep": 0})
    assert L.lrsa_store_append(p.ref(), ctypes.byref(lag), AT, AT, AT, 0, 1, AT, 1 << 30, None) == 1    # weights nobody keeps
    dec = lambda q=AT, n=1, o=AT, lse=None, ws=AT, size=need: L.lrsa_store_decode(p.ref(), s, q, n, o, lse, ws, size, None)
    assert dec(q=None) == 1 and dec(q=AT + 8) == 1 and dec(n=0) == 1 and dec(n=1001) == 1 and dec(o=None) == 1 and dec(o=AT + 4) == 1
    assert dec(lse=AT + 2) == 1 and dec(ws=None) == 1 and dec(ws=AT + 4) == 1 and dec(size=need - 1) == 3
    assert L.lrsa_store_rows(p.ref(), s, 7, AT, AT, None) == 1 and L.lrsa_store_rows(p.ref(), s, -1, AT, AT, None) == 1
    assert L.lrsa_store_rows(p.ref(), s, 1, None, AT, None) == 1 and L.lrsa_store_rows(p.ref(), s, 1, AT, AT + 4, None) == 1
    assert L.lrsa_store_rows(p.ref(), s, 0, None, None, None) == 0


def test_weights_and_select_calls():
    p, L = lrsa.Params(**GOOD), lrsa.lib()
    call = lambda q=AT, k=AT, e=AT, w=AT, ws=AT, size=256: L.lrsa_attn_weights(p.ref(), q, k, e, w, ws, size, None)
    assert call(q=None) == 1 and call(k=None) == 1 and call(e=None) == 1 and call(w=None) == 1 and call(ws=None) == 1
    assert call(q=AT + 8) == 1 and call(k=AT + 8) == 1 and call(e=AT + 2) == 1 and call(w=AT + 2) == 1 and call(ws=AT + 128) == 1
    assert call(size=255) == 3
    assert L.lrsa_weight_select(p.ref(), None, AT, None) == 1 and L.lrsa_weight_select(p.ref(), AT, None, None) == 1
    assert L.lrsa_weight_select(p.ref(), AT + 2, AT, None) == 1 and L.lrsa_weight_select(p.ref(), AT, AT + 2, None) == 1
    short = lrsa.Params(**{**GOOD, "seq_len": 100})          # no scored window: nothing to select, nothing launched
    assert L.lrsa_weight_select(short.ref(), AT, None, None) == 0 and L.lrsa_last_launch_count() == 0


def test_binding_refuses():
    p = lrsa.Params(**GOOD)
    for kw in (dict(dtype=torch.float16), dict(keep="heavy")):
        with pytest.raises(lrsa.LrsaError) as e:
            lrsa.KVStore(p, device="cpu", **kw)
        assert e.value.status == 1
    with pytest.raises(lrsa.LrsaError) as e:
        lrsa.KVStore(p, block=24, device="cpu")
    assert e.value.status == 2
    store = lrsa.KVStore(p, dtype=torch.int8, block=32, device="cpu")
    assert store.k_list.shape == (1, 2, 6 * 32, 128) and store.k_scale.shape == (1, 2, 6) and store.weight.shape == (1, 2, 256)
    k = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(lrsa.LrsaError) as e:      # the library has no CPU path
        store.append(k, k)
    assert e.value.status == 1 and store.n_tokens == 0
    bf = lrsa.KVStore(p, dtype=torch.bfloat16, keep="lag", device="cpu")
    assert bf.k_scale is None and bf.weight is None and bf.k_list.dtype == torch.bfloat16


def test_binding_mirrors_the_header():
    """The struct of the binding has the header's fields, in its order."""
    import os
    text = open(os.path.join(os.path.dirname(lib_build.__file__), "..", "include", "lrsa.h")).read()
    body = re.search(r"typedef struct lrsa_store \{(.*?)\} lrsa_store_t;", text, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert re.findall(r"(\w+);", body) == [n for n, _ in lrsa.lrsa_store_t._fields_]

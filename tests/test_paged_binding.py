"""The binding of the rotation and the paged cache on the CPU, with recorded calls: what the library is given after the caller has replaced
something, and what is told and held meanwhile."""
import gc
import pickle

import pytest
import torch

from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref
from tests.test_paged_abi import INVALID, P, STREAM, _built, bf, calls, good, i32  # noqa: F401  (fixtures)

ROPE_AT = {"paged_append": 19, "paged_attend": 22, "rotate": 5}     # where the five values of a rope begin


def every_call(cache, rope):
    a, b = good(cache)
    return [lambda: cache.append(**{**a, "rope": rope}, stream=STREAM), lambda: cache.attend(**{**b, "rope": rope}, stream=STREAM),
            lambda: lrsa.lrsa_rotate(P, bf(1, 8, 4000, 128), None, rope, positions=i32(4000), stream=STREAM)]


def given(calls):
    """The rope of the last three calls."""
    return [args[ROPE_AT[name]:ROPE_AT[name] + 5] for name, args in calls[-3:]]


def test_tables_of_a_rope_that_were_replaced(calls):
    """Longer tables, other angles of the same shape, the other pairing: the next call takes them."""
    cache, rope = lrsa.PagedCache(P, 5, device="cpu"), lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
    for rows in (64, 4096, 64):
        rope.cos, rope.sin = torch.ones(rows, 64), torch.ones(rows, 64)
        rope.interleaved = rows == 4096
        for call in every_call(cache, rope):
            call()
        assert given(calls) == [(rope.cos.data_ptr(), rope.sin.data_ptr(), rows, 128, int(rows == 4096))] * 3


def test_tables_of_a_rope_that_were_resized(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    for rows in (8, 5000):      # in their memory, and beyond it
        rope = lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
        every_call(cache, rope)[0]()
        rope.cos.resize_(rows, 64)
        rope.sin.resize_(rows, 64)
        for call in every_call(cache, rope):
            call()
        assert given(calls) == [(rope.cos.data_ptr(), rope.sin.data_ptr(), rows, 128, 0)] * 3


@pytest.mark.parametrize("used", [False, True], ids=["fresh", "used"])
@pytest.mark.parametrize("name", ["cos", "sin"])
def test_tables_of_a_rope_that_cannot_be_used(calls, name, used):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    other = {"cos": "sin", "sin": "cos"}[name]
    for bad in (torch.zeros(64, 64).double(), torch.zeros(65, 64), torch.zeros(64, 72), torch.zeros(64, 128)[:, ::2], torch.zeros(64 * 64),
                torch.zeros(64, 64, device="meta"), torch.zeros(64 * 64 + 1)[1:].view(64, 64), None, 3.0):
        rope = lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
        if used:
            every_call(cache, rope)[0]()
        n = len(calls)
        setattr(rope, name, bad)
        for call in every_call(cache, rope):
            with pytest.raises(lrsa.LrsaError) as e:
                call()
            assert e.value.status == INVALID
        assert len(calls) == n
        setattr(rope, name, torch.zeros_like(getattr(rope, other)))
        every_call(cache, rope)[0]()
        assert len(calls) == n + 1


def test_tables_of_a_rope_that_lost_their_memory(calls):
    cache, rope = lrsa.PagedCache(P, 5, device="cpu"), lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
    every_call(cache, rope)[0]()
    n = len(calls)
    rope.sin.untyped_storage().resize_(0)
    for call in every_call(cache, rope):
        with pytest.raises(lrsa.LrsaError):
            call()
    assert len(calls) == n


def test_status_is_asked_of_every_workspace(calls, monkeypatch):
    """A captured call goes on in the workspace that it was captured with, when the cache has a larger one."""
    cache = lrsa.PagedCache(P, 5, device="cpu")
    asked, told = [], {}

    class Library:
        def __getattr__(self, name):
            return getattr(lrsa._lib, name)

        def lrsa_paged_status(self, at, stream):
            asked.append(at)
            return told.pop(at, 0)

    library = Library()
    spaces = [cache.ws]
    for new in (20, 60, 130):
        cache.append(**good(cache, 1000 * new)[0], stream=STREAM)
        spaces.append(cache.ws)
    assert len({x.data_ptr() for x in spaces}) == 4 and all((x[:256] == 0).all() for x in spaces)
    monkeypatch.setattr(lrsa, "lib", lambda: library)
    for code in (1, 5):
        for space in spaces:
            told[space.data_ptr()] = code
            assert cache.status(STREAM) == code and cache.status(STREAM) == 0
    told.update({spaces[0].data_ptr(): 5, spaces[3].data_ptr(): 1})
    assert cache.status(STREAM) == 5
    assert set(asked) == {x.data_ptr() for x in spaces}


def test_status_without_a_workspace():
    assert lrsa.lib().lrsa_paged_status(None, None) == lrsa.lib().lrsa_paged_status(0x7f0000000080, None) == INVALID


def test_outputs_that_lie_over_one_another_or_over_the_inputs():
    """By the library, which knows the strides of all of them: 8/2 heads, d = 128, 16 tokens."""
    from tests.test_paged_abi import AT, attend, rows
    far = dict(q=rows(AT), k=rows(AT + (1 << 20)), v=rows(AT + (2 << 20)), ws_bytes=1 << 30)
    o = AT + (3 << 20)
    own = [(128, 128), (0, 1024), (128, 0), (64, 1024), (128, 64), (128, 1016), (136, 136), (2040, 128), (1024, 1024), (256, 384), (-128, 128),
           (128, -1016), (384, 256)]
    for head, token in own:
        assert attend(o=rows(o, head, token), **far) == INVALID, (head, token)
    for at in (AT, AT + 16, AT + 2 * (15 * 1024 + 7 * 128), AT - 2 * (15 * 1024 + 8 * 128 - 8)):      # q itself, parts of it, its last row, its first
        assert attend(o=rows(at), **far) == INVALID
        assert attend(o=rows(at, 16 * 128, 128), **far) == INVALID       # head by head
    for name in "kv":
        for at in (far[name].data, far[name].data + 2 * (15 * 1024 + 128), far[name].data - 2 * (15 * 1024 + 7 * 128)):
            assert attend(o=rows(at), **far) == INVALID
    # beside them in one buffer, a few elements too near
    fused = dict(q=rows(AT, 128, 2568), k=rows(AT + 2 * 1024, 128, 2568), v=rows(AT + 2 * 1280, 128, 2568), ws_bytes=1 << 30)
    assert attend(o=rows(AT + 2 * 1528, 128, 2568), **fused) == attend(o=rows(AT + 2 * 1552, 128, 2568), **fused) == INVALID
    assert attend(o=rows(AT + 2 * 1536, 128, 2560), **fused) == INVALID   # (the next pitch: only a later token's comes near)


def holders(storage):
    """Tensors anywhere in the process that hold a storage."""
    return sum(type(x) is torch.Tensor and x.untyped_storage()._cdata == storage for x in gc.get_objects())


@pytest.mark.parametrize("name", ["k_pages", "v_pages"])
def test_pages_that_were_replaced_are_let_go(calls, name):
    """A pool makes room for a larger one: nothing of the cache holds on to what was given up for it."""
    cache = lrsa.PagedCache(P, 5, device="cpu")
    cache.append(**good(cache)[0], stream=STREAM)
    storage = getattr(cache, name).untyped_storage()._cdata
    assert holders(storage) > 1
    setattr(cache, name, None)
    assert holders(storage) == 0


def test_tables_of_a_rope_that_were_replaced_are_let_go(calls):
    cache, rope = lrsa.PagedCache(P, 5, device="cpu"), lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
    every_call(cache, rope)[0]()
    storage = rope.cos.untyped_storage()._cdata
    rope.cos = None
    assert holders(storage) == 0


def test_the_layers_of_a_model_share_a_workspace(calls):
    """Their calls run one after the other: a workspace each would hold as many times what one call takes."""
    first = lrsa.PagedCache(P, 5, device="cpu")
    layers = [first] + [lrsa.PagedCache(p, 5, device="cpu", beside=first) for p in (P, lrsa.Params(1, 16, 4, 900, 64, 100, 30, 3))]
    assert len({x.ws.data_ptr() for x in layers}) == 1 and len({x.k_pages.data_ptr() for x in layers}) == 3
    for i, cache in enumerate(layers[:2]):
        cache.append(**good(cache, 20000 * (i + 1))[0], stream=STREAM)
        assert all(x.ws is cache.ws and x._old is cache._old for x in layers)
        assert calls[-1][1][25] == cache.ws.data_ptr()
    layers[0].attend(**good(layers[0])[1], max_new=6, stream=STREAM)
    assert calls[-1][1][31] == layers[2].ws.data_ptr() and calls[-1][1][32] == layers[2].ws.numel()
    alone = lrsa.PagedCache(P, 5, device="cpu")
    assert alone.ws is not first.ws
    a, b = pickle.loads(pickle.dumps(layers[:2]))
    assert a.ws is b.ws and a.ws.data_ptr() != first.ws.data_ptr()
    for other in (lrsa.PagedCache(P, 5, device="cpu"), None):
        if other is not None:
            other.ws = other.ws.to("meta")
        with pytest.raises(lrsa.LrsaError):
            lrsa.PagedCache(P, 5, device="cpu", beside=other or object())


@pytest.mark.parametrize("p", [P, lrsa.Params(1, 4, 2, 300, 64, 7, 3, 0), lrsa.Params(1, 4, 2, 300, 64, 16, 16, 40)])
def test_room_is_where_a_window_more_is_condensed(p):
    cache = lrsa.PagedCache(p, 5, device="cpu")
    n = torch.arange(250, dtype=torch.int32)
    room = cache.room(n)
    assert room.dtype is torch.int32
    for a, r in zip(n.tolist(), room.tolist()):
        assert r >= 1 and ref.cut(p, a + r - 1) == ref.cut(p, a) and ref.cut(p, a + r) == ref.cut(p, a) + 1


def test_a_cache_that_was_saved_with_a_workspace_of_its_own_works(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    state = cache.__getstate__()
    ws = torch.full_like(state.pop("_space").ws, 255)
    again = lrsa.PagedCache.__new__(lrsa.PagedCache)
    again.__setstate__({**state, "ws": ws, "_old": []})
    assert again.ws.numel() == ws.numel() and (again.ws[:256] == 0).all() and again._old == []
    again.append(**good(again)[0], stream=STREAM)
    assert calls[-1][1][25] == again.ws.data_ptr() and calls[-1][1][5] == again.k_pages.data_ptr()


def test_rotations_whose_outputs_lie_over_other_tensors():
    """In place is the same tensor; a part of it, or another of the call's tensors, would be read after it was written."""
    import ctypes
    from tests.test_paged_abi import AT, rope
    q, k = 8 * 4000 * 128 * 2, 2 * 4000 * 128 * 2      # bytes
    K, QO, KO = AT + (1 << 30), AT + (2 << 30), AT + (3 << 30)
    r = rope()
    call = lambda *at: lrsa.lib().lrsa_rotate(P.ref(), *at, ctypes.byref(r), None, 0, None)
    for at in ((AT, K, AT + 256, KO), (AT, K, AT - 16, KO), (AT, K, AT + q - 16, KO), (AT, K, QO, K + 16), (AT, K, QO, K - k + 16),
               (AT, K, K, KO), (AT, K, K - q + 16, KO), (AT, K, QO, AT), (AT, K, QO, AT + q - 16), (AT, K, QO, QO), (AT, K, QO, QO + q - 16),
               (AT, AT, AT, KO), (AT, AT + 16, QO, AT + 16 + k - 16), (AT, None, AT + 16, None), (None, K, None, K + 16)):
        assert call(*at) == INVALID, at

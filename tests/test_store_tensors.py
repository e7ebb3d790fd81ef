"""Tensors of a KVStore that were replaced: the next call takes them, or refuses before the library sees their addresses.
On the CPU, with a library that records its calls."""
import copy
import pickle

import pytest
import torch

from paper_2506_11498_b200 import build as lib_build
from paper_2506_11498_b200 import lrsa

P = lrsa.Params(1, 4, 2, 1000, 128, 128, 32, 4)
TENSORS = ("k_list", "v_list", "k_scale", "v_scale", "k_recent", "v_recent", "weight", "idx")
STREAM = type("S", (), {"cuda_stream": 0})


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def calls(monkeypatch):
    lrsa.lib()
    rec = Recorder()
    monkeypatch.setattr(lrsa, "_call", rec)
    monkeypatch.setattr(lrsa, "_device", lambda where, name, t: t.get_device())
    return rec.calls


def uses(store):
    """The three calls on a store."""
    k, q = torch.zeros(1, 2, 1, 128, dtype=torch.bfloat16), torch.zeros(1, 4, 128, dtype=torch.bfloat16)
    store.n_tokens = 500
    return (lambda: store.append(k, k, stream=STREAM), lambda: store.decode(q, stream=STREAM), lambda: store.rows(stream=STREAM))


def bad_ones(t):
    yield None
    yield [0.0]
    yield t[:, :, :-1].contiguous()                     # too short
    yield t[:, :, :-1]                                  # a view of the right memory, of another shape
    yield t.flatten()
    yield t.to(torch.float64)
    yield torch.zeros(t.shape[:2] + (2 * t.shape[2],) + t.shape[3:], dtype=t.dtype)[:, :, ::2]      # strided
    if t.shape[1] > 1:
        yield t[:, :1].expand_as(t)
    yield t.to("meta")


@pytest.mark.parametrize("name", TENSORS)
@pytest.mark.parametrize("used", [False, True], ids=["fresh", "used"])
def test_replaced_by_what_does_not_fit(calls, name, used):
    n = sum(1 for _ in bad_ones(getattr(lrsa.KVStore(P, block=32, device="cpu"), name)))
    for which in range(n):
        store = lrsa.KVStore(P, block=32, device="cpu")
        todo = uses(store)
        if used:
            [call() for call in todo]
            store.n_tokens = 500
        for x in list(bad_ones(getattr(store, name)))[which:which + 1]:
            setattr(store, name, x)
        del calls[:]
        for call in todo:
            with pytest.raises(lrsa.LrsaError) as e:
                call()
            assert e.value.status == 1 and name in str(e.value)
        assert not calls and store.n_tokens == 500


@pytest.mark.parametrize("name", TENSORS)
def test_changed_in_place(calls, name):
    """The tensor object is the same, its memory is not."""
    store = lrsa.KVStore(P, block=32, device="cpu")
    todo = uses(store)
    [call() for call in todo]
    store.n_tokens = 500
    del calls[:]
    old = getattr(store, name).data_ptr()
    for _ in range(3):     # (an allocator may hand out a dropped block again: not one that a store was last looked at with)
        getattr(store, name).data = torch.zeros(1, 2, 1, dtype=getattr(store, name).dtype)
        assert getattr(store, name).data_ptr() != old
        for call in todo:
            with pytest.raises(lrsa.LrsaError) as e:
                call()
            assert e.value.status == 1 and name in str(e.value)
    assert not calls
    store = lrsa.KVStore(P, block=32, device="cpu")
    todo = uses(store)
    [call() for call in todo]
    del calls[:]
    getattr(store, name).untyped_storage().resize_(16)
    for call in todo:
        with pytest.raises(lrsa.LrsaError):
            call()
    assert not calls


def test_replaced_by_its_like(calls):
    store = lrsa.KVStore(P, block=32, device="cpu")
    todo = uses(store)
    [call() for call in todo]
    del calls[:]
    for name in TENSORS:
        setattr(store, name, getattr(store, name).clone())
    [call() for call in todo]
    assert [name for name, _ in calls] == ["store_append", "store_decode", "store_rows"]
    for _, args in calls:
        assert args[1:4] == (1, 32, 1) and args[4:12] == tuple(getattr(store, name).data_ptr() for name in TENSORS)
    for name in TENSORS:                                 # in place, by as much
        getattr(store, name).data = getattr(store, name).clone()
    del calls[:]
    [call() for call in todo]
    for _, args in calls:
        assert args[4:12] == tuple(getattr(store, name).data_ptr() for name in TENSORS)


def test_what_a_store_without_scales_and_weights_takes(calls):
    store = lrsa.KVStore(P, dtype=torch.bfloat16, block=32, keep="lag", device="cpu")
    todo = uses(store)
    [call() for call in todo]
    assert all(args[6] is None and args[7] is None and args[10] is None for _, args in calls)
    for name in ("k_scale", "v_scale", "weight"):
        setattr(store, name, torch.zeros(1, 2, 6))
        for call in todo:
            with pytest.raises(lrsa.LrsaError) as e:
                call()
            assert e.value.status == 1
        setattr(store, name, None)
    [call() for call in todo]


@pytest.mark.parametrize("change", [dict(dtype=torch.bfloat16), dict(keep="lag"), dict(block=16), dict(ws=torch.zeros(8)),
                                    dict(params=lrsa.Params(2, 4, 2, 1000, 128, 128, 32, 4)), dict(params=lrsa.Params(1, 8, 2, 1000, 128, 128, 32, 4)),
                                    dict(params=lrsa.Params(1, 4, 2, 2000, 128, 128, 32, 4)), dict(params=lrsa.Params(1, 4, 2, 1000, 128, 64, 32, 4))],
                         ids=lambda c: "_".join(c))
def test_what_a_store_was_made_with_stays(calls, change):
    store = lrsa.KVStore(P, block=32, device="cpu")
    todo = uses(store)
    [call() for call in todo]
    store.n_tokens = 500
    del calls[:]
    for name, value in change.items():
        setattr(store, name, value)
    for call in todo:
        with pytest.raises(lrsa.LrsaError) as e:
            call()
        assert e.value.status == 1
    assert not calls


@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda s: pickle.loads(pickle.dumps(s))], ids=["copy", "deepcopy", "pickle"])
def test_copies(calls, how):
    store = lrsa.KVStore(P, dtype=torch.int8, block=32, device="cpu")     # (8-bit floats do not go through a plain pickle)
    [call() for call in uses(store)]
    other = how(store)
    del calls[:]
    [call() for call in uses(other)]
    for _, args in calls:
        assert args[4:12] == tuple(getattr(other, name).data_ptr() for name in TENSORS)
    other.k_list = other.k_list[:, :, :5]
    del calls[:]
    for call in uses(other):
        with pytest.raises(lrsa.LrsaError):
            call()
    assert not calls

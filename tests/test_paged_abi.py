"""The paged cache and the rotation on the CPU: what the library and the binding refuse before anything is launched, the shape of the page table,
and what survives a pickle."""
import ctypes
import pickle

import pytest
import torch

from paper_2506_11498_b200 import build as lib_build
from paper_2506_11498_b200 import lrsa
from tests import paged_reference as ref

P = lrsa.Params(1, 8, 2, 4000, 128, 128, 40, 5)
OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3
AT = 0x7f0000000000     # an address that nobody touches: every call here is refused


@pytest.fixture(scope="module", autouse=True)
def _built():
    lib_build.build()


def shape(p=P, page=64, n_seqs=4, n_new=16, max_new=4):
    out = ctypes.c_int32(-1), ctypes.c_int32(-1), ctypes.c_size_t(0)
    rc = lrsa.lib().lrsa_paged_shape(p.ref(), page, n_seqs, n_new, max_new, *(ctypes.byref(x) for x in out))
    return rc, *(x.value for x in out)


def with_(p, **kw):
    return lrsa.Params(**{**{k: getattr(p, k) for k in p.__dataclass_fields__}, **kw})


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("p", [P, lrsa.Params(1, 4, 4, 700, 64, 77, 19, 0), lrsa.Params(1, 4, 4, 90, 64, 77, 19, 33)])
def test_table(p, page):
    rc, width, cap, ws = shape(p, page)
    sinks, ring, kept = ref.pages_of(p, page)
    assert (rc, cap) == (OK, ref.cut(p, p.seq_len)) and width == sinks + 2 * ring + cap * kept and ws >= 256
    cache = lrsa.PagedCache(p, 3, page=page, device="cpu")
    assert (cache.table_width, cache.w_cap) == (width, cap)
    for n in (0, 1, p.n_sink, p.n_sink + 1, min(p.seq_len, p.n_sink + p.lag + 1), p.seq_len):
        want = {ref.place(p, page, x)[0] for x in range(n)}
        want |= {ref.kept_place(p, page, w, j)[0] for w in range(ref.cut(p, n)) for j in range(p.top_k)}
        cols = cache.columns(n)
        assert sorted(cols) == sorted(want) and len(set(cols)) == len(cols)
        assert all(0 <= c < width for c in cols)


def test_workspace_grows_with_the_call():
    sizes = [shape(n_seqs=s, n_new=n, max_new=m)[3] for s, n, m in ((1, 0, 0), (1, 1, 1), (4, 64, 32), (4, 256, 64), (64, 256, 64))]
    assert sizes == sorted(sizes) and sizes[0] == 256
    assert shape(n_seqs=1, n_new=1000, max_new=0)[3] >= 1000 * 2 * 128 * 2


@pytest.mark.parametrize("change, want", [
    (dict(page=0), UNSUPPORTED), (dict(page=48), UNSUPPORTED), (dict(page=256), UNSUPPORTED), (dict(n_seqs=-1), INVALID),
    (dict(n_new=-1), INVALID), (dict(max_new=-1), INVALID), (dict(p=with_(P, n_dense_prev=0)), UNSUPPORTED),
    (dict(p=with_(P, cu_seqlens=(0, 2000, 4000))), UNSUPPORTED), (dict(p=with_(P, head_dim=96)), UNSUPPORTED),
    (dict(p=with_(P, top_k=129)), INVALID)])
def test_shapes_that_are_refused(change, want):
    assert shape(**change)[0] == want


def paged(**kw):
    s = dict(page=64, n_pages=100, n_seqs=4, table_width=shape()[1], k_pages=AT, v_pages=AT, table=AT, n_tokens=AT)
    s.update(kw)
    return lrsa.lrsa_paged_t(**s)


def rows(data=AT, head=128, token=1024):
    return lrsa.lrsa_rows_t(data, head, token)


def rope(**kw):
    s = dict(cos=AT, sin=AT, n_pos=4096, dim=128, interleaved=0, reserved=0)
    s.update(kw)
    return lrsa.lrsa_rope_t(**s)


def append(p=P, cache=None, k=None, v=None, n_rows=16, cu=AT, n_new=16, idx=None, r=None, kept=None, ws=AT, ws_bytes=1 << 30):
    by = ctypes.byref
    return lrsa.lib().lrsa_paged_append(p.ref(), by(cache or paged()), by(k or rows()), by(v or rows()), n_rows, cu, n_new, idx,
                                        by(r or rope()), kept, ws, ws_bytes, None)


def attend(p=P, cache=None, q=None, k=None, v=None, o=None, cu=AT, n_new=16, max_new=4, parent=None, r=None, lse=AT, ws=AT, ws_bytes=1 << 30):
    by = ctypes.byref
    return lrsa.lib().lrsa_paged_attend(p.ref(), by(cache or paged()), by(q or rows()), by(k or rows()), by(v or rows()), cu, n_new, max_new,
                                        parent, by(r or rope()), by(o or rows()), lse, ws, ws_bytes, None)


CACHES = [(dict(page=24), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(n_seqs=0), INVALID), (dict(table_width=1), INVALID),
          (dict(k_pages=None), INVALID), (dict(v_pages=None), INVALID), (dict(table=None), INVALID), (dict(n_tokens=None), INVALID),
          (dict(k_pages=AT + 8), INVALID), (dict(v_pages=AT + 2), INVALID), (dict(table=AT + 2), INVALID), (dict(n_tokens=AT + 1), INVALID)]
ROPES = [dict(cos=AT + 4), dict(sin=AT + 8), dict(sin=None), dict(cos=None), dict(n_pos=0), dict(dim=0), dict(dim=24), dict(dim=144),
         dict(interleaved=2), dict(reserved=1)]
BAD_ROWS = [rows(None), rows(AT + 8), rows(head=4), rows(token=1020)]


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change, want", CACHES)
def test_caches_that_are_refused(call, change, want):
    assert call(cache=paged(**change)) == want


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change", ROPES)
def test_ropes_that_are_refused(call, change):
    assert call(r=rope(**change)) == INVALID
    r = rope(**change)
    assert lrsa.lib().lrsa_rotate(P.ref(), AT, AT, AT, AT, ctypes.byref(r), AT, 0, None) == INVALID


@pytest.mark.parametrize("call, name", [(append, "k"), (append, "v"), (attend, "q"), (attend, "k"), (attend, "v"), (attend, "o")])
@pytest.mark.parametrize("bad", range(len(BAD_ROWS)))
def test_rows_that_are_refused(call, name, bad):
    assert call(**{name: BAD_ROWS[bad]}) == INVALID


def test_other_arguments_that_are_refused():
    assert append(cu=None) == append(n_new=-1) == append(n_rows=-1) == append(n_new=17) == append(idx=AT, n_rows=0) == INVALID
    assert append(idx=AT + 2) == append(kept=AT + 1) == append(cu=AT + 2) == append(ws=None) == append(ws=AT + 128) == INVALID
    assert append(ws_bytes=255) == SMALL
    assert append(n_rows=1000, n_new=1000, ws_bytes=256) == SMALL       # the rotated keys of a prompt
    assert append(p=with_(P, lag=25500, seq_len=100000), cache=paged(table_width=shape(with_(P, lag=25500, seq_len=100000))[1])) == UNSUPPORTED
    assert attend(cu=None) == attend(n_new=-1) == attend(max_new=0) == attend(parent=AT + 2) == attend(lse=AT + 2) == INVALID
    assert attend(ws=None) == attend(ws=AT + 64) == attend(cu=AT + 1) == INVALID
    assert attend(max_new=129) == UNSUPPORTED
    assert attend(ws_bytes=shape()[3] - 1) == SMALL
    assert append(p=with_(P, n_dense_prev=0)) == attend(p=with_(P, n_dense_prev=0)) == UNSUPPORTED


def test_rotations_that_are_refused():
    def call(p=P, q=AT, k=AT, qo=AT, ko=AT, r=None, pos=None, inverse=0):
        r = r or rope()
        return lrsa.lib().lrsa_rotate(p.ref(), q, k, qo, ko, ctypes.byref(r), pos, inverse, None)
    assert call(q=None, k=None, qo=None, ko=None) == call(q=None) == call(ko=None) == call(q=AT + 8) == call(ko=AT + 2) == INVALID
    assert call(inverse=2) == call(pos=AT + 2) == INVALID
    assert call(r=rope(n_pos=3999)) == INVALID                                     # the last position is not in the tables
    assert call(with_(P, cu_seqlens=(0, 1000, 4000)), r=rope(n_pos=2999)) == INVALID
    assert lrsa.lib().lrsa_rotate(P.ref(), AT, AT, AT, AT, None, None, 0, None) == INVALID


# ---- the binding ----
STREAM = type("S", (), {"cuda_stream": 0})


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


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def good(cache, T=6):
    """Arguments of the two calls, three sequences."""
    table, n, cu = i32(3, cache.table_width), i32(3), i32(4)
    r = lrsa.Rope(torch.zeros(64, 64), torch.zeros(64, 64))
    return (dict(k_new=bf(2, T, 128), v_new=bf(T, 2, 128).transpose(0, 1), table=table, n_tokens=n, cu_new=cu, rows=i32(T), rope=r,
                 kept=i32(3, 2, cache.w_cap, 40)),
            dict(q=bf(T, 8, 128).transpose(0, 1), k=bf(2, T, 128), v=bf(2, T, 128), table=table, n_tokens=n, cu_new=cu, parent=i32(T), rope=r))


def test_calls_that_are_taken(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    for a, b in (good(cache), good(cache, 1), good(cache, 0)):
        cache.append(**a, stream=STREAM)
        o, lse = cache.attend(**b, stream=STREAM)
        assert o.shape == b["q"].shape and lse.shape == o.shape[:2]
    fused = bf(6, 12 * 128)                  # the projections' output: queries, keys, values of a token side by side
    q, k, v = (x.unflatten(1, (-1, 128)).transpose(0, 1) for x in fused.split((8 * 128, 2 * 128, 2 * 128), 1))
    a, b = good(cache)
    o, _ = cache.attend(**{**b, "q": q, "k": k, "v": v}, stream=STREAM)
    assert o.stride() == (128, 1024, 1)
    cache.append(**{**a, "k_new": k[:1].expand(2, -1, -1), "v_new": v}, stream=STREAM)
    assert [c[0] for c in calls] == ["paged_append", "paged_attend"] * 3 + ["paged_attend", "paged_append"]
    kinds = {"paged_append": 28, "paged_attend": 34}
    assert all(len(c[1]) == kinds[c[0]] for c in calls)
    at = calls[-2][1]
    assert (at[9], at[10], at[11]) == (fused.data_ptr(), 128, 1536) and at[14] == 1536


@pytest.mark.parametrize("name, make", [
    ("k_new", lambda: bf(2, 6, 64)), ("k_new", lambda: bf(3, 6, 128)), ("k_new", lambda: bf(2, 6, 128).float()), ("k_new", lambda: bf(2, 768)),
    ("k_new", lambda: bf(2, 6, 256)[..., ::2]), ("k_new", lambda: bf(2, 6, 132)[..., 4:]), ("v_new", lambda: bf(2, 5, 128)),
    ("v_new", lambda: bf(2, 6, 130)[..., :128]), ("table", lambda: i32(3, 5)), ("table", lambda: i32(3)), ("table", lambda: i32(3, 400).long()),
    ("n_tokens", lambda: i32(4)), ("n_tokens", lambda: torch.zeros(3)), ("cu_new", lambda: i32(3)), ("cu_new", lambda: i32(8)[::2]),
    ("rows", lambda: i32(6).long()), ("rows", lambda: i32(2, 3)), ("kept", lambda: i32(3, 2, 1, 40)), ("kept", lambda: bf(3, 2, 29, 40))])
def test_appends_that_are_refused(calls, name, make):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    with pytest.raises(lrsa.LrsaError) as e:
        cache.append(**{**good(cache)[0], name: make()}, stream=STREAM)
    assert e.value.status == INVALID and not calls


@pytest.mark.parametrize("name, make", [
    ("q", lambda: bf(7, 6, 128)), ("q", lambda: bf(8, 6, 128).half()), ("q", lambda: bf(8, 128)), ("k", lambda: bf(2, 5, 128)), ("v", lambda: bf(1, 6, 128)),
    ("v", lambda: bf(2, 128, 6).transpose(1, 2)), ("parent", lambda: i32(5)), ("parent", lambda: i32(6).long()), ("o", lambda: bf(8, 5, 128)),
    ("o", lambda: bf(8, 1, 128).expand(8, 6, 128)), ("o", lambda: bf(1, 6, 128).expand(8, 6, 128)), ("lse", lambda: torch.zeros(6, 8)),
    ("lse", lambda: bf(8, 6)), ("table", lambda: i32(2, 2)), ("cu_new", lambda: i32(5))])
def test_attends_that_are_refused(calls, name, make):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    with pytest.raises(lrsa.LrsaError) as e:
        cache.attend(**{**good(cache)[1], name: make()}, stream=STREAM)
    assert e.value.status == INVALID and not calls


@pytest.mark.parametrize("name", ["k_pages", "v_pages"])
@pytest.mark.parametrize("used", [False, True], ids=["fresh", "used"])
def test_pages_that_were_replaced(calls, name, used):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    a, b = good(cache)
    if used:
        cache.append(**a, stream=STREAM)
    t = getattr(cache, name)
    for bad in (t[:4], t.float(), t.transpose(1, 2), bf(*t.shape[:3], 256)[..., ::2], t.flatten(), t.to("meta"), None):
        setattr(cache, name, bad)
        n = len(calls)
        for call in (lambda: cache.append(**a, stream=STREAM), lambda: cache.attend(**b, stream=STREAM)):
            with pytest.raises(lrsa.LrsaError):
                call()
        assert len(calls) == n
    new = torch.ones_like(t)
    setattr(cache, name, new)
    cache.attend(**b, stream=STREAM)
    assert new.data_ptr() in calls[-1][1]


def test_a_workspace_that_was_outgrown_stays_where_it_was(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    first = cache.ws
    a, b = good(cache)
    cache.attend(**b, max_new=6, stream=STREAM)      # 24 rows of a KV head: another kernel, with more to keep
    assert cache.ws is not first and any(x is first for x in cache._old)
    small = cache.ws
    cache.attend(**b, max_new=1, stream=STREAM)
    assert cache.ws is small and calls[-1][1][32] == small.numel()


def test_workspaces_of_growing_calls_take_little(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    for T in range(4000, 60000, 4000):               # prompts, each longer than the last
        cache.append(**good(cache, T)[0], stream=STREAM)
        assert cache.ws.numel() >= cache.workspace_bytes(3, T, 0)
    assert cache._old and cache.ws.numel() <= 2 * cache.workspace_bytes(3, T, 0)
    assert sum(x.numel() for x in cache._old) <= cache.ws.numel()


def test_ropes():
    r = lrsa.Rope.of_base(10000.0, 64, 100, device="cpu")
    cos, sin = ref.angles(100, 64)
    assert torch.equal(r.cos, torch.from_numpy(cos)) and torch.equal(r.sin, torch.from_numpy(sin))
    again = pickle.loads(pickle.dumps(lrsa.Rope(r.cos, r.sin, True)))
    assert again.interleaved and torch.equal(again.cos, r.cos) and again._args[0] == again.cos.data_ptr()
    for cos, sin in ((r.cos.double(), r.sin), (r.cos, r.sin[:50]), (r.cos[:, :12], r.sin[:, :12]), (r.cos.flatten(), r.sin.flatten()),
                     (r.cos[:, :4].contiguous(), r.sin[:, :4].contiguous()), (r.cos[:0], r.sin[:0])):
        with pytest.raises(lrsa.LrsaError):
            lrsa.Rope(cos, sin)


def test_a_pickled_cache_works(calls):
    cache = lrsa.PagedCache(P, 5, device="cpu")
    cache.append(**good(cache)[0], stream=STREAM)
    again = pickle.loads(pickle.dumps(cache))
    again.append(**good(again)[0], stream=STREAM)
    assert calls[-1][1][5] == again.k_pages.data_ptr() != cache.k_pages.data_ptr()


@pytest.mark.parametrize("change", [dict(Q=bf(1, 8, 4000, 64)), dict(K=bf(1, 3, 4000, 128)), dict(Q=None, K=None), dict(K=None, K_out=bf(1, 2, 4000, 128)),
                                    dict(Q_out=bf(1, 8, 3999, 128)), dict(positions=i32(3999)), dict(positions=i32(4000).long())])
def test_rotations_that_the_binding_refuses(calls, change):
    args = dict(Q=bf(1, 8, 4000, 128), K=bf(1, 2, 4000, 128), rope=lrsa.Rope(torch.zeros(4000, 64), torch.zeros(4000, 64)))
    with pytest.raises(lrsa.LrsaError) as e:
        lrsa.lrsa_rotate(P, **{**args, **change}, stream=STREAM)
    assert e.value.status == INVALID and not calls
